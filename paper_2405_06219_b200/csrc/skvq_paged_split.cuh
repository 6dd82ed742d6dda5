// What the two kernels of skvq_paged_attention share: which rows go where, the workspace of items that several CTAs share, the
// merge of their partials, chained launches.
#pragma once
#include "skvq_paged.cuh"

namespace skvq {

// Sequences with at most this many packed rows (new tokens * Hq/Hkv) per KV head go to the kernel for few rows, the others to the
// tcgen05 kernel.  Measured on 16 sequences of 1024 to 16384 tokens, 8 KV heads of 128, bf16, in a graph: 8 rows 62 us here; 16 rows 102 here,
// 209 there; 20 rows (a second item per KV head here) 158 here, 198 there; 24 rows 147 and 198; 32 rows 171 and 231.  So the kernel for few
// rows would take up to 32 rows faster; above 16 it has not been tested.
constexpr int kFewRows = 16;

// Workspace of a kernel: descriptor [n_slots][8] ints, then partials [n_slots][2][rows per item][D + 4] floats {o[D], m (log2
// units), l, pad}.  A CTA's run holds at most one item that it continues (partial 0) and one that it begins and does not finish
// (partial 1; then the descriptor says {1, first packed row, new tokens, KV head, item, number of partials}).
constexpr int kDescInts = 8;
__host__ __device__ constexpr int partial_stride(int D) { return D + 4; }

// Joins the partials; `lse_offset`: log2 of the factor that the probabilities carry.  `row_warps` warps share an item's rows.
cudaError_t launch_paged_merge(const PagedAttnArgs &a, int n_slots, int rows, int row_warps, float lse_offset, cudaStream_t stream);

size_t prefill_workspace_bytes(const skvq_paged_config &cfg, const skvq_paged_batch &batch);
cudaError_t launch_paged_prefill(const PagedAttnArgs &a, cudaStream_t stream);

// A launch that may start while its predecessor on the stream drains; every kernel launched so waits (griddepcontrol.wait) before
// it touches memory.
template <typename Kern, typename Args>
inline cudaError_t launch_chained(Kern kern, dim3 grid, int threads, size_t smem, cudaStream_t stream, const Args &args)
{
    cudaLaunchConfig_t lc = {};
    lc.gridDim = grid;
    lc.blockDim = dim3(threads);
    lc.dynamicSmemBytes = smem;
    lc.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = attr;
    lc.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&lc, kern, args);
    if (e == cudaSuccess) count_launch();
    return e;
}

}  // namespace skvq
