// Private declarations of the paged cache and the rotation (shared by skvq_rope.cu, skvq_paged_*.cu).
#pragma once

#include <cuda_bf16.h>

#include "skvq_internal.cuh"

namespace skvq {

constexpr int kMaxPagedSeqs = 2048;

// Everything the paged kernels need, by value.
struct PagedArgs {
    skvq_paged_config cfg;
    skvq_paged_cache c;
    skvq_paged_batch batch;
    skvq_rope rope;      // table == NULL: no rotation
    int ng;
};

template <typename T> struct Elem;
template <> struct Elem<__half> {
    static __device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
    static __device__ __forceinline__ __half from_float(float x) { return __float2half_rn(x); }
};
template <> struct Elem<__nv_bfloat16> {
    static __device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
    static __device__ __forceinline__ __nv_bfloat16 from_float(float x) { return __float2bfloat16_rn(x); }
};
template <> struct Elem<float> {
    static __device__ __forceinline__ float to_float(float x) { return x; }
    static __device__ __forceinline__ float from_float(float x) { return x; }
};

#ifdef __CUDACC__
// One channel of a rotated pair: x c - x2 s for the first channel of the pair, x c + x1 s for the second (sign = -1 / +1).
// The products are rounded before the sum: the result does not depend on compiler contraction, so a rotation done on its
// own and one fused into another kernel give the same bits.
__device__ __forceinline__ float rotate_first(float x1, float x2, float c, float s) { return __fsub_rn(__fmul_rn(x1, c), __fmul_rn(x2, s)); }
__device__ __forceinline__ float rotate_second(float x1, float x2, float c, float s) { return __fadd_rn(__fmul_rn(x2, c), __fmul_rn(x1, s)); }

__device__ __forceinline__ void set_status(int32_t *status, int bits)
{
    if (status) atomicOr(status, bits);
}

struct PagedSeq {
    int len, n, row0, slot;     // tokens including the new ones, new ones, first packed row, ring slot
};

// What sequence b asks for; false when its entries are out of range (the caller reports and skips it).
// `causal_only`: attention may have more rows than tokens.
__device__ __forceinline__ bool paged_sequence(const PagedArgs &a, int b, bool rows_within_len, PagedSeq &q)
{
    const skvq_paged_batch &p = a.batch;
    const int s0 = p.starts[b], s1 = p.starts[b + 1];
    q.len = p.lens[b];
    q.row0 = s0;
    q.n = s1 - s0;
    q.slot = p.slots ? p.slots[b] : b;
    bool ok = s0 >= 0 && s1 >= s0 && s1 <= p.n_tokens && q.n <= p.max_new && q.len >= 0 && q.len <= p.max_len;
    if (rows_within_len) ok = ok && q.n <= q.len;
    if (a.rope.table) ok = ok && q.len <= a.rope.n_positions;
    if (a.cfg.window > 0) ok = ok && q.slot >= 0 && q.slot < a.cfg.n_slots;
    return ok;
}
#endif

cudaError_t launch_paged_append(const PagedArgs &a, const void *k, const void *v, int64_t k_stride, int64_t v_stride, cudaStream_t stream);
cudaError_t launch_paged_read(const PagedArgs &a, int window, void *k, void *v, int64_t k_stride, int64_t v_stride, cudaStream_t stream);

struct PagedAttnArgs {
    PagedArgs p;
    const void *q;
    void *out;
    float *lse;
    int64_t q_stride, out_stride;
    float sm_scale;
    int causal, n_splits;
    float *ws;
};
size_t paged_workspace_bytes(const skvq_paged_config &cfg, const skvq_paged_batch &batch, int n_splits);
cudaError_t launch_paged_attention(const PagedAttnArgs &a, cudaStream_t stream);

}  // namespace skvq
