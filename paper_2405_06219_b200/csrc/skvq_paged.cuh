// Private declarations of the paged cache and the rotation (shared by skvq_rope.cu, skvq_paged_*.cu).
#pragma once

#include <cuda_bf16.h>

#include "skvq_internal.cuh"

namespace skvq {

constexpr int kMaxPagedSeqs = 2048;
constexpr int kMaxPagedLen = 1 << 30;      // token numbers are ints, and kernels look some tiles past a sequence's end

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

// D/16 elements of the tensors' type: a lane's share of a row that sixteen lanes own.
template <typename T, int D> struct Row {
    static constexpr int C = D / 16;
    static constexpr int WORDS = C / 2;
    uint32_t w[WORDS];
    __device__ __forceinline__ void load(const T *p)
    {
        if constexpr (C == 8) { const uint4 v = *reinterpret_cast<const uint4 *>(p); w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w; }
        else { const uint2 v = *reinterpret_cast<const uint2 *>(p); w[0] = v.x; w[1] = v.y; }
    }
    __device__ __forceinline__ void store(T *p) const
    {
        if constexpr (C == 8) *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        else *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
    }
};
// Two elements in a register, as floats and back (rounded).
template <typename T> __device__ __forceinline__ float2 floats(uint32_t v);
template <> __device__ __forceinline__ float2 floats<__half>(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2 *>(&v)); }
template <> __device__ __forceinline__ float2 floats<__nv_bfloat16>(uint32_t v) { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u)); }
template <typename T> __device__ __forceinline__ uint32_t packed(float lo, float hi);
template <> __device__ __forceinline__ uint32_t packed<__half>(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <> __device__ __forceinline__ uint32_t packed<__nv_bfloat16>(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// Two fp32 in a 64-bit register: one instruction works on both, rounding each as the scalar form does.
__device__ __forceinline__ uint64_t pair(float a, float b)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpair(uint64_t v, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t pair_fma(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t pair_add(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// For products that are exact: the compiler contracts it with a sum that follows.
__device__ __forceinline__ uint64_t pair_mul(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// The two elements of a register as a pair of floats, and back (rounded).
template <typename T> __device__ __forceinline__ uint64_t pair_of(uint32_t v)
{
    const float2 f = floats<T>(v);
    return pair(f.x, f.y);
}
template <typename T> __device__ __forceinline__ uint32_t packed(uint64_t v)
{
    float lo, hi;
    unpair(v, lo, hi);
    return packed<T>(lo, hi);
}

// Rotates a lane's channels c0 .. c0 + C - 1 of a row; cs[j] = {cos, sin} of channel c0 + j.  `raw` is the row in shared memory, as read, for
// the partners of the half layout (interleaved pairs lie in one lane).  Rounded to T.
template <typename T, int D>
__device__ __forceinline__ void rotate_row(Row<T, D> &row, int c0, const float2 *cs, const T *raw, int rot_dim, bool interleaved)
{
    const int half = rot_dim / 2;
#pragma unroll
    for (int j = 0; j < Row<T, D>::C; j += 2) {
        const float2 x = floats<T>(row.w[j / 2]);
        float y0 = x.x, y1 = x.y;
        const int ca = c0 + j, cb = ca + 1;
        if (interleaved) {
            if (ca < rot_dim) {
                y0 = rotate_first(x.x, x.y, cs[j].x, cs[j].y);
                y1 = rotate_second(x.x, x.y, cs[j].x, cs[j].y);
            }
        } else {
            if (ca < rot_dim) {
                const float o = Elem<T>::to_float(raw[ca >= half ? ca - half : ca + half]);
                y0 = ca >= half ? rotate_second(o, x.x, cs[j].x, cs[j].y) : rotate_first(x.x, o, cs[j].x, cs[j].y);
            }
            if (cb < rot_dim) {
                const float o = Elem<T>::to_float(raw[cb >= half ? cb - half : cb + half]);
                y1 = cb >= half ? rotate_second(o, x.y, cs[j + 1].x, cs[j + 1].y) : rotate_first(x.y, o, cs[j + 1].x, cs[j + 1].y);
            }
        }
        row.w[j / 2] = packed<T>(y0, y1);
    }
}
// cos and sin of a lane's channels at position t ({1, 0} behind rot_dim).
template <int C>
__device__ __forceinline__ void load_angles(float2 (&cs)[C], const skvq_rope &rope, int t, int c0)
{
    const int half = rope.rot_dim / 2;
    const float2 *table = static_cast<const float2 *>(rope.table) + (int64_t)t * half;
#pragma unroll
    for (int j = 0; j < C; ++j) {
        const int c = c0 + j;
        cs[j] = make_float2(1.f, 0.f);
        if (c < rope.rot_dim) cs[j] = table[rope.interleaved ? c >> 1 : (c >= half ? c - half : c)];
    }
}

__device__ __forceinline__ void set_status(int32_t *status, int bits)
{
    if (status) atomicOr(status, bits);
}

struct PagedSeq {
    int len, n, row0, slot;     // tokens including the new ones, new ones, first packed row, ring slot
    int lq;                     // tokens below it are read from the pages, the others from the ring
};

// What sequence b asks for; false when its entries are out of range (the caller reports and skips it).
// `rows_within_len`: no more new tokens than the sequence is long (attention may have more rows).
__device__ __forceinline__ bool paged_sequence(const PagedArgs &a, int b, bool rows_within_len, PagedSeq &q)
{
    const skvq_paged_batch &p = a.batch;
    const int s0 = p.starts[b], s1 = p.starts[b + 1];
    q.len = p.lens[b];
    q.row0 = s0;
    q.n = s1 - s0;
    q.slot = p.slots ? p.slots[b] : b;
    q.lq = max(q.len - a.cfg.window, 0);
    if (p.ring_from) q.lq = max(q.lq, min(p.ring_from[b], q.len));
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

struct PagedWeightArgs {
    PagedArgs p;
    const void *q;
    const float *lse;
    const float *w_in;      // NULL: zeros
    float *w_out;
    int64_t q_stride;
    float sm_scale;
    int causal, last, capacity;
    uint8_t *ws;
};
size_t paged_weights_workspace_bytes(const skvq_paged_config &cfg, const skvq_paged_batch &batch, int last);
cudaError_t launch_paged_weights(const PagedWeightArgs &a, cudaStream_t stream);

constexpr int kMaxRingMoved = 8192;      // ring rows of a sequence that an eviction moves at most
struct PagedEvictArgs {
    PagedArgs p;
    skvq_paged_evict_args e;
    int max_kept;      // min(keep, max_len)
};
size_t paged_evict_workspace_bytes(const skvq_paged_batch &batch);
cudaError_t launch_paged_evict(const PagedEvictArgs &a, cudaStream_t stream);

}  // namespace skvq
