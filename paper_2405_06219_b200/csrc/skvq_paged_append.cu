// skvq_paged_append and skvq_paged_read: rotated, reordered, 4-bit quantized rows into pages, and back.
//
// A warp owns one row (one token of one KV head, keys or values).  A lane holds D/32 neighbouring channels: the row is read
// coalesced, rotated (the partner channel comes through shared memory), put into shared memory, and gathered from there in
// stored order; group extremes are reduced by shuffles over the G/(D/32) lanes of a group.
// The quantizer arithmetic is explicitly rounded fp32: codes and parameters do not depend on compiler contraction.
#include "skvq_paged.cuh"

namespace skvq {
namespace {

constexpr int kWarpsPerCta = 8;      // even: warps 0, 2, ... take keys, 1, 3, ... values
constexpr int kTokensPerWarp = 8;

struct AppendIo {
    const void *k, *v;
    int64_t k_stride, v_stride;
};

template <typename T, int D>
__global__ void __launch_bounds__(kWarpsPerCta * 32) paged_append_kernel(const __grid_constant__ PagedArgs a, AppendIo io)
{
    constexpr int C = D / 32;      // channels per lane
    __shared__ __align__(16) T rows[kWarpsPerCta][2][D];
    const int b = blockIdx.z, h = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    PagedSeq seq;
    if (!paged_sequence(a, b, true, seq)) {
        if (blockIdx.x == 0 && h == 0 && threadIdx.x == 0) set_status(a.c.status, SKVQ_STATUS_BAD_BATCH);
        return;
    }
    const int pairs = (blockDim.x >> 5) >> 1;
    const int i0 = blockIdx.x * pairs * kTokensPerWarp + (warp >> 1) * kTokensPerWarp;
    if (i0 >= seq.n) return;
    const bool is_v = warp & 1;
    const skvq_paged_config &cfg = a.cfg;
    const int G = cfg.group_size, P = cfg.page_tokens;
    const int lanes_per_group = G / C, g = lane / lanes_per_group;
    int idx[C];
    const int32_t *reorder = is_v ? a.c.reorder_v : a.c.reorder_k;
#pragma unroll
    for (int j = 0; j < C; ++j) idx[j] = reorder ? reorder[h * D + lane * C + j] & (D - 1) : lane * C + j;
    const float *alphas = is_v ? a.c.alpha_v : a.c.alpha_k;
    const float alpha = alphas ? alphas[h * a.ng + g] : 1.0f;
    const bool rot = !is_v && a.rope.table;
    const int half = a.rope.rot_dim / 2;
    T *raw = rows[warp][0], *turned = rows[warp][1];
    const T *src = static_cast<const T *>(is_v ? io.v : io.k) + (int64_t)h * D + lane * C;
    const int64_t stride = is_v ? io.v_stride : io.k_stride;
    struct alignas(sizeof(T) * C) Piece { T v[C]; };

    for (int i = i0; i < min(i0 + kTokensPerWarp, seq.n); ++i) {
        const int t = seq.len - seq.n + i;
        Piece p = *reinterpret_cast<const Piece *>(src + (seq.row0 + i) * stride);
        if (rot) {
            *reinterpret_cast<Piece *>(raw + lane * C) = p;
            __syncwarp();
            const float2 *table = static_cast<const float2 *>(a.rope.table) + (int64_t)t * half;
#pragma unroll
            for (int j = 0; j < C; ++j) {
                const int c = lane * C + j;
                if (c < a.rope.rot_dim) {
                    const bool second = a.rope.interleaved ? c & 1 : c >= half;
                    const int pair = a.rope.interleaved ? c >> 1 : (second ? c - half : c);
                    const int partner = a.rope.interleaved ? c ^ 1 : (second ? c - half : c + half);
                    const float2 cs = table[pair];
                    const float own = Elem<T>::to_float(p.v[j]), other = Elem<T>::to_float(raw[partner]);
                    p.v[j] = Elem<T>::from_float(second ? rotate_second(other, own, cs.x, cs.y) : rotate_first(own, other, cs.x, cs.y));
                }
            }
        }
        *reinterpret_cast<Piece *>(turned + lane * C) = p;
        __syncwarp();
        float x[C];
#pragma unroll
        for (int j = 0; j < C; ++j) { p.v[j] = turned[idx[j]]; x[j] = Elem<T>::to_float(p.v[j]); }
        __syncwarp();

        float mn = x[0], mx = x[0];
#pragma unroll
        for (int j = 1; j < C; ++j) { mn = fminf(mn, x[j]); mx = fmaxf(mx, x[j]); }
        for (int m = 1; m < lanes_per_group; m <<= 1) {
            mn = fminf(mn, __shfl_xor_sync(0xffffffffu, mn, m));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, m));
        }
        const float lo = __fadd_rn(__fmul_rn(alpha, mn), 0.0f), hi = __fadd_rn(__fmul_rn(alpha, mx), 0.0f);
        const __half2 hz = __halves2half2(__float2half_rn(__fmul_rn(__fsub_rn(hi, lo), 1.0f / 15.0f)), __float2half_rn(lo));
        const float hf = __low2float(hz), zf = __high2float(hz);
        uint32_t codes = 0u;
#pragma unroll
        for (int j = 0; j < C; ++j) {
            float c = hf != 0.0f ? rintf(__fdiv_rn(__fsub_rn(x[j], zf), hf)) : 0.0f;
            c = fminf(fmaxf(c, 0.0f), 15.0f);
            codes |= (uint32_t)(int)c << (4 * j);
        }
        const int page = a.batch.page_table[(int64_t)b * a.batch.max_pages + t / P];
        if (page < 0 || page >= cfg.n_pages) {
            if (lane == 0) set_status(a.c.status, SKVQ_STATUS_BAD_PAGE);
            continue;
        }
        const int64_t row = ((int64_t)page * cfg.n_kv_heads + h) * P + t % P;
        uint8_t *out = static_cast<uint8_t *>(is_v ? a.c.v_codes : a.c.k_codes) + row * (D / 2);
        if constexpr (C == 4) reinterpret_cast<uint16_t *>(out)[lane] = (uint16_t)codes;
        else out[lane] = (uint8_t)codes;
        if (lane % lanes_per_group == 0)
            static_cast<__half2 *>(is_v ? a.c.v_meta : a.c.k_meta)[row * a.ng + g] = hz;
        if (cfg.window > 0 && t >= seq.len - cfg.ring_tokens) {
            T *win = static_cast<T *>(is_v ? a.c.v_win : a.c.k_win) +
                     (((int64_t)seq.slot * cfg.n_kv_heads + h) * cfg.ring_tokens + t % cfg.ring_tokens) * D;
            *reinterpret_cast<Piece *>(win + lane * C) = p;
        }
    }
}

struct ReadIo {
    void *k, *v;
    int64_t k_stride, v_stride;
    int window;
};

template <typename T, int D>
__global__ void __launch_bounds__(kWarpsPerCta * 32) paged_read_kernel(const __grid_constant__ PagedArgs a, ReadIo io)
{
    constexpr int C = D / 32;
    __shared__ __align__(16) T rows[kWarpsPerCta][D];
    const int b = blockIdx.z, h = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    PagedSeq seq;
    if (!paged_sequence(a, b, true, seq)) {
        if (blockIdx.x == 0 && h == 0 && threadIdx.x == 0) set_status(a.c.status, SKVQ_STATUS_BAD_BATCH);
        return;
    }
    const int pairs = (blockDim.x >> 5) >> 1;
    const int i0 = blockIdx.x * pairs * kTokensPerWarp + (warp >> 1) * kTokensPerWarp;
    const bool is_v = warp & 1;
    T *dst = static_cast<T *>(is_v ? io.v : io.k);
    if (i0 >= seq.n || !dst) return;
    const skvq_paged_config &cfg = a.cfg;
    const int P = cfg.page_tokens, g = lane / (cfg.group_size / C);
    int idx[C];
    const int32_t *reorder = is_v ? a.c.reorder_v : a.c.reorder_k;
#pragma unroll
    for (int j = 0; j < C; ++j) idx[j] = reorder ? reorder[h * D + lane * C + j] & (D - 1) : lane * C + j;
    const int64_t stride = is_v ? io.v_stride : io.k_stride;
    dst += (int64_t)h * D + lane * C;
    T *turned = rows[warp];
    struct alignas(sizeof(T) * C) Piece { T v[C]; };

    for (int i = i0; i < min(i0 + kTokensPerWarp, seq.n); ++i) {
        const int t = seq.len - seq.n + i;
        Piece p;
        if (io.window && t >= seq.len - cfg.window) {
            const T *win = static_cast<const T *>(is_v ? a.c.v_win : a.c.k_win) +
                           (((int64_t)seq.slot * cfg.n_kv_heads + h) * cfg.ring_tokens + t % cfg.ring_tokens) * D;
            p = *reinterpret_cast<const Piece *>(win + lane * C);
        } else {
            const int page = a.batch.page_table[(int64_t)b * a.batch.max_pages + t / P];
            if (page < 0 || page >= cfg.n_pages) {
                if (lane == 0) set_status(a.c.status, SKVQ_STATUS_BAD_PAGE);
                continue;
            }
            const int64_t row = ((int64_t)page * cfg.n_kv_heads + h) * P + t % P;
            const uint8_t *in = static_cast<const uint8_t *>(is_v ? a.c.v_codes : a.c.k_codes) + row * (D / 2);
            uint32_t codes;
            if constexpr (C == 4) codes = reinterpret_cast<const uint16_t *>(in)[lane];
            else codes = in[lane];
            const __half2 hz = static_cast<const __half2 *>(is_v ? a.c.v_meta : a.c.k_meta)[row * a.ng + g];
            const float hf = __low2float(hz), zf = __high2float(hz);
#pragma unroll
            for (int j = 0; j < C; ++j)
                p.v[j] = Elem<T>::from_float(__fadd_rn(__fmul_rn(hf, (float)((codes >> (4 * j)) & 15u)), zf));
        }
#pragma unroll
        for (int j = 0; j < C; ++j) turned[idx[j]] = p.v[j];
        __syncwarp();
        *reinterpret_cast<Piece *>(dst + (seq.row0 + i) * stride) = *reinterpret_cast<const Piece *>(turned + lane * C);
        __syncwarp();
    }
}

// Grid of a warp-per-row kernel: tokens of the longest sequence, KV heads, sequences.  Steps of a few tokens get small CTAs.
dim3 row_grid(const PagedArgs &a, int &threads)
{
    int pairs = kWarpsPerCta / 2;
    while (pairs > 1 && (pairs / 2) * kTokensPerWarp >= a.batch.max_new) pairs /= 2;
    threads = pairs * 64;
    const int per = pairs * kTokensPerWarp;
    return dim3((a.batch.max_new + per - 1) / per, a.cfg.n_kv_heads, a.batch.n_seqs);
}

}  // namespace

cudaError_t launch_paged_append(const PagedArgs &a, const void *k, const void *v, int64_t k_stride, int64_t v_stride, cudaStream_t stream)
{
    int threads;
    const dim3 grid = row_grid(a, threads);
    const AppendIo io{k, v, k_stride, v_stride};
    const bool f16 = a.cfg.dtype == SKVQ_F16, d128 = a.cfg.head_dim == 128;
    if (f16 && d128) paged_append_kernel<__half, 128><<<grid, threads, 0, stream>>>(a, io);
    else if (f16) paged_append_kernel<__half, 64><<<grid, threads, 0, stream>>>(a, io);
    else if (d128) paged_append_kernel<__nv_bfloat16, 128><<<grid, threads, 0, stream>>>(a, io);
    else paged_append_kernel<__nv_bfloat16, 64><<<grid, threads, 0, stream>>>(a, io);
    count_launch();
    return cudaGetLastError();
}

cudaError_t launch_paged_read(const PagedArgs &a, int window, void *k, void *v, int64_t k_stride, int64_t v_stride, cudaStream_t stream)
{
    int threads;
    const dim3 grid = row_grid(a, threads);
    const ReadIo io{k, v, k_stride, v_stride, window};
    const bool f16 = a.cfg.dtype == SKVQ_F16, d128 = a.cfg.head_dim == 128;
    if (f16 && d128) paged_read_kernel<__half, 128><<<grid, threads, 0, stream>>>(a, io);
    else if (f16) paged_read_kernel<__half, 64><<<grid, threads, 0, stream>>>(a, io);
    else if (d128) paged_read_kernel<__nv_bfloat16, 128><<<grid, threads, 0, stream>>>(a, io);
    else paged_read_kernel<__nv_bfloat16, 64><<<grid, threads, 0, stream>>>(a, io);
    count_launch();
    return cudaGetLastError();
}

}  // namespace skvq
