// skvq_paged_append and skvq_paged_read: rotated, reordered, 4-bit quantized rows into pages, and back.
//
// Sixteen lanes own a row (one token of one KV head, keys or values), D/16 neighbouring channels a lane; a warp works on two rows at
// a time: two tokens of the same head (bulk), or two heads of the same token (steps of few tokens, where latency counts), and walks
// over heads, so a token's angles stay in registers.  The row is read coalesced, rotated (partner channels come through shared
// memory), and gathered from shared memory in stored order; a group's extremes are reduced by shuffles.
// What bounds it is instructions, not bytes (about 90 per key row and lane group, 65 per value row): so min and max travel as one
// packed pair, and the code is formed without a division,
//   code = rint(d / h): t = fma(d, RN(1/h), 1.5 2^23) holds rint(d RN(1/h)); the remainder d - code h tells whether the quotient can be
//   near k + 0.5 (|remainder| >= h/2 (1 - 2^-18)); only then (ties included) the rows concerned divide.
// The quantizer arithmetic is explicitly rounded fp32: codes and parameters do not depend on compiler contraction.
#include "skvq_paged_split.cuh"

namespace skvq {
namespace {

constexpr int kRowWarps = 4;
constexpr int kRowThreads = kRowWarps * 32;
constexpr int kBulkTokens = 2 * kRowWarps;      // tokens of a CTA when they lie side by side

struct AppendIo {
    PagedArgs p;
    const void *k, *v;
    int64_t k_stride, v_stride;
    int heads;       // heads a CTA walks over
    int bulk;        // 1: half-warps take tokens; 0: heads of one token
};

template <typename T> __device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b);
template <> __device__ __forceinline__ uint32_t min2<__half>(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("min.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
template <> __device__ __forceinline__ uint32_t min2<__nv_bfloat16>(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("min.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// The row's position and place, or valid = false.
struct RowPlace {
    bool valid;
    int t, page;
};

template <typename T, int D, int NG, bool IS_V>
__device__ __forceinline__ void append_rows(const AppendIo &io, const PagedSeq &seq, int b, int i, int h_first, int h_step, int h_end, bool any, T *raw, T *turned)
{
    using R = Row<T, D>;
    constexpr int C = R::C, LANES = 16 / NG;      // lanes of a group
    const PagedArgs &a = io.p;
    const skvq_paged_config &cfg = a.cfg;
    const int sub = threadIdx.x & 15, P = cfg.page_tokens;
    const bool have = any && i < seq.n;
    const int t = seq.len - seq.n + i;
    int page = -1;
    if (have) {
        page = a.batch.page_table[(int64_t)b * a.batch.max_pages + t / P];
        if (page < 0 || page >= cfg.n_pages) {
            page = -1;
            if (sub == 0) set_status(a.c.status, SKVQ_STATUS_BAD_PAGE);
        }
    }
    const bool rot = !IS_V && a.rope.table;
    const int c0 = sub * C;
    const bool inter = a.rope.interleaved;
    float2 cs[IS_V ? 1 : C];
    if constexpr (!IS_V) {
        if (rot && have) load_angles(cs, a.rope, t, c0);
    }
    const T *src = static_cast<const T *>(IS_V ? io.v : io.k) + (int64_t)(seq.row0 + i) * (IS_V ? io.v_stride : io.k_stride) + c0;
    const int32_t *reorder = IS_V ? a.c.reorder_v : a.c.reorder_k;
    const float *alphas = IS_V ? a.c.alpha_v : a.c.alpha_k;
    const int64_t page_row = ((int64_t)page * cfg.n_kv_heads) * P + t % P;
    uint8_t *codes_pool = static_cast<uint8_t *>(IS_V ? a.c.v_codes : a.c.k_codes);
    uint32_t *meta_pool = static_cast<uint32_t *>(IS_V ? a.c.v_meta : a.c.k_meta);
    const bool keep = cfg.window > 0 && t >= seq.len - cfg.ring_tokens;
    const int ring = cfg.ring_tokens > 0 ? t % cfg.ring_tokens : 0;
    T *win = static_cast<T *>(IS_V ? a.c.v_win : a.c.k_win);

    R next;
#pragma unroll
    for (int k = 0; k < R::WORDS; ++k) next.w[k] = 0u;
    if (have && h_first < h_end) next.load(src + (int64_t)h_first * D);
    for (int h0 = h_first; __any_sync(0xffffffffu, h0 < h_end); h0 += h_step) {
        const bool here = have && h0 < h_end;
        const int h = min(h0, h_end - 1);
        int idx[C];
#pragma unroll
        for (int j = 0; j < C; j += 4) {
            int4 v = make_int4(c0 + j, c0 + j + 1, c0 + j + 2, c0 + j + 3);
            if (reorder) {
                const int32_t *r = reorder + h * D + c0 + j;
                v = make_int4(r[0], r[1], r[2], r[3]);
            }
            idx[j] = v.x & (D - 1); idx[j + 1] = v.y & (D - 1); idx[j + 2] = v.z & (D - 1); idx[j + 3] = v.w & (D - 1);
        }
        const float alpha = alphas ? alphas[h * NG + sub / LANES] : 1.0f;
        R row = next;
        if (have && h0 + h_step < h_end) next.load(src + (int64_t)(h0 + h_step) * D);
        if constexpr (!IS_V) {
            if (rot) {
                if (!inter) {
                    row.store(raw + c0);
                    __syncwarp();
                }
                if (here) rotate_row<T, D>(row, c0, cs, raw, a.rope.rot_dim, inter);
            }
        }
        row.store(turned + c0);
        __syncwarp();
        const uint16_t *from = reinterpret_cast<const uint16_t *>(turned);
#pragma unroll
        for (int j = 0; j < C; j += 2) row.w[j / 2] = (uint32_t)from[idx[j]] | (uint32_t)from[idx[j + 1]] << 16;
        __syncwarp();

        // extremes as the pair {min, -max}: min serves both
        uint32_t mn = row.w[0], ng = row.w[0] ^ 0x80008000u;
#pragma unroll
        for (int k = 1; k < R::WORDS; ++k) { mn = min2<T>(mn, row.w[k]); ng = min2<T>(ng, row.w[k] ^ 0x80008000u); }
        uint32_t ext = min2<T>(__byte_perm(mn, ng, 0x5410), __byte_perm(mn, ng, 0x7632));
#pragma unroll
        for (int m = 1; m < LANES; m <<= 1) ext = min2<T>(ext, __shfl_xor_sync(0xffffffffu, ext, m));
        const float2 e = floats<T>(ext);
        const float lo = __fadd_rn(__fmul_rn(alpha, e.x), 0.0f), hi = __fadd_rn(__fmul_rn(alpha, -e.y), 0.0f);
        const __half2 hz = __halves2half2(__float2half_rn(__fmul_rn(__fsub_rn(hi, lo), 1.0f / 15.0f)), __float2half_rn(lo));
        const float hf = __low2float(hz), zf = __high2float(hz);
        constexpr float MAGIC = 12582912.0f;      // 1.5 2^23: a sum with it is rounded to an integer, ties to even
        const float r = hf != 0.0f ? __frcp_rn(hf) : 0.0f;
        float far = 0.f, p[C / 4];      // largest remainder; four codes in a sum
#pragma unroll
        for (int j = 0; j < C; j += 2) {
            const float2 x = floats<T>(row.w[j / 2]);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float d = __fsub_rn(k ? x.y : x.x, zf);
                const float c = __fsub_rn(__fmaf_rn(d, r, MAGIC), MAGIC);
                far = fmaxf(far, fabsf(__fmaf_rn(-c, hf, d)));
                const float q = fminf(fmaxf(c, 0.0f), 15.0f);
                const int n = j + k;
                p[n / 4] = n % 4 == 0 ? q : __fmaf_rn(q, (float)(1 << (4 * (n % 4))), p[n / 4]);
            }
        }
        uint32_t codes = (uint32_t)(int)p[0];
        if constexpr (C == 8) codes |= (uint32_t)(int)p[1] << 16;
        // (also taken for quotients beyond 2^22, which the sum with MAGIC cannot round, and for infinities)
        if (!(far < 0.5f * hf * (1.0f - 3.814697265625e-06f)) && hf != 0.0f) {
            codes = 0u;
#pragma unroll
            for (int j = 0; j < C; ++j) {
                const float2 x = floats<T>(row.w[j / 2]);
                const float c = fminf(fmaxf(rintf(__fdiv_rn(__fsub_rn(j & 1 ? x.y : x.x, zf), hf)), 0.0f), 15.0f);
                codes |= (uint32_t)(int)c << (4 * j);
            }
        }
        if (hf == 0.0f) codes = 0u;
        if (here && page >= 0) {
            const int64_t at = page_row + (int64_t)h * P;
            if constexpr (C == 8) reinterpret_cast<uint32_t *>(codes_pool + at * (D / 2))[sub] = codes;
            else reinterpret_cast<uint16_t *>(codes_pool + at * (D / 2))[sub] = (uint16_t)codes;
            if (sub % LANES == 0) meta_pool[at * NG + sub / LANES] = *reinterpret_cast<const uint32_t *>(&hz);
            if (keep) row.store(win + (((int64_t)seq.slot * cfg.n_kv_heads + h) * cfg.ring_tokens + ring) * D + c0);
        }
    }
}

// blockIdx: x = tokens of a sequence, y = runs of heads, keys and values in turn, z = sequences.
template <typename T, int D, int NG>
__global__ void __launch_bounds__(kRowThreads) paged_append_kernel(const __grid_constant__ AppendIo io)
{
    __shared__ __align__(16) T rows[2 * kRowWarps][2][D + 8];      // a half-warp each: as read, rotated; the two rows of a warp start 4 banks apart
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const PagedArgs &a = io.p;
    const int b = blockIdx.z, unit = threadIdx.x >> 4;      // half-warp
    PagedSeq seq;
    if (!paged_sequence(a, b, true, seq)) {
        if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) set_status(a.c.status, SKVQ_STATUS_BAD_BATCH);
        return;
    }
    const int i0 = io.bulk ? blockIdx.x * kBulkTokens : blockIdx.x;
    if (i0 >= seq.n) return;
    const int i = io.bulk ? i0 + unit : i0, h0 = (blockIdx.y >> 1) * io.heads, h1 = min(h0 + io.heads, a.cfg.n_kv_heads);
    const int first = io.bulk ? h0 : h0 + unit, step = io.bulk ? 1 : 2 * kRowWarps;
    if (blockIdx.y & 1) append_rows<T, D, NG, true>(io, seq, b, i, first, step, h1, true, rows[unit][0], rows[unit][1]);
    else append_rows<T, D, NG, false>(io, seq, b, i, first, step, h1, true, rows[unit][0], rows[unit][1]);
}

struct ReadIo {
    PagedArgs p;
    void *k, *v;
    int64_t k_stride, v_stride;
    int window, heads, bulk;
};

template <typename T, int D, int NG>
__global__ void __launch_bounds__(kRowThreads) paged_read_kernel(const __grid_constant__ ReadIo io)
{
    using R = Row<T, D>;
    constexpr int C = R::C, LANES = 16 / NG;
    __shared__ __align__(16) T rows[2 * kRowWarps][D + 8];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const PagedArgs &a = io.p;
    const skvq_paged_config &cfg = a.cfg;
    const int b = blockIdx.z, unit = threadIdx.x >> 4, sub = threadIdx.x & 15;
    PagedSeq seq;
    if (!paged_sequence(a, b, true, seq)) {
        if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) set_status(a.c.status, SKVQ_STATUS_BAD_BATCH);
        return;
    }
    const bool is_v = blockIdx.y & 1;
    T *dst = static_cast<T *>(is_v ? io.v : io.k);
    const int i0 = io.bulk ? blockIdx.x * kBulkTokens : blockIdx.x;
    if (i0 >= seq.n || !dst) return;
    const int i = io.bulk ? i0 + unit : i0, h_begin = (blockIdx.y >> 1) * io.heads, h_end = min(h_begin + io.heads, cfg.n_kv_heads);
    const int first = io.bulk ? h_begin : h_begin + unit, step = io.bulk ? 1 : 2 * kRowWarps;
    const int P = cfg.page_tokens, t = seq.len - seq.n + i, c0 = sub * C;
    bool have = i < seq.n;
    const bool recent = io.window && cfg.window > 0 && t >= seq.len - cfg.window;
    int page = 0;
    if (have && !recent) {
        page = a.batch.page_table[(int64_t)b * a.batch.max_pages + t / P];
        if (page < 0 || page >= cfg.n_pages) {
            have = false;
            if (sub == 0) set_status(a.c.status, SKVQ_STATUS_BAD_PAGE);
        }
    }
    const int32_t *reorder = is_v ? a.c.reorder_v : a.c.reorder_k;
    const int64_t page_row = ((int64_t)page * cfg.n_kv_heads) * P + t % P;
    const uint8_t *codes_pool = static_cast<const uint8_t *>(is_v ? a.c.v_codes : a.c.k_codes);
    const uint32_t *meta_pool = static_cast<const uint32_t *>(is_v ? a.c.v_meta : a.c.k_meta);
    const T *win = static_cast<const T *>(is_v ? a.c.v_win : a.c.k_win);
    dst += (int64_t)(seq.row0 + i) * (is_v ? io.v_stride : io.k_stride) + c0;
    uint16_t *mine = reinterpret_cast<uint16_t *>(rows[unit]);
    auto load = [&](int h, uint32_t &codes, uint32_t &hz) {
        const int64_t at = page_row + (int64_t)h * P;
        codes = C == 8 ? reinterpret_cast<const uint32_t *>(codes_pool + at * (D / 2))[sub] : reinterpret_cast<const uint16_t *>(codes_pool + at * (D / 2))[sub];
        hz = meta_pool[at * NG + sub / LANES];
    };
    uint32_t codes_next = 0u, hz_next = 0u;
    if (have && !recent && first < h_end) load(first, codes_next, hz_next);
    for (int h0 = first; __any_sync(0xffffffffu, h0 < h_end); h0 += step) {
        const bool here = have && h0 < h_end;
        const int h = min(h0, h_end - 1);
        const uint32_t codes = codes_next;
        const __half2 hz = *reinterpret_cast<const __half2 *>(&hz_next);
        if (have && !recent && h0 + step < h_end) load(h0 + step, codes_next, hz_next);
        R row;
        if (recent) {
            if (here) row.load(win + (((int64_t)seq.slot * cfg.n_kv_heads + h) * cfg.ring_tokens + t % cfg.ring_tokens) * D + c0);
        } else {
            const float hf = __low2float(hz), zf = __high2float(hz);
            float v[C];
#pragma unroll
            for (int j = 0; j < C; ++j)      // 2^23 + code, minus 2^23
                v[j] = __fadd_rn(__fmul_rn(hf, __fsub_rn(__uint_as_float(0x4B000000u | ((codes >> (4 * j)) & 15u)), 8388608.0f)), zf);
#pragma unroll
            for (int k = 0; k < R::WORDS; ++k) row.w[k] = packed<T>(v[2 * k], v[2 * k + 1]);
        }
        if (reorder) {
            const int32_t *idx = reorder + h * D + c0;
#pragma unroll
            for (int k = 0; k < R::WORDS; ++k) {
                mine[idx[2 * k] & (D - 1)] = (uint16_t)row.w[k];
                mine[idx[2 * k + 1] & (D - 1)] = (uint16_t)(row.w[k] >> 16);
            }
            __syncwarp();
            row.load(rows[unit] + c0);
            __syncwarp();
        }
        if (here) row.store(dst + (int64_t)h * D);
    }
}

// Grid: tokens of the longest sequence, runs of heads for keys and for values, sequences.  Side-by-side tokens need at least two; a run
// is as long as keeps several waves of CTAs (the angles are loaded once per run).
template <typename Io> dim3 row_grid(const PagedArgs &a, Io &io)
{
    const int H = a.cfg.n_kv_heads;
    io.bulk = a.batch.max_new >= 4 ? 1 : 0;
    const long long tokens = io.bulk ? (a.batch.max_new + kBulkTokens - 1) / kBulkTokens : a.batch.max_new;
    if (io.bulk) {
        io.heads = H;
        while (io.heads > 4 && tokens * a.batch.n_seqs * 2 * ((H + io.heads - 1) / io.heads) < 32LL * sm_count()) io.heads = (io.heads + 1) / 2;
    } else {
        io.heads = H < 2 * kRowWarps ? H : 2 * kRowWarps;
    }
    return dim3((unsigned)tokens, 2 * ((H + io.heads - 1) / io.heads), a.batch.n_seqs);
}

template <typename T> cudaError_t append_by_shape(const dim3 &grid, cudaStream_t stream, const AppendIo &io)
{
    if (io.p.cfg.head_dim == 128)
        return io.p.ng == 1   ? launch_chained(paged_append_kernel<T, 128, 1>, grid, kRowThreads, 0, stream, io)
               : io.p.ng == 2 ? launch_chained(paged_append_kernel<T, 128, 2>, grid, kRowThreads, 0, stream, io)
                              : launch_chained(paged_append_kernel<T, 128, 4>, grid, kRowThreads, 0, stream, io);
    return io.p.ng == 1 ? launch_chained(paged_append_kernel<T, 64, 1>, grid, kRowThreads, 0, stream, io)
                        : launch_chained(paged_append_kernel<T, 64, 2>, grid, kRowThreads, 0, stream, io);
}
template <typename T> cudaError_t read_by_shape(const dim3 &grid, cudaStream_t stream, const ReadIo &io)
{
    if (io.p.cfg.head_dim == 128)
        return io.p.ng == 1   ? launch_chained(paged_read_kernel<T, 128, 1>, grid, kRowThreads, 0, stream, io)
               : io.p.ng == 2 ? launch_chained(paged_read_kernel<T, 128, 2>, grid, kRowThreads, 0, stream, io)
                              : launch_chained(paged_read_kernel<T, 128, 4>, grid, kRowThreads, 0, stream, io);
    return io.p.ng == 1 ? launch_chained(paged_read_kernel<T, 64, 1>, grid, kRowThreads, 0, stream, io)
                        : launch_chained(paged_read_kernel<T, 64, 2>, grid, kRowThreads, 0, stream, io);
}

}  // namespace

cudaError_t launch_paged_append(const PagedArgs &a, const void *k, const void *v, int64_t k_stride, int64_t v_stride, cudaStream_t stream)
{
    AppendIo io{a, k, v, k_stride, v_stride, 0, 0};
    const dim3 grid = row_grid(a, io);
    return a.cfg.dtype == SKVQ_F16 ? append_by_shape<__half>(grid, stream, io) : append_by_shape<__nv_bfloat16>(grid, stream, io);
}

cudaError_t launch_paged_read(const PagedArgs &a, int window, void *k, void *v, int64_t k_stride, int64_t v_stride, cudaStream_t stream)
{
    ReadIo io{a, k, v, k_stride, v_stride, window, 0, 0};
    const dim3 grid = row_grid(a, io);
    return a.cfg.dtype == SKVQ_F16 ? read_by_shape<__half>(grid, stream, io) : read_by_shape<__nv_bfloat16>(grid, stream, io);
}

}  // namespace skvq
