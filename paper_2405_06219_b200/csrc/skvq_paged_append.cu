// skvq_paged_append and skvq_paged_read: rotated, reordered, 4-bit quantized rows into pages, and back.
//
// Sixteen lanes own the rows of two neighbouring tokens (of one KV head, keys or values), D/16 neighbouring channels a lane; the half-warps
// of a CTA take token pairs (bulk) or heads of the same pair (steps of few tokens, where latency counts) and walk over heads, so a token's
// angles stay in registers.  The rows are read coalesced and put into shared memory interleaved, a 32-bit word holding one channel
// of both tokens: partner channels of the rotation, and the gather in stored order, then take one shared-memory access for
// two rows, the arithmetic is on pairs of fp32, and minimum and maximum are one packed instruction for both.  A group's extremes are reduced by
// shuffles.  Measured: a 32k-token prompt of 32 heads of 128 channels, rotated and appended, 325 us, read back 182 (floors of 105 each); a decode
// step of 64 sequences 6.9 and 4.1 us in a graph.
// What bounds the append is instructions, not bytes (68 % of the issue slots at a quarter of the DRAM rate), so the code is formed without a
// division,
//   code = rint(d / h): t = fma(d, RN(1/h), 1.5 2^23) holds rint(d RN(1/h)); the remainder d - code h tells whether the quotient can be
//   near k + 0.5 (|remainder| >= h/2 (1 - 2^-18)); only then is more done.
// The quantizer arithmetic is explicitly rounded fp32: codes and parameters do not depend on compiler contraction.
#include "skvq_paged_split.cuh"

namespace skvq {
namespace {

constexpr int kRowWarps = 4;
constexpr int kRowThreads = kRowWarps * 32;
constexpr int kBulkTokens = 4 * kRowWarps;      // tokens of a CTA when they lie side by side

struct AppendIo {
    PagedArgs p;
    const void *k, *v;
    int64_t k_stride, v_stride;
    int heads;       // heads a CTA walks over
    int bulk;        // 1: half-warps take tokens; 0: heads of one token
    uint64_t nothing = 0x8000000080000000ull;      // a pair of -0: a product with it added is the rounded product (a plain paired product before
                                                  // a paired sum is contracted with it; a value from outside is not)
};

template <typename T> __device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b);
template <typename T> __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b);
template <> __device__ __forceinline__ uint32_t min2<__half>(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("min.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
template <> __device__ __forceinline__ uint32_t max2<__half>(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
template <> __device__ __forceinline__ uint32_t min2<__nv_bfloat16>(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("min.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
template <> __device__ __forceinline__ uint32_t max2<__nv_bfloat16>(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// Two rows <-> words {channel of the first, channel of the second}.
template <typename T, int D> __device__ __forceinline__ void interleave(const Row<T, D> (&row)[2], uint32_t (&w)[Row<T, D>::C])
{
#pragma unroll
    for (int k = 0; k < Row<T, D>::WORDS; ++k) {
        w[2 * k] = __byte_perm(row[0].w[k], row[1].w[k], 0x5410);
        w[2 * k + 1] = __byte_perm(row[0].w[k], row[1].w[k], 0x7632);
    }
}
template <typename T, int D> __device__ __forceinline__ void separate(const uint32_t (&w)[Row<T, D>::C], Row<T, D> (&row)[2])
{
#pragma unroll
    for (int k = 0; k < Row<T, D>::WORDS; ++k) {
        row[0].w[k] = __byte_perm(w[2 * k], w[2 * k + 1], 0x5410);
        row[1].w[k] = __byte_perm(w[2 * k], w[2 * k + 1], 0x7632);
    }
}
template <int C> __device__ __forceinline__ void put_words(uint32_t *p, const uint32_t (&w)[C])
{
#pragma unroll
    for (int k = 0; k < C; k += 4) *reinterpret_cast<uint4 *>(p + k) = make_uint4(w[k], w[k + 1], w[k + 2], w[k + 3]);
}
template <int C> __device__ __forceinline__ void get_words(const uint32_t *p, uint32_t (&w)[C])
{
#pragma unroll
    for (int k = 0; k < C; k += 4) {
        const uint4 v = *reinterpret_cast<const uint4 *>(p + k);
        w[k] = v.x; w[k + 1] = v.y; w[k + 2] = v.z; w[k + 3] = v.w;
    }
}
// A lane's C gather indices of a head (identity without a reorder index).
template <int C, int D> __device__ __forceinline__ void load_index(int (&idx)[C], const int32_t *reorder, int h, int c0)
{
#pragma unroll
    for (int j = 0; j < C; j += 4) {
        int4 v = make_int4(c0 + j, c0 + j + 1, c0 + j + 2, c0 + j + 3);
        if (reorder) {
            const int32_t *r = reorder + h * D + c0 + j;
            v = make_int4(r[0], r[1], r[2], r[3]);
        }
        idx[j] = v.x & (D - 1); idx[j + 1] = v.y & (D - 1); idx[j + 2] = v.z & (D - 1); idx[j + 3] = v.w & (D - 1);
    }
}

template <typename T, int D, int NG, bool IS_V>
__device__ __forceinline__ void append_rows(const AppendIo &io, const PagedSeq &seq, int b, int i, int h_first, int h_step, int h_end, uint32_t *raw, uint32_t *turned)
{
    using R = Row<T, D>;
    constexpr int C = R::C, LANES = 16 / NG;      // lanes of a group
    const PagedArgs &a = io.p;
    const skvq_paged_config &cfg = a.cfg;
    const int sub = threadIdx.x & 15, P = cfg.page_tokens, c0 = sub * C;
    const bool rot = !IS_V && a.rope.table, inter = a.rope.interleaved;
    const int rot_dim = a.rope.rot_dim, half = rot_dim / 2;
    const bool straight = (inter ? rot_dim : half) % C == 0;      // a lane's channels are all rotated or none, its partners lie side by side
    bool have[2], keep[2];
    int page[2], ring[2];
    int64_t page_row[2];
    uint64_t cosine[IS_V ? 1 : C], sine[IS_V ? 1 : C];      // of both tokens
    const T *src[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int t = seq.len - seq.n + i + k;
        have[k] = i + k < seq.n;
        page[k] = -1;
        if (have[k]) {
            page[k] = a.batch.page_table[(int64_t)b * a.batch.max_pages + t / P];
            if (page[k] < 0 || page[k] >= cfg.n_pages) {
                page[k] = -1;
                if (sub == 0) set_status(a.c.status, SKVQ_STATUS_BAD_PAGE);
            }
        }
        src[k] = static_cast<const T *>(IS_V ? io.v : io.k) + (int64_t)(seq.row0 + i + k) * (IS_V ? io.v_stride : io.k_stride) + c0;
        page_row[k] = ((int64_t)page[k] * cfg.n_kv_heads) * P + t % P;
        keep[k] = cfg.window > 0 && have[k] && page[k] >= 0 && t >= seq.len - cfg.ring_tokens;
        ring[k] = cfg.ring_tokens > 0 ? t % cfg.ring_tokens : 0;
    }
    if constexpr (!IS_V) {
        float2 cs[2][C];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
#pragma unroll
            for (int j = 0; j < C; ++j) cs[k][j] = make_float2(0.f, 0.f);
            if (rot && have[k]) load_angles(cs[k], a.rope, seq.len - seq.n + i + k, c0);
        }
#pragma unroll
        for (int j = 0; j < C; ++j) {
            const float sign = (inter ? !((c0 + j) & 1) : c0 + j < half) ? -1.f : 1.f;
            cosine[j] = pair(cs[0][j].x, cs[1][j].x);
            sine[j] = pair(sign * cs[0][j].y, sign * cs[1][j].y);
        }
    }
    const int32_t *reorder = IS_V ? a.c.reorder_v : a.c.reorder_k;
    const float *alphas = IS_V ? a.c.alpha_v : a.c.alpha_k;
    uint8_t *codes_pool = static_cast<uint8_t *>(IS_V ? a.c.v_codes : a.c.k_codes);
    uint32_t *meta_pool = static_cast<uint32_t *>(IS_V ? a.c.v_meta : a.c.k_meta);
    T *win = static_cast<T *>(IS_V ? a.c.v_win : a.c.k_win);

    R next[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
        for (int m = 0; m < R::WORDS; ++m) next[k].w[m] = 0u;
        if (have[k] && h_first < h_end) next[k].load(src[k] + (int64_t)h_first * D);
    }
    for (int h0 = h_first; __any_sync(0xffffffffu, h0 < h_end); h0 += h_step) {
        const bool here = h0 < h_end;
        const int h = min(h0, h_end - 1);
        int idx[C];
        load_index<C, D>(idx, reorder, h, c0);
        const float alpha = alphas ? alphas[h * NG + sub / LANES] : 1.0f;
        uint32_t w[C];
        interleave<T, D>(next, w);
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (have[k] && h0 + h_step < h_end) next[k].load(src[k] + (int64_t)(h0 + h_step) * D);
        if constexpr (!IS_V) {
            if (rot) {
                // y = x c + o s with the partner o and, for the first channel of a pair, the sine negated: the roundings of x c - o s
                uint32_t o[C];
                if (inter) {
#pragma unroll
                    for (int j = 0; j < C; ++j) o[j] = w[j ^ 1];
                } else {
                    put_words(raw + c0, w);
                    __syncwarp();
                    if (straight) get_words(raw + (c0 < half ? c0 + half : (c0 < rot_dim ? c0 - half : c0)), o);
                    else {
#pragma unroll
                        for (int j = 0; j < C; ++j) {
                            const int c = c0 + j;
                            o[j] = raw[c < half ? c + half : (c < rot_dim ? c - half : c)];
                        }
                    }
                }
                if (c0 < rot_dim) {
#pragma unroll
                    for (int j = 0; j < C; ++j) {
                        const uint32_t v = packed<T>(pair_add(pair_fma(pair_of<T>(w[j]), cosine[j], io.nothing), pair_fma(pair_of<T>(o[j]), sine[j], io.nothing)));
                        if (straight || c0 + j < rot_dim) w[j] = v;
                    }
                }
            }
        }
        put_words(turned + c0, w);
        __syncwarp();
#pragma unroll
        for (int j = 0; j < C; ++j) w[j] = turned[idx[j]];
        __syncwarp();

        uint32_t mn = w[0], mx = w[0];
#pragma unroll
        for (int j = 1; j < C; ++j) { mn = min2<T>(mn, w[j]); mx = max2<T>(mx, w[j]); }
#pragma unroll
        for (int m = 1; m < LANES; m <<= 1) {
            mn = min2<T>(mn, __shfl_xor_sync(0xffffffffu, mn, m));
            mx = max2<T>(mx, __shfl_xor_sync(0xffffffffu, mx, m));
        }
        const float2 mnf = floats<T>(mn), mxf = floats<T>(mx);
        constexpr float MAGIC = 12582912.0f;      // 1.5 2^23: a sum with it is rounded to an integer, ties to even
        __half2 hz2[2];
        float h2[2], z2[2], r2[2], far2[2] = {0.f, 0.f};      // far2: largest remainder
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const float lo = __fadd_rn(__fmul_rn(alpha, k ? mnf.y : mnf.x), 0.0f), hi = __fadd_rn(__fmul_rn(alpha, k ? mxf.y : mxf.x), 0.0f);
            hz2[k] = __halves2half2(__float2half_rn(__fmul_rn(__fsub_rn(hi, lo), 1.0f / 15.0f)), __float2half_rn(lo));
            h2[k] = __low2float(hz2[k]);
            z2[k] = __high2float(hz2[k]);
            r2[k] = h2[k] != 0.0f ? __frcp_rn(h2[k]) : 0.0f;
        }
        uint32_t code[2];
        {
            const uint64_t neg_z = pair(-z2[0], -z2[1]), neg_h = pair(-h2[0], -h2[1]), inverse = pair(r2[0], r2[1]);
            const uint64_t magic = pair(MAGIC, MAGIC), neg_magic = pair(-MAGIC, -MAGIC);
            uint32_t q[C];      // both tokens' codes as fp16, clamped
#pragma unroll
            for (int j = 0; j < C; ++j) {
                const uint64_t d = pair_add(pair_of<T>(w[j]), neg_z), c = pair_add(pair_fma(d, inverse, magic), neg_magic);
                float e0, e1, c0f, c1f;
                unpair(pair_fma(c, neg_h, d), e0, e1);
                unpair(c, c0f, c1f);
                far2[0] = fmaxf(far2[0], fabsf(e0));
                far2[1] = fmaxf(far2[1], fabsf(e1));
                asm("{\n .reg .b32 t;\n cvt.rn.relu.f16x2.f32 t, %1, %2;\n min.f16x2 %0, t, %3;\n}" : "=r"(q[j]) : "f"(c1f), "f"(c0f), "r"(0x4B804B80u));      // 15
            }
            // 1024 + first + 16 second: exact, and the fp16's low byte is the codes' byte
            uint32_t u[C / 2];
#pragma unroll
            for (int j = 0; j < C / 2; ++j)
                asm("{\n .reg .b32 t;\n add.rn.f16x2 t, %1, %3;\n fma.rn.f16x2 %0, %2, %4, t;\n}" : "=r"(u[j]) : "r"(q[2 * j]), "r"(q[2 * j + 1]), "r"(0x64006400u), "r"(0x4C004C00u));
            const uint32_t lo = __byte_perm(u[0], u[1], 0x6240);      // bytes: first token's two, second token's two
            if constexpr (C == 8) {
                const uint32_t hi = __byte_perm(u[2], u[3], 0x6240);
                code[0] = __byte_perm(lo, hi, 0x5410);
                code[1] = __byte_perm(lo, hi, 0x7632);
            } else {
                code[0] = lo & 0xFFFFu;
                code[1] = lo >> 16;
            }
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const float hf = h2[k], zf = z2[k], r = r2[k], far = far2[k];
            const __half2 hz = hz2[k];
            uint32_t codes = code[k];
            // In doubt (fp16 values meet k + 1/2 often: two iterations in five have such an element somewhere in the warp): the remainder
            // is exact, so a tie shows as |remainder| = h/2 and goes to the even code; what is near a tie but none, and quotients
            // beyond 2^22 or infinite, take the division.
            const float hh = 0.5f * hf;
            if (!(far < hh * (1.0f - 3.814697265625e-06f)) && hf != 0.0f) {
                bool hard = false;
                codes = 0u;
#pragma unroll
                for (int j = 0; j < C; ++j) {
                    const float2 x = floats<T>(w[j]);
                    const float d = __fsub_rn(k ? x.y : x.x, zf), t = __fmaf_rn(d, r, MAGIC);
                    float c = __fsub_rn(t, MAGIC);
                    const float e = __fmaf_rn(-c, hf, d);
                    if (fabsf(e) == hh) {
                        if (__float_as_int(t) & 1) c += e > 0.f ? 1.f : -1.f;
                    } else if (!(fabsf(e) < hh * (1.0f - 3.814697265625e-06f))) {
                        hard = true;
                    }
                    codes |= (uint32_t)(int)fminf(fmaxf(c, 0.0f), 15.0f) << (4 * j);
                }
                if (hard) {
                    codes = 0u;
#pragma unroll
                    for (int j = 0; j < C; ++j) {
                        const float2 x = floats<T>(w[j]);
                        const float c = fminf(fmaxf(rintf(__fdiv_rn(__fsub_rn(k ? x.y : x.x, zf), hf)), 0.0f), 15.0f);
                        codes |= (uint32_t)(int)c << (4 * j);
                    }
                }
            }
            if (hf == 0.0f) codes = 0u;
            if (here && page[k] >= 0) {
                const int64_t at = page_row[k] + (int64_t)h * P;
                if constexpr (C == 8) reinterpret_cast<uint32_t *>(codes_pool + at * (D / 2))[sub] = codes;
                else reinterpret_cast<uint16_t *>(codes_pool + at * (D / 2))[sub] = (uint16_t)codes;
                if (sub % LANES == 0) meta_pool[at * NG + sub / LANES] = *reinterpret_cast<const uint32_t *>(&hz);
            }
        }
        if (here && (keep[0] || keep[1])) {
            R out[2];
            separate<T, D>(w, out);
#pragma unroll
            for (int k = 0; k < 2; ++k)
                if (keep[k]) out[k].store(win + (((int64_t)seq.slot * cfg.n_kv_heads + h) * cfg.ring_tokens + ring[k]) * D + c0);
        }
    }
}

// blockIdx: x = tokens of a sequence (16, or a pair), y = runs of heads, keys and values in turn, z = sequences.
// Five CTAs per SM: what spills (angles of the key rows) costs less than the warps that 150 registers would leave out (32k-token prompt,
// append and read back: 542 us against 595).
template <typename T, int D, int NG>
__global__ void __launch_bounds__(kRowThreads, 5) paged_append_kernel(const __grid_constant__ AppendIo io)
{
    __shared__ __align__(16) uint32_t rows[2 * kRowWarps][2][D + 4];      // a half-warp each: as read, rotated
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const PagedArgs &a = io.p;
    const int b = blockIdx.z, unit = threadIdx.x >> 4;      // half-warp
    PagedSeq seq;
    if (!paged_sequence(a, b, true, seq)) {
        if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) set_status(a.c.status, SKVQ_STATUS_BAD_BATCH);
        return;
    }
    const int i0 = blockIdx.x * (io.bulk ? kBulkTokens : 2);
    if (i0 >= seq.n) return;
    const int i = io.bulk ? i0 + 2 * unit : i0, h0 = (blockIdx.y >> 1) * io.heads, h1 = min(h0 + io.heads, a.cfg.n_kv_heads);
    const int first = io.bulk ? h0 : h0 + unit, step = io.bulk ? 1 : 2 * kRowWarps;
    if (blockIdx.y & 1) append_rows<T, D, NG, true>(io, seq, b, i, first, step, h1, rows[unit][0], rows[unit][1]);
    else append_rows<T, D, NG, false>(io, seq, b, i, first, step, h1, rows[unit][0], rows[unit][1]);
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
    __shared__ __align__(16) uint32_t rows[2 * kRowWarps][D + 4];
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
    const int i0 = blockIdx.x * (io.bulk ? kBulkTokens : 2);
    if (i0 >= seq.n || !dst) return;
    const int i = io.bulk ? i0 + 2 * unit : i0, h_begin = (blockIdx.y >> 1) * io.heads, h_end = min(h_begin + io.heads, cfg.n_kv_heads);
    const int first = io.bulk ? h_begin : h_begin + unit, step = io.bulk ? 1 : 2 * kRowWarps;
    const int P = cfg.page_tokens, c0 = sub * C;
    bool have[2], recent[2];
    int64_t page_row[2], win_row[2];
    T *out[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int t = seq.len - seq.n + i + k;
        have[k] = i + k < seq.n;
        recent[k] = io.window && t >= seq.lq;
        int page = 0;
        if (have[k]) {
            page = a.batch.page_table[(int64_t)b * a.batch.max_pages + t / P];
            if (page < 0 || page >= cfg.n_pages) {
                have[k] = false;
                if (sub == 0) set_status(a.c.status, SKVQ_STATUS_BAD_PAGE);
            }
        }
        page_row[k] = ((int64_t)page * cfg.n_kv_heads) * P + t % P;
        win_row[k] = recent[k] ? (int64_t)seq.slot * cfg.n_kv_heads * cfg.ring_tokens + t % cfg.ring_tokens : 0;
        out[k] = dst + (int64_t)(seq.row0 + i + k) * (is_v ? io.v_stride : io.k_stride) + c0;
    }
    const int32_t *reorder = is_v ? a.c.reorder_v : a.c.reorder_k;
    const uint8_t *codes_pool = static_cast<const uint8_t *>(is_v ? a.c.v_codes : a.c.k_codes);
    const uint32_t *meta_pool = static_cast<const uint32_t *>(is_v ? a.c.v_meta : a.c.k_meta);
    const T *win = static_cast<const T *>(is_v ? a.c.v_win : a.c.k_win);
    uint32_t *mine = rows[unit];
    uint32_t codes_next[2] = {0u, 0u}, hz_next[2] = {0u, 0u};
    auto load = [&](int h) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (have[k] && !recent[k] && h < h_end) {
                const int64_t at = page_row[k] + (int64_t)h * P;
                codes_next[k] = C == 8 ? reinterpret_cast<const uint32_t *>(codes_pool + at * (D / 2))[sub] : reinterpret_cast<const uint16_t *>(codes_pool + at * (D / 2))[sub];
                hz_next[k] = meta_pool[at * NG + sub / LANES];
            }
        }
    };
    load(first);
    for (int h0 = first; __any_sync(0xffffffffu, h0 < h_end); h0 += step) {
        const bool here = h0 < h_end;
        const int h = min(h0, h_end - 1);
        // 2^23 + 16^p code, minus 2^23, times h / 16^p (all exact but the product), for nibbles p = 0 .. 4 in place, then from bit 20 on
        uint32_t w[C];
        {
            const float2 par0 = __half22float2(*reinterpret_cast<const __half2 *>(&hz_next[0])), par1 = __half22float2(*reinterpret_cast<const __half2 *>(&hz_next[1]));
            const uint64_t z = pair(par0.y, par1.y), neg = pair(-8388608.0f, -8388608.0f), down = pair(0.0625f, 0.0625f);
            uint64_t h = pair(par0.x, par1.x);
            uint64_t hs[5];
#pragma unroll
            for (int p = 0; p < 5; ++p) { hs[p] = h; h = pair_mul(h, down); }
#pragma unroll
            for (int j = 0; j < C; ++j) {
                const int p = j < 5 ? j : j - 5;
                const uint32_t a0 = j < 5 ? codes_next[0] : codes_next[0] >> 20, a1 = j < 5 ? codes_next[1] : codes_next[1] >> 20;
                const uint64_t c = pair_add(pair(__uint_as_float(0x4B000000u | (a0 & (15u << (4 * p)))), __uint_as_float(0x4B000000u | (a1 & (15u << (4 * p))))), neg);
                w[j] = packed<T>(pair_add(pair_mul(hs[p], c), z));
            }
        }
        R row[2];
        if ((recent[0] && have[0]) || (recent[1] && have[1])) {
            separate<T, D>(w, row);
#pragma unroll
            for (int k = 0; k < 2; ++k)
                if (recent[k] && have[k] && here) row[k].load(win + (win_row[k] + (int64_t)h * cfg.ring_tokens) * D + c0);
            interleave<T, D>(row, w);
        }
        load(h0 + step);
        if (reorder) {
            int idx[C];
            load_index<C, D>(idx, reorder, h, c0);
#pragma unroll
            for (int j = 0; j < C; ++j) mine[idx[j]] = w[j];
            __syncwarp();
            get_words(mine + c0, w);
            __syncwarp();
        }
        separate<T, D>(w, row);
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (here && have[k]) row[k].store(out[k] + (int64_t)h * D);
    }
}

// Grid: tokens of the longest sequence, runs of heads for keys and for values, sequences.  A run
// is as long as keeps several waves of CTAs (the angles are loaded once per run).
template <typename Io> dim3 row_grid(const PagedArgs &a, Io &io)
{
    const int H = a.cfg.n_kv_heads;
    io.bulk = a.batch.max_new >= 8 ? 1 : 0;
    const long long tokens = io.bulk ? (a.batch.max_new + kBulkTokens - 1) / kBulkTokens : (a.batch.max_new + 1) / 2;
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
