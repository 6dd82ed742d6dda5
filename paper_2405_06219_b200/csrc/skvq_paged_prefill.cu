// skvq_paged_attention for many query rows per (sequence, KV head): prompts and chunks of prompts, on tcgen05.
//
// One CTA per SM works on items of up to 256 packed rows (row = new token * (Hq/Hkv) + query head) of one KV head, as two row
// blocks of 128, over 128-token tiles of the cache.  Three kinds of warps, ordered by mbarriers:
//   dequantizers  4 warps, a thread per token of the tile: codes and parameters come from the pages into registers one tile ahead,
//                 leave as fp16(h c + z) (one rounding) in the 128-byte swizzle that both products read -- the key tile as the
//                 K-major B operand of Q K^T, the value tile, same picture, as the MN-major B operand of P V; window tokens are
//                 copied.  Two buffers of each.
//   softmax       2 x 4 warps, a thread per row: S from tensor memory, probabilities back, in place, as the fp16 A operand; the row
//                 sum in fp32.  The reference of a row is raised, and O multiplied, only when a score exceeds it by more than
//                 2^kLazy: O is then read and written about once or twice per item.
//   issuers       a warp per row block: O += P V~, then, behind it in the tensor core's queue, the next tile's S = Q K~^T.  (Issuing
//                 blocks while the queue is full: from a softmax warp it cost the whole block that time.)
// A tile's scores come as two halves of 64 tokens with a buffer each: while one half becomes probabilities, the products of the other
// half and of the other block run, so a softmax warp finds its next scores waiting.
// A nibble pair (i, i + 4) of a code word becomes two neighbouring fp16, so the channels of each run of eight lie in the order
// 0 4 1 5 2 6 3 7 in the operands; the queries are laid out the same way and the outputs put back.
// Items are laid end to end, priced in tiles (causal limits included), and cut into equal runs, one per CTA; an item that several
// runs share goes through the workspace to the merge kernel.
// Measured: 2048 queries at the end of 32k tokens, 32 heads over 8, D = 128: 1216 to 1290 us, 0.83 to 0.88 PFLOP/s (tensor core 61 % busy); ragged
// prompts up to 4095 tokens, 32 heads of 64: 558 to 571 us, of it 74 for the queries.  At D = 128 the chain of a row block bounds it: scores out
// of tensor memory, exponentials, probabilities back, product, about 4600 clocks a tile of 256 x 128 where the products alone take 2048;
// more stages need more than tensor memory's 512 columns.  At D = 64, whose items are short (9 tiles on average in those prompts), what
// lies between items is as much: queries, first scores, last products and rows follow one another, and 128 columns stay idle.
#include <math_constants.h>

#include "skvq_mma_common.cuh"
#include "skvq_paged.cuh"
#include "skvq_paged_split.cuh"
#include "skvq_tcgen05.cuh"

namespace skvq {
namespace {

using mmak::and_or;
using mmak::ex2_approx;
using mmak::mbar_init;
using mmak::mbar_try_wait;
using mmak::smem_u32;
using namespace tc5;

constexpr int kBlock = 128;                     // rows of a row block, tokens of a tile
constexpr int kSoftmaxThreads = 2 * kBlock;     // warps 0-7
constexpr int kDequantThreads = kBlock;         // warps 8-11
constexpr int kPrefillThreads = kSoftmaxThreads + kDequantThreads + 128;      // warps 12, 13 issue the products of a row block each
constexpr float kLazy = 8.f;                    // log2 of how far a score may exceed its row's reference
constexpr float kPOffset = 6.f;                 // probabilities are held times 2^6: up to 2^14 in fp16, down to 2^-30 of the reference

struct PrefillArgs {
    PagedAttnArgs a;
    int n_slots;
    __half *queries;      // [Hkv][T * Hq/Hkv][D], by paged_queries_kernel
    float *scales;        // [Hkv][T * Hq/Hkv]
};

template <int D>
struct PGeo {
    static constexpr int HALVES = D / 64;                      // 64-channel halves of an operand tile: 128-byte rows
    static constexpr int HALF_BYTES = kBlock * 128;
    static constexpr int TILE_BYTES = HALVES * HALF_BYTES;      // one 128 x D fp16 operand
    static constexpr int Q = 0;                                // 2 row blocks; at the end of an item its output rows
    static constexpr int K = 2 * TILE_BYTES;                   // 2 buffers
    static constexpr int V = 4 * TILE_BYTES;                   // 2 buffers
    static constexpr int SMEM = 6 * TILE_BYTES + 1024;         // and room to align to 1024 bytes
    static constexpr int TMEM_S = 0, TMEM_O = 256;             // columns: S (P in place) 2 blocks x 2 halves x 64, O 2 x D
};

// Shared-memory matrix descriptors in the 128-byte swizzle.  K-major: 8-row groups 1024 bytes apart.  MN-major: 64-element runs of
// the MN dimension `mn_stride` bytes apart, groups of 8 along K 1024 bytes apart.
__device__ __forceinline__ uint64_t desc_k_major(uint32_t addr)
{
    return (uint64_t)((addr >> 4) & 0x3FFFu) | ((uint64_t)1 << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ uint64_t desc_mn_major(uint32_t addr, uint32_t mn_stride)
{
    return (uint64_t)((addr >> 4) & 0x3FFFu) | ((uint64_t)(mn_stride >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// D (tensor memory) = A (tensor memory, fp16 pairs along the columns) B + D
__device__ __forceinline__ void umma_f16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
                 " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
                 ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t addr, const uint32_t (&r)[32])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
                 "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
                 ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
                 "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
                 "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
                 "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t (&r)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
                 "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// Waits for this thread's tensor-memory loads; the registers that were in flight pass through the statement.
__device__ __forceinline__ void tmem_wait_ld32(float (&r)[32])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(r[0]), "+f"(r[1]), "+f"(r[2]), "+f"(r[3]), "+f"(r[4]), "+f"(r[5]), "+f"(r[6]), "+f"(r[7]),
                   "+f"(r[8]), "+f"(r[9]), "+f"(r[10]), "+f"(r[11]), "+f"(r[12]), "+f"(r[13]), "+f"(r[14]), "+f"(r[15]),
                   "+f"(r[16]), "+f"(r[17]), "+f"(r[18]), "+f"(r[19]), "+f"(r[20]), "+f"(r[21]), "+f"(r[22]), "+f"(r[23]),
                   "+f"(r[24]), "+f"(r[25]), "+f"(r[26]), "+f"(r[27]), "+f"(r[28]), "+f"(r[29]), "+f"(r[30]), "+f"(r[31])
                 :: "memory");
}
__device__ __forceinline__ bool elect_one()      // true in one lane of a converged warp
{
    uint32_t r;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(r));
    return r != 0;
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ uint32_t h2(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t h2_sub(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t h2_fma(uint32_t a, uint32_t b, uint32_t c)
{
    uint32_t r;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}
template <typename T> __device__ __forceinline__ uint32_t to_h2(uint32_t v);      // see as_h2 of the kernel for few rows
template <> __device__ __forceinline__ uint32_t to_h2<__half>(uint32_t v) { return v; }
template <> __device__ __forceinline__ uint32_t to_h2<__nv_bfloat16>(uint32_t v) { return h2(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u)); }

// Poll with a limit in clock cycles (about a tenth of a second); false: it ran out.
__device__ __forceinline__ bool mbar_wait_cycles(uint32_t bar, uint32_t parity)
{
    if (mbar_try_wait(bar, parity)) return true;
    const long long t0 = clock64();
    for (;;) {
#pragma unroll 1
        for (int i = 0; i < 64; ++i)
            if (mbar_try_wait(bar, parity)) return true;
        if (clock64() - t0 > 200000000ll) return false;
    }
}

// 2^a and 2^b by multiply-adds: x = n + f with n the nearest integer, a polynomial of degree 4 for 2^f on [-1/2, 1/2] (fitted for the
// smallest relative error: 3e-6, a hundredth of the fp16 step that the result is rounded to), n added to the exponent.  Arguments below
// -126, -infinity among them, give 2^-126.
constexpr int kPolynomial = 2;
__device__ __forceinline__ void exp2_pair(float &a, float &b)
{
    constexpr float MAGIC = 12582912.0f;      // 1.5 2^23: the sum's low bits hold the rounded integer
    const uint64_t x = pair(fmaxf(a, -126.0f), fmaxf(b, -126.0f));
    const uint64_t t = pair_add(x, pair(MAGIC, MAGIC));
    const uint64_t f = pair_fma(pair_add(t, pair(-MAGIC, -MAGIC)), pair(-1.f, -1.f), x);
    uint64_t p = pair_fma(f, pair(0.00957010f, 0.00957010f), pair(0.05591786f, 0.05591786f));
    p = pair_fma(f, p, pair(0.24024744f, 0.24024744f));
    p = pair_fma(f, p, pair(0.69312179f, 0.69312179f));
    p = pair_fma(f, p, pair(0.99999928f, 0.99999928f));
    float p0, p1, t0, t1;
    unpair(p, p0, p1);
    unpair(t, t0, t1);
    a = __int_as_float(__float_as_int(p0) + (__float_as_int(t0) << 23));
    b = __int_as_float(__float_as_int(p1) + (__float_as_int(t1) << 23));
}

// Position 0..7 inside a run of eight operand channels -> stored channel.
__device__ __forceinline__ int channel_at(int pos) { return (pos >> 1) + 4 * (pos & 1); }

// The items of one sequence: per KV head, blocks of 256 rows; tiles that block m looks at.
struct PItems {
    int rep, n, len, lq, causal, tiles_c;
    __device__ __forceinline__ void set(const PrefillArgs &a, const PagedSeq &s)
    {
        rep = a.a.p.cfg.n_q_heads / a.a.p.cfg.n_kv_heads;
        n = s.n;
        len = s.len;
        lq = s.lq;
        causal = a.a.causal;
        tiles_c = (lq + kBlock - 1) / kBlock;
    }
    __device__ __forceinline__ int rows() const { return n * rep; }
    __device__ __forceinline__ int blocks() const { return rows() > kFewRows ? (rows() + 2 * kBlock - 1) / (2 * kBlock) : 0; }      // the others are the other kernel's
    __device__ __forceinline__ int limit(int row) const { return causal ? min(len, len - n + row / rep + 1) : len; }      // tokens below it are seen
    __device__ __forceinline__ int tiles(int m) const
    {
        const int lim = limit(min((m + 1) * 2 * kBlock, rows()) - 1);
        if (lim <= 0) return 0;
        return lim <= lq ? (lim + kBlock - 1) / kBlock : tiles_c + (lim - lq + kBlock - 1) / kBlock;
    }
    __device__ __forceinline__ int cost(int m) const { return max(tiles(m), 1); }
};

// What a role of the CTA works on: block m of KV head hk of sequence b, tiles [t0, t1) of `total`.  It lives in shared memory: kept in
// registers it spilled, and with 220 KB of shared memory in use a spilled register comes back from the L2 cache, a thousand cycles
// later.
struct PSegment {
    long long f, f1;         // what is left of the CTA's run
    int valid, b, hk, m, t0, t1, total, parts;      // parts: CTAs that share the rest of the item
    PagedSeq seq;
    PItems it;
};

// The next segment, by one thread of the role.
__device__ __noinline__ void next_segment(const PrefillArgs &a, const long long *pre, long long ups, PSegment &s)
{
    long long f = s.f;
    if (f >= s.f1) { s.valid = 0; return; }
    int b = s.b;
    while (pre[b + 1] <= f) ++b;
    PagedSeq seq;
    PItems it;
    paged_sequence(a.a.p, b, false, seq);
    it.set(a, seq);
    const long long per_head = (pre[b + 1] - pre[b]) / a.a.p.cfg.n_kv_heads;
    long long at = f - pre[b];
    const int hk = (int)(at / per_head);
    at -= hk * per_head;
    int m = 0, c = it.cost(0);
    while (at >= c) { at -= c; c = it.cost(++m); }
    const int take = (int)min((long long)(c - at), s.f1 - f);
    s.b = b;
    s.hk = hk;
    s.m = m;
    s.total = it.tiles(m);
    s.t0 = (int)at;
    s.t1 = min((int)at + take, s.total);
    s.parts = (int)((f - at + c - 1) / ups - blockIdx.x + 1);
    s.seq = seq;
    s.it = it;
    s.f = f + take;
    s.valid = 1;
}

// The queries as rows of the A operand, for all row blocks at once: rotated, rounded to T, reordered, in the operand's channel order, fp16
// times a power of two per row; packed row (token * Hq/Hkv + query head of the KV head) of KV head h in row h * T * Hq/Hkv + it.  Sixteen
// lanes own a row; a half-warp takes a token and walks over the heads with the token's angles in registers.  (Prepared by the softmax
// warps, item by item, this took 35,000 cycles per item of 256 rows.)
constexpr int kQueryThreads = 128;
constexpr int kQueryTokens = kQueryThreads / 16;
struct QueryArgs {
    PrefillArgs f;
    int heads;      // query heads a CTA walks over
};
template <typename T, int D>
__global__ void __launch_bounds__(kQueryThreads) paged_queries_kernel(const __grid_constant__ QueryArgs args)
{
    using R = Row<T, D>;
    constexpr int C = R::C;
    __shared__ __align__(16) T rows[kQueryTokens][2][D + 8];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const PagedAttnArgs &a = args.f.a;
    const PagedArgs &p = a.p;
    const int unit = threadIdx.x >> 4, sub = threadIdx.x & 15, c0 = sub * C, rep = p.cfg.n_q_heads / p.cfg.n_kv_heads;
    PagedSeq seq;
    if (!paged_sequence(p, blockIdx.z, false, seq) || seq.n * rep <= kFewRows) return;
    if ((int)blockIdx.x * kQueryTokens >= seq.n) return;
    const int i = blockIdx.x * kQueryTokens + unit, pos = seq.len - seq.n + i;
    const int h0 = blockIdx.y * args.heads, h1 = min(h0 + args.heads, p.cfg.n_q_heads);
    const bool have = i < seq.n, turn = p.rope.table && have && pos >= 0;
    const int64_t tok = seq.row0 + i, all = (int64_t)p.batch.n_tokens * rep;
    float2 cs[C];
    if (turn) load_angles(cs, p.rope, pos, c0);
    const T *src = static_cast<const T *>(a.q) + tok * a.q_stride + c0;
    T *raw = rows[unit][0], *turned = rows[unit][1];
    const float sign = a.sm_scale < 0.f ? -1.f : (a.sm_scale == 0.f ? 0.f : 1.f);      // the rows' scale is positive
    const float scale = (sign == 0.f ? 1.f : fabsf(a.sm_scale)) * 1.4426950408889634f;
    int from[C], hk = -1;
    R next;
#pragma unroll
    for (int k = 0; k < R::WORDS; ++k) next.w[k] = 0u;
    if (have && h0 < h1) next.load(src + (int64_t)h0 * D);
    for (int h = h0; h < h1; ++h) {
        if (h / rep != hk) {
            hk = h / rep;
#pragma unroll
            for (int j = 0; j < C; ++j) {
                const int c = (c0 & ~7) + channel_at((c0 + j) & 7);
                from[j] = p.c.reorder_k ? p.c.reorder_k[hk * D + c] & (D - 1) : c;
            }
        }
        R row = next;
        if (have && h + 1 < h1) next.load(src + (int64_t)(h + 1) * D);
        if (p.rope.table) {
            if (!p.rope.interleaved) {
                row.store(raw + c0);
                __syncwarp();
            }
            if (turn) rotate_row<T, D>(row, c0, cs, raw, p.rope.rot_dim, p.rope.interleaved);
        }
        row.store(turned + c0);
        __syncwarp();
        float x[C], mx = 0.f;
#pragma unroll
        for (int j = 0; j < C; ++j) { x[j] = Elem<T>::to_float(turned[from[j]]); mx = fmaxf(mx, fabsf(x[j])); }
        __syncwarp();
#pragma unroll
        for (int d = 1; d < 16; d <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
        float up = 1.f;      // the row's largest to [2^4, 2^5): exact, and far from fp16's ends whatever the type's range
        if (mx > 0.f && mx < CUDART_INF_F) up = __int_as_float((127 + min(4 - (__float_as_int(mx) >> 23) + 127, 60)) << 23);
        if (!have) continue;
        const float f = mx < CUDART_INF_F ? up * sign : CUDART_NAN_F;      // an infinite query: see the kernel for few rows
        const int64_t at = hk * all + tok * rep + (h - hk * rep);
        __half *dst = args.f.queries + at * D + c0;
        if constexpr (C == 8)
            *reinterpret_cast<uint4 *>(dst) = make_uint4(h2(x[0] * f, x[1] * f), h2(x[2] * f, x[3] * f), h2(x[4] * f, x[5] * f), h2(x[6] * f, x[7] * f));
        else *reinterpret_cast<uint2 *>(dst) = make_uint2(h2(x[0] * f, x[1] * f), h2(x[2] * f, x[3] * f));
        if (sub == 0) args.f.scales[at] = scale / up;
    }
}

// A row block's queries and their scales into shared memory, and the source channel of every output column.  Not inlined, like write_rows:
// what they keep in registers would spill in the loop over tiles.
template <int D>
__device__ __noinline__ void load_queries(const PrefillArgs &args, const PSegment &s, int rows, int row_base, uint8_t *q_tile, float *row_scale, uint16_t *out_channel)
{
    using Geo = PGeo<D>;
    const int row = threadIdx.x & (kBlock - 1), hk = s.hk;
    const int32_t *reorder_v = args.a.p.c.reorder_v;
    const int64_t at = (int64_t)hk * args.a.p.batch.n_tokens * s.it.rep + (int64_t)s.seq.row0 * s.it.rep + row_base;
    const uint4 *src = reinterpret_cast<const uint4 *>(args.queries + at * D);
#pragma unroll
    for (int e0 = 0; e0 < kBlock * D / 8; e0 += 8 * kBlock) {      // 8 loads in flight
        uint4 v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int e = e0 + k * kBlock + row;
            v[k] = make_uint4(0u, 0u, 0u, 0u);
            if (e / (D / 8) < rows) v[k] = src[e];
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int e = e0 + k * kBlock + row, r = e / (D / 8), c8 = e % (D / 8);
            *reinterpret_cast<uint4 *>(q_tile + (c8 >> 3) * Geo::HALF_BYTES + r * 128 + (((c8 & 7) ^ (r & 7)) << 4)) = v[k];
        }
    }
    row_scale[row] = row < rows ? args.scales[at + row] : 0.f;
    for (int c = row; c < D; c += kBlock) {
        const int st = (c & ~7) + channel_at(c & 7);
        out_channel[c] = (uint16_t)(reorder_v ? reorder_v[hk * D + st] & (D - 1) : st);
    }
}

// The result of a row block: finished rows, or (a share of an item) sums that the merge kernel joins.  `failed`: a wait ran out, what the
// block holds is worth nothing; its rows become NaN, and so does what a share is joined with.
template <typename T, int D>
__device__ __noinline__ void write_rows(const PagedAttnArgs &args, const PSegment &s, int rows, int row_base, bool work, bool failed, uint32_t o_addr, float ref, float l,
                                        float rs, uint8_t *q_tile, const uint16_t *out_channel, bool whole, float *part)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, row = threadIdx.x & (kBlock - 1);
    // read once, together: through the reference every field is a memory access
    void *const out = args.out;
    float *const lse = args.lse;
    const int64_t out_stride = args.out_stride;
    const int n_q_heads = args.p.cfg.n_q_heads;
    const int rep = s.it.rep, hk = s.hk, row0 = s.seq.row0;
    const int i = (row_base + row) / rep, head = hk * rep + (row_base + row) - i * rep;
    if (failed) work = false;
    const bool none = !work || (ref == -CUDART_INF_F && l == l);      // no token seen; a query that is not a number leaves its mark in l
    const float blank = failed ? CUDART_NAN_F : 0.f;
    if (whole) {
        const float inv = 1.f / l;
        T *rows_out = reinterpret_cast<T *>(q_tile);      // [128][D], 16-byte pieces of a row at piece ^ (row & 7); all products have been read
#pragma unroll 1
        for (int c0 = 0; c0 < D; c0 += 16) {
            float x[16];
            if (work) {
                tmem_ld16f(o_addr + c0, x);
                tmem_wait_ld16f(x);
            }
#pragma unroll
            for (int c = 0; c < 16; ++c) {
                const int dst = work ? out_channel[c0 + c] : c0 + c;
                rows_out[row * D + ((((dst >> 3) ^ (row & 7))) << 3) + (dst & 7)] = Elem<T>::from_float(none ? blank : x[c] * inv);
            }
        }
        if (lse && row < rows)
            lse[(int64_t)(row0 + i) * n_q_heads + head] = failed ? blank : none ? -CUDART_INF_F : (ref * rs + log2f(l) - kPOffset) * 0.6931471805599453f;
        __syncwarp();
        constexpr int PER_ROW = D / 8;
        for (int e = lane; e < 32 * PER_ROW; e += 32) {      // this warp's 32 rows, 16 bytes a lane
            const int r = (warp & 3) * 32 + e / PER_ROW, c8 = e % PER_ROW;
            if (r < rows) {
                const int ri = (row_base + r) / rep, rh = hk * rep + (row_base + r) - ri * rep;
                *reinterpret_cast<uint4 *>(static_cast<T *>(out) + (int64_t)(row0 + ri) * out_stride + (int64_t)rh * D + c8 * 8) =
                    *reinterpret_cast<const uint4 *>(rows_out + r * D + ((c8 ^ (r & 7)) << 3));
            }
        }
        __syncwarp();
    } else {
        // a share of an item: unscaled sums, stored channels in order
        part += row * partial_stride(D);
#pragma unroll 1
        for (int c0 = 0; c0 < D; c0 += 16) {
            float x[16];
            if (work) {
                tmem_ld16f(o_addr + c0, x);
                tmem_wait_ld16f(x);
            }
            if (row < rows) {
#pragma unroll
                for (int c = 0; c < 16; c += 8) {
                    *reinterpret_cast<float4 *>(part + c0 + c) = none ? make_float4(blank, blank, blank, blank) : make_float4(x[c], x[c + 2], x[c + 4], x[c + 6]);
                    *reinterpret_cast<float4 *>(part + c0 + c + 4) = none ? make_float4(blank, blank, blank, blank) : make_float4(x[c + 1], x[c + 3], x[c + 5], x[c + 7]);
                }
            }
        }
        if (row < rows) {
            part[D] = failed || ref == -CUDART_INF_F ? -CUDART_INF_F : ref * rs;
            part[D + 1] = none ? blank : l;
        }
    }
}

template <typename T, int D, int NG>
__global__ void __launch_bounds__(kPrefillThreads, 1) paged_prefill_kernel(const __grid_constant__ PrefillArgs args)
{
    using Geo = PGeo<D>;
    const PagedAttnArgs &a = args.a;
    const PagedArgs &p = a.p;
    const skvq_paged_config &cfg = p.cfg;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    long long *pre = reinterpret_cast<long long *>(smem + Geo::SMEM - 1024);
    __shared__ __align__(8) uint64_t bars[24];
    __shared__ uint32_t tmem_sh;
    __shared__ int fail_sh;
    __shared__ long long scan_sh[16];
    __shared__ float row_scale[2 * kBlock];
    __shared__ uint16_t out_channel[2][D];      // source channel of every operand column, per row block
    __shared__ PSegment seg_sh[5];              // of the two row blocks' softmax, of the dequantizers, of the two issuers
    __shared__ uint32_t bad_sh[4][4];           // of the last four tiles: tokens without a page, a bit each (a tile's are read until its
                                                // probabilities are written, when the tile two further on may be in the making)
    const int tid = threadIdx.x, lane = tid & 31, B = p.batch.n_seqs;
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);      // one value per warp, and the compiler knows: descriptors stay in uniform registers

    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");

    // ---- the flat partition
    {
        long long carry = 0;
        for (int base = 0; base < B; base += kPrefillThreads) {
            const int b = base + tid;
            long long c = 0;
            if (b < B) {
                PagedSeq s;
                if (paged_sequence(p, b, false, s)) {
                    PItems it;
                    it.set(args, s);
                    const int blocks = it.blocks();
                    for (int m = 0; m < blocks; ++m) c += it.cost(m);
                    c *= cfg.n_kv_heads;
                }      // the kernel for few rows reports the others
            }
            long long incl = c;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const long long v = __shfl_up_sync(0xffffffffu, incl, d);
                if (lane >= d) incl += v;
            }
            if (lane == 31) scan_sh[warp] = incl;
            __syncthreads();
            long long before = carry;
            for (int w = 0; w < kPrefillThreads / 32; ++w) {
                if (w < warp) before += scan_sh[w];
                carry += scan_sh[w];
            }
            if (b < B) pre[b] = before + incl - c;
            __syncthreads();
        }
        if (tid == 0) pre[B] = carry;
    }
    // ---- barriers, tensor memory
    const uint32_t bar0 = smem_u32(bars);
    const uint32_t k_full = bar0, k_empty = bar0 + 16, v_full = bar0 + 32, v_empty = bar0 + 48;      // + 8 * buffer
    const uint32_t s_full = bar0 + 64, pv_done = bar0 + 96;                                          // + 16 * row block + 8 * half
    const uint32_t p_full = bar0 + 128, q_full = bar0 + 160, drained = bar0 + 176;                  // the same; + 8 * row block
    if (tid == 0) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            mbar_init(k_full + 8 * i, kDequantThreads);
            mbar_init(k_empty + 8 * i, 2);      // both row blocks' products
            mbar_init(v_full + 8 * i, kDequantThreads);
            mbar_init(v_empty + 8 * i, 2);
            mbar_init(s_full + 16 * i, 1);
            mbar_init(s_full + 16 * i + 8, 1);
            mbar_init(pv_done + 16 * i, 1);
            mbar_init(pv_done + 16 * i + 8, 1);
            mbar_init(p_full + 16 * i, 4);      // an arrival per warp
            mbar_init(p_full + 16 * i + 8, 4);
            mbar_init(q_full + 8 * i, 4);
            mbar_init(drained + 8 * i, 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fail_sh = 0;
    }
    if (warp == 0) tmem_alloc(smem_u32(&tmem_sh), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_sh;
    const long long total = pre[B], ups = max((total + args.n_slots - 1) / args.n_slots, 1LL);
    int *desc = reinterpret_cast<int *>(a.ws) + (size_t)blockIdx.x * kDescInts;
    if (tid < 5) {
        PSegment &first = seg_sh[tid];
        first.f = blockIdx.x * ups;
        first.f1 = min(first.f + ups, total);
        first.b = 0;
        if (first.f < first.f1) {
            int lo = 0, hi = B - 1;
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (pre[mid] <= first.f) lo = mid; else hi = mid - 1;
            }
            first.b = lo;
        }
    }
    if (tid == 0) desc[0] = 0;
    __syncthreads();
    // A wait that runs out is reported; the thread then goes through its loops without waiting.  The flag is set before anything that
    // follows from it, so that a row block that has read spoilt operands finds it set when it comes to write its rows.
    bool alive = true;
    volatile int *fail = &fail_sh;
    auto wait = [&](uint32_t bar, uint32_t parity) {      // by whole warps
        if (alive && !mbar_wait_cycles(bar, parity)) {
            alive = false;
            *fail = 1;
            set_status(p.c.status, SKVQ_STATUS_COPY_TIMEOUT);
        }
    };
    // A role is 128 threads (block 0, block 1, the dequantizers) or a warp (an issuer).
    const int role = warp < 12 ? warp >> 2 : 3 + (warp & 1);
    const PSegment &s = seg_sh[role];
    auto role_sync = [&]() {
        if (warp < 12) asm volatile("bar.sync %0, 128;" ::"r"(1 + role) : "memory");
        else __syncwarp();
    };
    auto next = [&]() {
        role_sync();
        if ((warp < 12 ? tid & 127 : lane) == 0) next_segment(args, pre, ups, seg_sh[role]);
        role_sync();
        return s.valid != 0;
    };

    if (warp >= 8 && warp < 12) {
        // ================================================================ dequantizers
        const int row = tid - kSoftmaxThreads;      // token of the tile
        const int P = cfg.page_tokens, page_shift = __ffs(P) - 1;
        constexpr int PIECES = D / 32;              // 16-byte pieces of a code row
        uint32_t n = 0;                             // tiles so far
        while (next()) {
            const int32_t *table = p.batch.page_table + (int64_t)s.b * p.batch.max_pages;
            const int64_t win_row0 = ((int64_t)s.seq.slot * cfg.n_kv_heads + s.hk) * cfg.ring_tokens;
            uint4 kc[PIECES], vc[PIECES];
            uint32_t km[NG], vm[NG];
            int page = -1;
            // this thread's token in tile t
            auto token_of = [&](int t) { return (t < s.it.tiles_c ? t * kBlock : s.it.lq + (t - s.it.tiles_c) * kBlock) + row; };
            // its page (of a window token too: one without a page is left out); -1: no such token, -2: no such page
            auto page_of = [&](int t) {
                const int tok = token_of(t);
                if (t >= s.t1 || tok >= (t < s.it.tiles_c ? s.it.lq : s.seq.len)) return -1;
                const int id = table[tok >> page_shift];
                if (id < 0 || id >= cfg.n_pages) { set_status(p.c.status, SKVQ_STATUS_BAD_PAGE); return -2; }
                return id;
            };
            auto load_codes = [&](int t) {      // of tile t, with `page`
                if (page >= 0 && t < s.it.tiles_c) {
                    const int64_t at = ((int64_t)page * cfg.n_kv_heads + s.hk) * P + ((t * kBlock + row) & (P - 1));
#pragma unroll
                    for (int i = 0; i < PIECES; ++i) {
                        kc[i] = reinterpret_cast<const uint4 *>(static_cast<const uint8_t *>(p.c.k_codes) + at * (D / 2))[i];
                        vc[i] = reinterpret_cast<const uint4 *>(static_cast<const uint8_t *>(p.c.v_codes) + at * (D / 2))[i];
                    }
#pragma unroll
                    for (int g = 0; g < NG; ++g) {
                        km[g] = static_cast<const uint32_t *>(p.c.k_meta)[at * NG + g];
                        vm[g] = static_cast<const uint32_t *>(p.c.v_meta)[at * NG + g];
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < PIECES; ++i) kc[i] = vc[i] = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                    for (int g = 0; g < NG; ++g) km[g] = vm[g] = 0u;      // rows that hold nothing become zeros
                }
            };
            page = page_of(s.t0);
            load_codes(s.t0);
            int page_next = page_of(s.t0 + 1);
            for (int t = s.t0; t < s.t1; ++t, ++n) {
                const uint32_t buf = n & 1, phase = (n >> 1) & 1;
                if (*fail) alive = false;
                uint8_t *kt = smem + Geo::K + buf * Geo::TILE_BYTES + row * 128, *vt = smem + Geo::V + buf * Geo::TILE_BYTES + row * 128;
                // one code word -> one 16-byte piece of the operand row
                auto piece = [&](uint8_t *base, int c8, uint32_t w, uint32_t hh, uint32_t zz) {
                    constexpr uint32_t M = 0x64006400u, SIXTEENTH = 0x2C002C00u, MINUS64 = 0xD400D400u;
                    const uint32_t u = w >> 8;
                    uint4 r;
                    r.x = h2_fma(h2_sub(and_or(w, 0x000F000Fu, M), M), hh, zz);
                    r.y = h2_fma(h2_fma(and_or(w, 0x00F000F0u, M), SIXTEENTH, MINUS64), hh, zz);
                    r.z = h2_fma(h2_sub(and_or(u, 0x000F000Fu, M), M), hh, zz);
                    r.w = h2_fma(h2_fma(and_or(u, 0x00F000F0u, M), SIXTEENTH, MINUS64), hh, zz);
                    *reinterpret_cast<uint4 *>(base + (c8 >> 3) * Geo::HALF_BYTES + (((c8 & 7) ^ (row & 7)) << 4)) = r;
                };
                auto expand = [&](uint8_t *base, const uint4 (&c)[PIECES], const uint32_t (&m)[NG]) {
#pragma unroll
                    for (int i = 0; i < PIECES; ++i) {      // 32 channels
                        const uint32_t hz = m[i * NG / PIECES], hh = __byte_perm(hz, hz, 0x1010), zz = __byte_perm(hz, hz, 0x3232);
                        piece(base, 4 * i, c[i].x, hh, zz);
                        piece(base, 4 * i + 1, c[i].y, hh, zz);
                        piece(base, 4 * i + 2, c[i].z, hh, zz);
                        piece(base, 4 * i + 3, c[i].w, hh, zz);
                    }
                };
                auto copy_row = [&](uint8_t *base, const void *pool, bool have, int64_t r) {
#pragma unroll 4
                    for (int i = 0; i < D / 8; ++i) {
                        uint4 x = make_uint4(0u, 0u, 0u, 0u);
                        if (have) x = reinterpret_cast<const uint4 *>(static_cast<const T *>(pool) + r * D)[i];
                        x.x = to_h2<T>(x.x); x.y = to_h2<T>(x.y); x.z = to_h2<T>(x.z); x.w = to_h2<T>(x.w);
                        *reinterpret_cast<uint4 *>(base + (i >> 3) * Geo::HALF_BYTES + (((i & 7) ^ (row & 7)) << 4)) =
                            make_uint4(__byte_perm(x.x, x.z, 0x5410), __byte_perm(x.x, x.z, 0x7632), __byte_perm(x.y, x.w, 0x5410), __byte_perm(x.y, x.w, 0x7632));
                    }
                };
                const bool quantized = t < s.it.tiles_c;
                const bool have = !quantized && page >= 0;      // a window token
                const int64_t r = have ? win_row0 + token_of(t) % cfg.ring_tokens : 0;
                if (n >= 2) wait(k_empty + 8 * buf, phase ^ 1u);
                {
                    const uint32_t gone = __ballot_sync(0xffffffffu, page == -2);
                    if (lane == 0) bad_sh[n & 3][warp - 8] = gone;
                }
                if (alive) {
                    if (quantized) expand(kt, kc, km);
                    else copy_row(kt, p.c.k_win, have, r);
                }
                proxy_fence();
                mbar_arrive(k_full + 8 * buf);
                if (n >= 2) wait(v_empty + 8 * buf, phase ^ 1u);
                if (alive) {
                    if (quantized) expand(vt, vc, vm);
                    else copy_row(vt, p.c.v_win, have, r);
                }
                proxy_fence();
                mbar_arrive(v_full + 8 * buf);
                page = page_next;
                load_codes(t + 1);      // in flight until the next tile's buffer is free; behind the fence, which would wait for them
                page_next = page_of(t + 2);
            }
        }
    } else if (warp >= 12) {
        // ================================================================ products of a row block
        if (warp < 14) {
            const int blk = warp & 1;
            constexpr uint32_t kIdescS = idesc_f16_f32(kBlock, kBlock / 2);
            constexpr uint32_t kIdescO = idesc_f16_f32(kBlock, D) | (1u << 16);      // B is MN-major
            const uint32_t smem_base = smem_u32(smem);
            // S = Q K~^T of half `hf` of tile number `tile`.  The whole warp runs these (addresses are warp-uniform), one lane issues.
            auto issue_scores = [&](uint32_t tile, int hf) {
                const uint32_t buf = tile & 1;
                const uint64_t dq = desc_k_major(smem_base + Geo::Q + blk * Geo::TILE_BYTES), dk = desc_k_major(smem_base + Geo::K + buf * Geo::TILE_BYTES + hf * 64 * 128);
                if (hf == 0) wait(k_full + 8 * buf, (tile >> 1) & 1);
                tc_fence_after();
                if (elect_one()) {
    #pragma unroll
                    for (int ks = 0; ks < D / 16; ++ks) {
                        constexpr uint32_t half = Geo::HALF_BYTES >> 4;
                        umma_f16(tmem + Geo::TMEM_S + blk * kBlock + hf * 64, dq + (ks >> 2) * half + (ks & 3) * 2, dk + (ks >> 2) * half + (ks & 3) * 2, kIdescS, ks > 0);
                    }
                    umma_commit(s_full + 16 * blk + 8 * hf);
                    if (hf) umma_commit(k_empty + 8 * buf);
                }
                __syncwarp();
            };
            auto issue_values = [&](uint32_t tile, int hf, bool first) {
                const uint32_t buf = tile & 1;
                const uint64_t dv = desc_mn_major(smem_base + Geo::V + buf * Geo::TILE_BYTES + hf * 64 * 128, Geo::HALF_BYTES);
                if (hf == 0) wait(v_full + 8 * buf, (tile >> 1) & 1);
                tc_fence_after();
                if (elect_one()) {
    #pragma unroll
                    for (int ks = 0; ks < kBlock / 32; ++ks)
                        umma_f16_ts(tmem + Geo::TMEM_O + blk * D, tmem + Geo::TMEM_S + blk * kBlock + hf * 64 + ks * 8, dv + ks * (2048 >> 4), kIdescO, !first || ks > 0);
                    umma_commit(pv_done + 16 * blk + 8 * hf);
                    if (hf) umma_commit(v_empty + 8 * buf);
                }
                __syncwarp();
            };
            uint32_t n = 0, ns = 0, nq = 0;      // tiles so far (both blocks'), of this block, items of this block
            while (next()) {
                if (*fail) alive = false;
                if (s.it.rows() <= (s.m * 2 + blk) * kBlock) {
                    // A block without rows follows the tiles all the same: it frees the buffers on its side, and it must not reach a
                    // later item while a barrier is still two phases behind what it would wait for.
                    for (int t = s.t0; t < s.t1; ++t, ++n) {
                        wait(k_full + 8 * (n & 1), (n >> 1) & 1);
                        if (lane == 0) mbar_arrive(k_empty + 8 * (n & 1));
                        wait(v_full + 8 * (n & 1), (n >> 1) & 1);
                        if (lane == 0) mbar_arrive(v_empty + 8 * (n & 1));
                    }
                    continue;
                }
                if (s.t0 >= s.t1) continue;
                wait(q_full + 8 * blk, nq & 1);
                ++nq;
                issue_scores(n, 0);
                issue_scores(n, 1);
                for (int t = s.t0; t < s.t1; ++t, ++n, ++ns) {
    #pragma unroll 1
                    for (int hf = 0; hf < 2; ++hf) {
                        wait(p_full + 16 * blk + 8 * hf, ns & 1);
                        issue_values(n, hf, t == s.t0 && hf == 0);
                        if (t + 1 < s.t1) issue_scores(n + 1, hf);
                    }
                }
            }
            if (__any_sync(0xffffffffu, *fail != 0)) {      // nobody may have waited for the last products: they must not outlive the CTA
                if (elect_one()) umma_commit(drained + 8 * blk);
                mbar_wait_cycles(drained + 8 * blk, 0);
            }
        }
    } else {
        // ================================================================ softmax
        const int blk = warp >> 2, row = tid & (kBlock - 1);                       // row block, row = lane of the tensor memory
        const uint32_t quad = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t s_addr = tmem + Geo::TMEM_S + blk * kBlock + quad, o_addr = tmem + Geo::TMEM_O + blk * D + quad;
        uint8_t *q_tile = smem + Geo::Q + blk * Geo::TILE_BYTES;
        uint32_t n = 0, ns = 0;      // tiles so far (both blocks'), tiles of this block so far
        while (next()) {
            const int rows = min(s.it.rows() - (s.m * 2 + blk) * kBlock, kBlock);      // of this block; may be <= 0
            const int row_base = (s.m * 2 + blk) * kBlock;
            const bool whole = s.t0 == 0 && s.t1 == s.total;
            const bool work = s.t0 < s.t1 && rows > 0;
            if (*fail) alive = false;
            if (work) {
                load_queries<D>(args, s, rows, row_base, q_tile, row_scale + blk * kBlock, out_channel[blk]);
                proxy_fence();
                __syncwarp();
                if (lane == 0) mbar_arrive(q_full + 8 * blk);
                role_sync();      // row_scale and out_channel of the whole block
            }
            const float rs = work ? row_scale[blk * kBlock + row] : 1.f;
            const int lim = s.it.limit(row_base + min(row, max(rows, 1) - 1));
            float ref = -CUDART_INF_F, l = 0.f;      // reference (unscaled score), sum of probabilities
            if (!work) n += max(s.t1 - s.t0, 0);
            for (int t = s.t0; work && t < s.t1; ++t, ++n) {
                const bool quantized = t < s.it.tiles_c;
                const int tok0 = quantized ? t * kBlock : s.it.lq + (t - s.it.tiles_c) * kBlock;
                const int seen_tile = min(lim, quantized ? s.it.lq : s.seq.len) - tok0;      // tokens of the tile below it are seen
#pragma unroll 1
                for (int hf = 0; hf < 2; ++hf) {
                    const uint32_t h_addr = s_addr + hf * 64;
                    const int seen = seen_tile - hf * 64;
                    const bool first = t == s.t0 && hf == 0;
                    wait(s_full + 16 * blk + 8 * hf, ns & 1);
                    tc_fence_after();
                    float x[32], y[32];
                    tmem_ld32(h_addr, x);
                    tmem_ld32(h_addr + 32, y);
                    const bool edge = __any_sync(0xffffffffu, seen < 64 || (bad_sh[n & 3][2 * hf] | bad_sh[n & 3][2 * hf + 1]) != 0u);
                    tmem_wait_ld32(x);
                    tmem_wait_ld32(y);
                    if (edge) {
                        // hidden columns become -infinity in place; the code below then is the same for all tiles
#pragma unroll 1
                        for (int run = 0; run < 2; ++run) {
                            const int left = seen - 32 * run;      // which of its 32 columns the row sees, one bit each
                            uint32_t v = left >= 32 ? 0xFFFFFFFFu : (left <= 0 ? 0u : (1u << left) - 1u);
                            v &= ~bad_sh[n & 3][2 * hf + run];
                            tmem_ld32(h_addr + 32 * run, x);
                            tmem_wait_ld32(x);
                            uint32_t w[32];
#pragma unroll
                            for (int c = 0; c < 32; ++c) w[c] = (v >> c) & 1u ? __float_as_uint(x[c]) : 0xFF800000u;
                            tmem_st32(h_addr + 32 * run, w);
                        }
                        tmem_wait_st();
                        tmem_ld32(h_addr, x);
                        tmem_ld32(h_addr + 32, y);
                        tmem_wait_ld32(x);
                        tmem_wait_ld32(y);
                    }
                    float mx;
                    {
                        float m0 = fmaxf(x[0], y[0]), m1 = fmaxf(x[1], y[1]), m2 = fmaxf(x[2], y[2]), m3 = fmaxf(x[3], y[3]);
#pragma unroll
                        for (int c = 4; c < 32; c += 4) {
                            m0 = fmaxf(fmaxf(m0, x[c]), y[c]);
                            m1 = fmaxf(fmaxf(m1, x[c + 1]), y[c + 1]);
                            m2 = fmaxf(fmaxf(m2, x[c + 2]), y[c + 2]);
                            m3 = fmaxf(fmaxf(m3, x[c + 3]), y[c + 3]);
                        }
                        mx = fmaxf(fmaxf(m0, m1), fmaxf(m2, m3));
                    }
                    // ---- raise the reference: at first, then only when a score exceeds it by 2^kLazy
                    float down = 1.f;
                    const bool raise = !first && __any_sync(0xffffffffu, (mx - ref) * rs > kLazy);
                    if (first) ref = mx;
                    else if (raise && mx > ref) {
                        down = ref == -CUDART_INF_F ? 0.f : ex2_approx((ref - mx) * rs);
                        ref = mx;
                        l *= down;
                    }
                    const float base = kPOffset - (ref == -CUDART_INF_F ? 0.f : ref * rs);
                    const uint64_t rs2 = pair(rs, rs), base2 = pair(base, base);
                    uint64_t l0 = 0ull, l1 = 0ull;      // pairs of sums
                    // Of every eight exponentials the last kPolynomial are computed with multiply-adds: the special-function unit, at 16 a
                    // clock for the SM, would alone take as long as the tensor core.
                    auto probabilities = [&](float (&v)[32], int run) {
                        uint32_t w[16];
#pragma unroll
                        for (int c = 0; c < 32; c += 8) {
#pragma unroll
                            for (int k = c; k < c + 8; k += 2) {
                                unpair(pair_fma(pair(v[k], v[k + 1]), rs2, base2), v[k], v[k + 1]);
                                if (k % 8 < 8 - kPolynomial) { v[k] = ex2_approx(v[k]); v[k + 1] = ex2_approx(v[k + 1]); }
                                else exp2_pair(v[k], v[k + 1]);
                                if (k & 2) l1 = pair_add(l1, pair(v[k], v[k + 1]));
                                else l0 = pair_add(l0, pair(v[k], v[k + 1]));
                                w[k / 2] = h2(v[k], v[k + 1]);
                            }
                        }
                        tmem_st16(h_addr + run * 16, w);      // over scores that are in registers
                    };
                    probabilities(x, 0);
                    probabilities(y, 1);
                    {
                        float a0, a1;
                        unpair(pair_add(l0, l1), a0, a1);
                        l += a0 + a1;
                    }
                    if (raise) {      // O follows the reference, once the products of the half before have landed in it
                        if (hf) wait(pv_done + 16 * blk, ns & 1);
                        else wait(pv_done + 16 * blk + 8, (ns - 1) & 1);
                        tc_fence_after();
#pragma unroll 1
                        for (int c0 = 0; c0 < D; c0 += 32) {
                            tmem_ld32(o_addr + c0, x);
                            tmem_wait_ld32(x);
                            uint32_t w[32];
#pragma unroll
                            for (int c = 0; c < 32; ++c) w[c] = __float_as_uint(x[c] * down);
                            tmem_st32(o_addr + c0, w);
                        }
                    }
                    tmem_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(p_full + 16 * blk + 8 * hf);
                }
                ++ns;
            }
            if (rows <= 0) continue;
            // ---- the block's result
            if (work) {
                wait(pv_done + 16 * blk + 8, (ns - 1) & 1);
                tc_fence_after();
            }
            alive = __all_sync(0xffffffffu, alive && !*fail);
            write_rows<T, D>(a, s, rows, row_base, work, !alive, o_addr, ref, l, rs, q_tile, out_channel[blk], whole,
                             a.ws + (size_t)args.n_slots * kDescInts + (((size_t)blockIdx.x * 2 + (s.t0 == 0 ? 1 : 0)) * 2 * kBlock + blk * kBlock) * partial_stride(D));
            if (!whole && s.t0 == 0 && tid == 0) {
                desc[1] = s.seq.row0; desc[2] = s.seq.n; desc[3] = s.hk; desc[4] = s.m;
                desc[5] = s.parts;
                desc[0] = 1;
            }
            tc_fence_before();
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 0) tmem_dealloc(tmem, 512);
}

int prefill_slots(const skvq_paged_config &cfg, const skvq_paged_batch &batch)
{
    const long long rows = (long long)batch.max_new * (cfg.n_q_heads / cfg.n_kv_heads);
    const long long items = (long long)batch.n_seqs * cfg.n_kv_heads * ((rows + 2 * kBlock - 1) / (2 * kBlock));
    const long long tiles = items * (((long long)batch.max_len + kBlock - 1) / kBlock + 1);
    long long slots = sm_count();
    if (slots > tiles / 2) slots = tiles / 2;
    return slots < 1 ? 1 : (int)slots;
}

size_t partials_bytes(const skvq_paged_config &cfg, const skvq_paged_batch &batch)
{
    const size_t slots = prefill_slots(cfg, batch);
    return slots * kDescInts * 4 + slots * 2 * (2 * kBlock) * partial_stride(cfg.head_dim) * 4;      // a multiple of 16
}

template <typename T, int D, int NG>
cudaError_t launch_prefill(const PagedAttnArgs &a, cudaStream_t stream)
{
    const skvq_paged_config &cfg = a.p.cfg;
    const skvq_paged_batch &batch = a.p.batch;
    char *ws = reinterpret_cast<char *>(a.ws) + partials_bytes(cfg, batch);
    const PrefillArgs s{a, prefill_slots(cfg, batch), reinterpret_cast<__half *>(ws), reinterpret_cast<float *>(ws + (size_t)batch.n_tokens * cfg.n_q_heads * D * 2)};
    QueryArgs q{s, cfg.n_q_heads};
    const long long tokens = (batch.max_new + kQueryTokens - 1) / kQueryTokens;
    while (q.heads > 4 && tokens * batch.n_seqs * ((cfg.n_q_heads + q.heads - 1) / q.heads) < 32LL * sm_count()) q.heads = (q.heads + 1) / 2;
    cudaError_t e = launch_chained(paged_queries_kernel<T, D>, dim3((unsigned)tokens, (cfg.n_q_heads + q.heads - 1) / q.heads, batch.n_seqs), kQueryThreads, 0, stream, q);
    if (e != cudaSuccess) return e;
    static unsigned long long done = 0;
    e = configure_smem_once(paged_prefill_kernel<T, D, NG>, PGeo<D>::SMEM + (int)sizeof(long long) * (kMaxPagedSeqs + 1), done);
    if (e != cudaSuccess) return e;
    e = launch_chained(paged_prefill_kernel<T, D, NG>, dim3(s.n_slots), kPrefillThreads, PGeo<D>::SMEM + sizeof(long long) * (batch.n_seqs + 1), stream, s);
    if (e != cudaSuccess) return e;
    return launch_paged_merge(a, s.n_slots, 2 * kBlock, 2 * kBlock / 4, kPOffset, stream);
}

template <typename T> cudaError_t prefill_by_shape(const PagedAttnArgs &a, cudaStream_t stream)
{
    if (a.p.cfg.head_dim == 128)
        return a.p.ng == 1 ? launch_prefill<T, 128, 1>(a, stream) : a.p.ng == 2 ? launch_prefill<T, 128, 2>(a, stream) : launch_prefill<T, 128, 4>(a, stream);
    return a.p.ng == 1 ? launch_prefill<T, 64, 1>(a, stream) : launch_prefill<T, 64, 2>(a, stream);
}

}  // namespace

size_t prefill_workspace_bytes(const skvq_paged_config &cfg, const skvq_paged_batch &batch)
{
    return partials_bytes(cfg, batch) + (size_t)batch.n_tokens * cfg.n_q_heads * (cfg.head_dim * 2 + 4);
}

cudaError_t launch_paged_prefill(const PagedAttnArgs &a, cudaStream_t stream)
{
    return a.p.cfg.dtype == SKVQ_F16 ? prefill_by_shape<__half>(a, stream) : prefill_by_shape<__nv_bfloat16>(a, stream);
}

}  // namespace skvq
