// skvq_paged_weights: the probabilities that a step's rows gave each token, added up per token and KV head.
//
//   w[t] += sum_r exp(sm_scale q'_r . K~_t - lse_r)
//
// The softmax denominators are given, so a token's sum needs no other token: a thread or lane owns tokens, walks over the rows, and
// nothing is joined across the context.  A first kernel lays the counted queries out once per step -- rotated, reordered, fp16 -- for
// all tiles of the cache that read them; the score of a quantized token is formed from its codes and parameters,
//   q'.K~_t = sum_g h_{t,g} (sum_{j in g} q'_j c_{t,j}) + sum_g z_{t,g} (sum_{j in g} q'_j),
// since a key rounded to fp16 would put an error of 2^-11 of its largest terms into the exponent.
#include <math_constants.h>

#include <algorithm>
#include <cmath>

#include "skvq_mma_common.cuh"
#include "skvq_paged.cuh"
#include "skvq_paged_split.cuh"
#include "skvq_tcgen05.cuh"

namespace skvq {
namespace {

using mmak::bulk_g2s;
using mmak::ex2_approx;
using mmak::mbar_arrive;
using mmak::mbar_expect_tx;
using mmak::mbar_init;
using mmak::mbar_wait_cycles;
using mmak::mma16816;
using mmak::smem_u32;
using namespace tc5;

constexpr float kCodeUnit = 1.f / 4194304.f;        // 2^-22: what a code's lowest bit stands for as an operand, four of fp16's least subnormals
constexpr float kLog2E = 1.4426950408889634f;      // applied to score - lse, which is small where it matters: their own products with it would lose 2^-24 of 20 or 30
constexpr float kZeroScale = 1.f / 1024.f;           // brings a sum of 128 operands below 2^14 into fp16's range
constexpr int kQueryThreads = 128;
constexpr int kTileRows = 128;      // rows of a query tile

// A query tile: kTileRows rows of D fp16, 64-channel halves one after the other, a half's rows 128 bytes each with 16-byte piece c of row r
// at c ^ (r & 7) (the 128-byte swizzle of the tensor core's operands); then for every two rows four floats: the factors of their scores, minus their
// lse (minus infinity: the row adds nothing).
struct WeightPlan {
    PagedWeightArgs a;
    int seq_tiles;        // > 0: sequence b's tiles begin at b * seq_tiles; 0: at starts[b] * Hq/Hkv / kTileRows + b
    int heads;            // query heads that a CTA of the first kernel walks over
    float many_scale;     // what the kernel for many rows multiplies its scores by: sm_scale, or the fp32 number above it (ManyGeo::CUT)
};
__host__ __device__ constexpr int tile_bytes(int D) { return kTileRows * (D * 2 + 8); }

// What a sequence contributes.
struct WeightSeq {
    PagedSeq s;
    int rep, m, rows;      // query heads per KV head, counted tokens, counted rows
    bool ok;
};
__device__ __forceinline__ void weight_sequence(const PagedWeightArgs &a, int b, WeightSeq &w)
{
    w.ok = paged_sequence(a.p, b, false, w.s) && w.s.slot >= 0 && w.s.slot < a.p.cfg.n_slots;
    w.rep = a.p.cfg.n_q_heads / a.p.cfg.n_kv_heads;
    w.m = a.last ? min(w.s.n, a.last) : w.s.n;
    w.rows = w.m * w.rep;
}
__device__ __forceinline__ const uint8_t *query_tile(const WeightPlan &p, const WeightSeq &w, int b, int h, int tile)
{
    const int64_t base = p.seq_tiles ? (int64_t)b * p.seq_tiles : (int64_t)w.s.row0 * w.rep / kTileRows + b;
    return p.a.ws + ((base + tile) * p.a.p.cfg.n_kv_heads + h) * tile_bytes(p.a.p.cfg.head_dim);
}

// Token t of KV head h gains `sum`; an old entry of a new token is not read.
__device__ __forceinline__ void write_weight(const PagedWeightArgs &a, const WeightSeq &w, int h, int t, float sum)
{
    const int64_t at = ((int64_t)w.s.slot * a.p.cfg.n_kv_heads + h) * a.capacity + t;
    a.w_out[at] = (a.w_in && t < w.s.len - w.s.n ? a.w_in[at] : 0.f) + sum;
}

// Position 0..7 inside a run of eight operand channels -> stored channel: nibbles i and i + 4 of a code word become neighbours.
__device__ __forceinline__ int channel_at(int pos) { return (pos >> 1) + 4 * (pos & 1); }

// The power of two that brings a row's largest magnitude to [2^13, 2^14): exact, whatever the type's range.
__device__ __forceinline__ float row_factor(float mx)
{
    return mx > 0.f ? __int_as_float((127 + min(13 - (__float_as_int(mx) >> 23) + 127, 60)) << 23) : 1.f;
}
__device__ __forceinline__ uint32_t sixteenth(uint32_t v)      // of two fp16
{
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(v), "r"(0x2C002C00u));
    return r;
}
// d = a b + c with an accumulator of its own
__device__ __forceinline__ void mma16816_from(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, float c0,
                                              float c1, float c2, float c3)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
}
__device__ __forceinline__ void load_matrices(uint32_t (&r)[4], uint32_t addr)      // four 8 x 8 matrices of 16-bit elements
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void cp16(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
// A pair of elements of the cache's type as fp16 (bf16: exact between 2^-14 and 65504, off by 2^-25 at most below).
template <typename T> __device__ __forceinline__ uint32_t as_h2(uint32_t v);
template <> __device__ __forceinline__ uint32_t as_h2<__half>(uint32_t v) { return v; }
template <> __device__ __forceinline__ uint32_t as_h2<__nv_bfloat16>(uint32_t v)
{
    return packed<__half>(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u));
}

// ------------------------------------------------------------------------------------------------ few rows: single tokens, drafts
// Sequences with at most 16 rows per KV head.  What bounds it is reading the keys' codes once; every warp works for itself.
// The (sequence, KV head) pairs are laid end to end, priced in 32-token tiles (16 tokens of the unquantized window: kRingCost), and cut into
// equal runs, one per warp.  A warp streams its tiles through a ring of its own in shared memory; 16 tokens' codes are the A
// operand of mma.m16n8k16, 8 rows the B operand, one accumulator per group.  A nibble between zeros is an fp16 subnormal, c 2^-22 (or
// 16 c 2^-22, against q/16), so codes enter the product as they are, exactly.  The product's sums keep 25 bits below the largest
// term, a subnormal counted as 2^-14, here 256 codes: moved up two bits from where a byte has them, small entries of a query then keep
// two bits more (one query over 4096 tokens, one group of 128: 5e-7 against 64 bits instead of 2.4e-6, root mean square).  The zero points' share, the sum over groups of z sum q',
// is one more product: the parameters' words {h, z} are its A operand as they lie in memory, {0, sum q'} in two fp16 parts (22 bits)
// the B operand.  With at most 4 rows they take every other column, and a lane has one row instead of two.
// Measured: a decode step of 64 sequences of 1024 to 16384 tokens, 32 heads, 295 us (4.8 TB/s); 4 sequences of 131072 tokens, 32 heads over
// 8, 85 us (4.3 TB/s); one query over 4096 tokens 9.3 us.  Instruction issue (60 % of the slots, the logic pipe half busy) and latency bound
// it together.  Steps on the way, same cases: codes as they are 377 and 115; zero points as a product, a row per lane 325 and 97; pool rows looked up
// once per block 298 and 90.  Accumulators that start at minus 8 times the group's sum (codes about their middle) cost 303 and 92 us instead of 296
// and 87 and bring these cases nothing (2.8e-8 and 2.3e-8 of all weights either way); with one group of 128 they take 9e-8 to 5e-8.
constexpr int kFewRowTile = 8;
constexpr int kTile = 32;
constexpr int kRingTile = 16;
constexpr int kRingCost = 2;
constexpr int kFewWarps = 4;
constexpr int kFewThreads = kFewWarps * 32;
constexpr int kFewStages = 3;

template <int D, int NG, int NT, int E> struct FewGeo {
    static constexpr int ROW = D / 2, CHUNKS = ROW / 16;
    static constexpr int CODES = kTile * ROW, META = kTile * NG * 4, STAGE = CODES + META;
    static constexpr int SETS = D / 32;                      // 32-channel granules: 16-byte pieces of a code row
    static constexpr int RROW = D * 2, RCHUNKS = RROW / 16;
    static constexpr int RING = kFewStages * STAGE;
    static constexpr int ROWS = kFewRowTile * NT * E / 2, QROW = D + 8;      // E rows per lane and tile: 2, or 1
    static constexpr int QUERIES = RING, RAW = QUERIES + ROWS * QROW * 2, CONSTANTS = RAW + D * 2;
    static constexpr int WARP = CONSTANTS + ROWS * (2 + NG) * 4;
    static constexpr int SMEM = kFewWarps * WARP;
    static_assert(kRingTile * RROW <= RING, "a window tile fits the warp's ring");
    static_assert(WARP % 16 == 0 && QUERIES % 16 == 0 && RAW % 16 == 0, "16-byte pieces");
};
// Position of 16-byte piece c of row t: the eight rows that a matrix load touches lie in different banks.
template <int D> __device__ __forceinline__ int piece_at(int t, int c) { return D == 128 ? c ^ ((t >> 1) & 3) : c ^ ((t >> 2) & 1); }

struct FewCost {
    int tiles_c, tiles_r, cost;
};
__device__ __forceinline__ FewCost few_cost(const PagedWeightArgs &a, const WeightSeq &w)
{
    FewCost c;
    c.tiles_c = (w.s.lq + kTile - 1) / kTile;
    c.tiles_r = (w.s.len - w.s.lq + kRingTile - 1) / kRingTile;
    c.cost = w.rows > kFewRows || (w.rows == 0 && a.w_in == a.w_out) ? 0 : c.tiles_c + kRingCost * c.tiles_r;
    return c;
}

template <int N> struct alignas(4 * N) Words { uint32_t w[N]; };

constexpr int kFewCtas = 4;      // per SM: 128 registers a thread; with 5 (spills) the serving mix took 301 us against 306, 4 x 131072 tokens 91 against 88

template <typename T, int D, int NG, int NT, int E>
__global__ void __launch_bounds__(kFewThreads, kFewCtas) weight_few_kernel(const __grid_constant__ WeightPlan plan)
{
    using Geo = FewGeo<D, NG, NT, E>;
    const PagedWeightArgs &a = plan.a;
    const PagedArgs &p = a.p;
    const skvq_paged_config &cfg = p.cfg;
    extern __shared__ __align__(128) uint8_t smem[];
    long long *pre = reinterpret_cast<long long *>(smem + Geo::SMEM);      // [n_seqs + 1] cost of the sequences before b
    __shared__ long long scan_sh[kFewWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, j = lane & 3, B = p.batch.n_seqs, H = cfg.n_kv_heads;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    // ---- the flat partition: exclusive prefix of the sequences' costs
    {
        long long carry = 0;
        for (int base = 0; base < B; base += kFewThreads) {
            const int b = base + tid;
            long long c = 0;
            if (b < B) {
                WeightSeq w;
                weight_sequence(a, b, w);
                if (w.ok) c = (long long)few_cost(a, w).cost * H;
                else if (blockIdx.x == 0) set_status(p.c.status, SKVQ_STATUS_BAD_BATCH);
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
            for (int k = 0; k < kFewWarps; ++k) {
                if (k < warp) before += scan_sh[k];
                carry += scan_sh[k];
            }
            if (b < B) pre[b] = before + incl - c;
            __syncthreads();
        }
        if (tid == 0) pre[B] = carry;
        __syncthreads();
    }
    const long long total = pre[B], runs = (long long)gridDim.x * kFewWarps, per = max((total + runs - 1) / runs, 1LL);
    long long f = ((long long)blockIdx.x * kFewWarps + warp) * per;
    const long long f1 = min(f + per, total);
    if (f >= f1) return;
    int b;
    {
        int lo = 0, hi = B - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (pre[mid] <= f) lo = mid; else hi = mid - 1;
        }
        b = lo;
    }
    uint8_t *mine = smem + warp * Geo::WARP;
    const uint32_t ring = smem_u32(mine);
    __half *queries = reinterpret_cast<__half *>(mine + Geo::QUERIES);      // [ROWS][QROW], runs of eight in the order 0 4 1 5 2 6 3 7
    T *raw = reinterpret_cast<T *>(mine + Geo::RAW);
    float *constants = reinterpret_cast<float *>(mine + Geo::CONSTANTS);    // [ROWS][2 + NG]: factor, minus lse, sums of the groups
    const int P = cfg.page_tokens, page_shift = __ffs(P) - 1;

    while (f < f1) {
        while (pre[b + 1] <= f) ++b;
        WeightSeq w;
        weight_sequence(a, b, w);
        const FewCost fc = few_cost(a, w);
        const int item = (int)((f - pre[b]) / fc.cost), off = (int)(f - pre[b] - (long long)item * fc.cost), hk = item;
        const int take = (int)min((long long)(fc.cost - off), f1 - f);
        f += take;
        const int L = w.s.len, lq = w.s.lq, R = w.rows, fresh = L - w.s.n;      // tokens at or beyond `fresh` are new
        auto tile_of = [&](int x) { return x <= fc.tiles_c ? x : fc.tiles_c + (x - fc.tiles_c + kRingCost - 1) / kRingCost; };
        const int seg0 = tile_of(off), seg1 = tile_of(off + take);
        const int q0 = min(seg0, fc.tiles_c), q1 = min(seg1, fc.tiles_c), r0 = max(seg0, fc.tiles_c), r1 = max(seg1, fc.tiles_c);
        const int64_t weight_row = ((int64_t)w.s.slot * H + hk) * a.capacity;
        const float *w_in = a.w_in ? a.w_in + weight_row : nullptr;
        float *w_out = a.w_out + weight_row;
        auto old_weight = [&](int t) { return w_in && t < fresh ? w_in[t] : 0.f; };
        if (R == 0) {
            for (int t = q0 * kTile + lane; t < min(q1 * kTile, lq); t += 32) w_out[t] = old_weight(t);
            for (int t = lq + (r0 - fc.tiles_c) * kRingTile + lane; t < min(lq + (r1 - fc.tiles_c) * kRingTile, L); t += 32) w_out[t] = old_weight(t);
            continue;
        }
        const int32_t *table = p.batch.page_table + (int64_t)b * p.batch.max_pages;
        // The pool's row of the first token of 32 consecutive 16-token blocks, one per lane; negative past the quantized tokens and
        // for an id outside the pool.
        auto load_pages = [&](int block) {
            const int t = (block + lane) * 16;
            long long row = -1;
            if (t < lq) {
                const int id = table[t >> page_shift];
                if (id >= 0 && id < cfg.n_pages) row = ((long long)id * H + hk) * P + (t & (P - 1));
                else set_status(p.c.status, SKVQ_STATUS_BAD_PAGE);
            }
            return row;
        };
        int block = q0 * 2 & 31;      // the next tile's first block among the 32
        long long pages = -1, pages_next = -1;
        if (q0 < q1) {
            pages = load_pages(q0 * 2 - block);
            pages_next = load_pages(q0 * 2 - block + 32);
        }
        uint32_t bad = 0;      // bit 2 * stage + block: the block has no page
        const uint8_t *codes_src = static_cast<const uint8_t *>(p.c.k_codes) + lane * 16, *meta_src = static_cast<const uint8_t *>(p.c.k_meta) + lane * 16;
        const uint32_t codes_dst = ring + (lane / Geo::CHUNKS) * Geo::ROW + piece_at<D>(lane / Geo::CHUNKS, lane % Geo::CHUNKS) * 16, meta_dst = ring + Geo::CODES + lane * 16;
        auto fetch = [&](int tile, int stage) {
            if (tile < q1) {
                if (block == 32) {
                    block = 0;
                    pages = pages_next;
                    pages_next = load_pages(tile * 2 + 32);
                }
                bad &= ~(3u << (2 * stage));
                constexpr int HALF = Geo::CHUNKS / 2, STEP = 32 / Geo::CHUNKS;      // copies of a block; rows that one covers
                static_assert(STEP % 8 == 0, "the pieces' places repeat every eight rows");
#pragma unroll
                for (int blk = 0; blk < 2; ++blk) {
                    const long long row = __shfl_sync(0xffffffffu, pages, block + blk);
                    if (row >= 0) {
#pragma unroll
                        for (int k = 0; k < HALF; ++k)
                            cp16(codes_dst + stage * Geo::STAGE + (16 * blk + k * STEP) * Geo::ROW, codes_src + row * Geo::ROW + k * 512);
                        if (lane < 4 * NG) cp16(meta_dst + stage * Geo::STAGE + blk * (64 * NG), meta_src + row * (NG * 4));
                    } else {
                        bad |= 1u << (2 * stage + blk);
                    }
                }
                block += 2;
            }
            cp_commit();
        };
#pragma unroll
        for (int k = 0; k < kFewStages - 1; ++k) fetch(q0 + k, k);

        // ---- the rows: rotate, round to T, reorder, fp16 times a power of two; the sums of the groups
        {
            constexpr int C = D / 32;
            const float2 *rope = static_cast<const float2 *>(p.rope.table);
            const int half = p.rope.rot_dim / 2;
            int from[C];
#pragma unroll
            for (int k = 0; k < C; ++k) {
                const int pos = lane * C + k, c = (pos & ~7) + channel_at(pos & 7);
                from[k] = p.c.reorder_k ? p.c.reorder_k[hk * D + c] & (D - 1) : c;
            }
#pragma unroll 1
            for (int r = 0; r < Geo::ROWS; ++r) {
                if (r >= R) {
                    if constexpr (C == 4) *reinterpret_cast<uint2 *>(queries + r * Geo::QROW + lane * C) = make_uint2(0u, 0u);
                    else *reinterpret_cast<uint32_t *>(queries + r * Geo::QROW + lane * C) = 0u;
                    if (lane < 2 + NG) constants[r * (2 + NG) + lane] = lane == 1 ? -CUDART_INF_F : 0.f;
                    continue;
                }
                const int i = r / w.rep, head = hk * w.rep + r - i * w.rep, pos = L - w.m + i;
                const int64_t tok = w.s.row0 + w.s.n - w.m + i;
                const T *src = static_cast<const T *>(a.q) + tok * a.q_stride + (int64_t)head * D;
                const float lse = a.lse[tok * cfg.n_q_heads + head];
                __syncwarp();
#pragma unroll
                for (int k = 0; k < C; ++k) {
                    const int c = lane + 32 * k;
                    T x = src[c];
                    if (rope && c < p.rope.rot_dim && pos >= 0) {
                        const bool second = p.rope.interleaved ? c & 1 : c >= half;
                        const int at = p.rope.interleaved ? c >> 1 : (second ? c - half : c), partner = p.rope.interleaved ? c ^ 1 : (second ? c - half : c + half);
                        const float2 cs = rope[(int64_t)pos * half + at];
                        const float own = Elem<T>::to_float(x), other = Elem<T>::to_float(src[partner]);
                        x = Elem<T>::from_float(second ? rotate_second(other, own, cs.x, cs.y) : rotate_first(own, other, cs.x, cs.y));
                    }
                    raw[c] = x;
                }
                __syncwarp();
                float x[C], mx = 0.f, sum = 0.f;
                bool finite = fabsf(lse) < CUDART_INF_F;
#pragma unroll
                for (int k = 0; k < C; ++k) {
                    x[k] = Elem<T>::to_float(raw[from[k]]);
                    mx = fmaxf(mx, fabsf(x[k]));
                    finite = finite && fabsf(x[k]) < CUDART_INF_F;
                }
                const bool counts = __all_sync(0xffffffffu, finite);
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
                const float up = counts ? row_factor(mx) : 0.f;
                uint32_t v[C / 2];
#pragma unroll
                for (int k = 0; k < C; k += 2) {
                    v[k / 2] = counts ? packed<__half>(x[k] * up, x[k + 1] * up) : 0u;
                    const float2 q = floats<__half>(v[k / 2]);
                    sum += q.x + q.y;
                }
#pragma unroll
                for (int d = 1; d < 32 / NG; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
                if constexpr (C == 4) *reinterpret_cast<uint2 *>(queries + r * Geo::QROW + lane * C) = make_uint2(v[0], v[1]);
                else *reinterpret_cast<uint32_t *>(queries + r * Geo::QROW + lane * C) = v[0];
                if (lane == 0) {
                    constants[r * (2 + NG)] = counts ? a.sm_scale / up : 0.f;
                    constants[r * (2 + NG) + 1] = counts ? -lse : -CUDART_INF_F;
                }
                if (lane % (32 / NG) == 0) constants[r * (2 + NG) + 2 + lane / (32 / NG)] = sum;
            }
            __syncwarp();
        }
        // column g of tile n is row 8 n + g, or, E = 1, row g / 2 where g is even; a lane's columns of the result are 2 j and 2 j + 1
        uint32_t bq[NT][Geo::SETS * 2][2], bz[NT][2];
        float rs[NT][E], nl[NT][E];
        int lim[NT][E];      // this lane's rows see tokens below it
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int r = E == 2 ? 8 * n + g : g >> 1;
            const bool column = E == 2 || g % 2 == 0;
#pragma unroll
            for (int st = 0; st < Geo::SETS; ++st) {
                uint4 x = *reinterpret_cast<const uint4 *>(queries + r * Geo::QROW + 32 * st + 8 * j);
                if (!column) x = make_uint4(0u, 0u, 0u, 0u);
                bq[n][2 * st][0] = x.x;
                bq[n][2 * st][1] = sixteenth(x.y);
                bq[n][2 * st + 1][0] = x.z;
                bq[n][2 * st + 1][1] = sixteenth(x.w);
            }
            const float q = column && j < NG ? constants[r * (2 + NG) + 2 + j] * kZeroScale : 0.f;      // of group j
            const float high = __half2float(__float2half_rn(q));
            bz[n][0] = packed<__half>(0.f, high);
            bz[n][1] = packed<__half>(0.f, q - high);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int own = E == 2 ? 8 * n + 2 * j + e : j;
                rs[n][e] = constants[own * (2 + NG)] * (1.f / kZeroScale);
                nl[n][e] = constants[own * (2 + NG) + 1];
                lim[n][e] = a.causal ? min(L, L - w.m + min(own, R - 1) / w.rep + 1) : L;
            }
        }
        const int lowest = a.causal ? min(L, L - w.m + 1) : L;      // the first row's limit

        // ---- quantized tokens
        int stage = 0;
        const uint32_t matrix_row = (lane & 7) + ((lane >> 3) & 1) * 8, matrix_piece = lane >> 4;      // what this lane's address stands for in a load of four matrices
        float old_next = q0 < q1 && q0 * kTile + 8 * j + g < lq ? old_weight(q0 * kTile + 8 * j + g) : 0.f;
#pragma unroll 1
        for (int tile = q0; tile < q1; ++tile) {
            fetch(tile + kFewStages - 1, stage == 0 ? kFewStages - 1 : stage - 1);
            const int t0 = tile * kTile, own = t0 + 8 * j + g;
            const float old = old_next;
            if (tile + 1 < q1) old_next = own + kTile < lq ? old_weight(own + kTile) : 0.f;
            cp_wait<kFewStages - 1>();
            __syncwarp();
            const uint32_t buf = ring + stage * Geo::STAGE;
            const uint32_t *km = reinterpret_cast<const uint32_t *>(mine + stage * Geo::STAGE + Geo::CODES);
            const uint32_t bad_here = (bad >> (2 * stage)) & 3u;
            const bool edge = t0 + kTile > min(lq, lowest) || bad_here;      // some row or some token of the tile is masked
            float sums[2][2];      // tokens 16 u + g and 16 u + 8 + g
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                float acc[NT][NG][4], zero[NT][4];
                {
                    const int group = NG == 4 ? j : j % NG;
                    const uint32_t x = km[(16 * u + g) * NG + group], y = km[(16 * u + 8 + g) * NG + group];
#pragma unroll
                    for (int n = 0; n < NT; ++n) mma16816_from(zero[n], x, y, x, y, bz[n][0], bz[n][1], 0.f, 0.f, 0.f, 0.f);
                }
#pragma unroll
                for (int s2 = 0; s2 < Geo::SETS; s2 += 2) {
                    const int row = 16 * u + matrix_row;
                    uint32_t c[4];      // words of tokens g and g + 8, granule s2; the same of granule s2 + 1
                    load_matrices(c, buf + row * Geo::ROW + piece_at<D>(row, s2 + matrix_piece) * 16);
#pragma unroll
                    for (int h2 = 0; h2 < 2; ++h2) {
                        const int st = s2 + h2;
                        constexpr int PER = Geo::SETS / NG;      // granules per group
                        const uint32_t x = c[2 * h2] << 2, y = c[2 * h2 + 1] << 2, xs = c[2 * h2] >> 6, ys = c[2 * h2 + 1] >> 6;
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            float (&d)[4] = acc[n][st / PER];
                            const uint32_t x0 = x & 0x003C003Cu, y0 = y & 0x003C003Cu, x1 = x & 0x03C003C0u, y1 = y & 0x03C003C0u;
                            if (st % PER == 0) mma16816_from(d, x0, y0, x1, y1, bq[n][2 * st][0], bq[n][2 * st][1], 0.f, 0.f, 0.f, 0.f);
                            else mma16816(d, x0, y0, x1, y1, bq[n][2 * st][0], bq[n][2 * st][1]);
                            mma16816(d, xs & 0x003C003Cu, ys & 0x003C003Cu, xs & 0x03C003C0u, ys & 0x03C003C0u, bq[n][2 * st + 1][0], bq[n][2 * st + 1][1]);
                        }
                    }
                }
                float s[2][NT][E];
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    float h[NG];
                    {
                        const Words<NG> m = reinterpret_cast<const Words<NG> *>(km)[16 * u + 8 * half + g];
#pragma unroll
                        for (int k = 0; k < NG; ++k) h[k] = floats<__half>(m.w[k]).x;
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < E; ++e) {
                            float x = h[0] * acc[n][0][2 * half + e];
#pragma unroll
                            for (int k = 1; k < NG; ++k) x = fmaf(h[k], acc[n][k][2 * half + e], x);
                            s[half][n][e] = fmaf(fmaf(x, kZeroScale / kCodeUnit, zero[n][2 * half + e]), rs[n][e], nl[n][e]) * kLog2E;
                        }
                }
                if (edge) {
#pragma unroll
                    for (int half = 0; half < 2; ++half)
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int e = 0; e < E; ++e)
                                if (t0 + 16 * u + 8 * half + g >= min(lq, lim[n][e]) || ((bad_here >> u) & 1u)) s[half][n][e] = -CUDART_INF_F;
                }
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    sums[u][half] = 0.f;
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < E; ++e) sums[u][half] += ex2_approx(s[half][n][e]);
                }
            }
            // lane (g, j) gets token 8 j + g, added up over the lanes that hold the other rows
            {
                const bool hi = j & 2, odd = j & 1;
                float x0 = hi ? sums[1][0] : sums[0][0], x1 = hi ? sums[1][1] : sums[0][1];
                x0 += __shfl_xor_sync(0xffffffffu, hi ? sums[0][0] : sums[1][0], 2);
                x1 += __shfl_xor_sync(0xffffffffu, hi ? sums[0][1] : sums[1][1], 2);
                const float x = (odd ? x1 : x0) + __shfl_xor_sync(0xffffffffu, odd ? x0 : x1, 1);
                if (own < lq) w_out[own] = old + x;
            }
            __syncwarp();
            stage = stage + 1 == kFewStages ? 0 : stage + 1;
        }
        cp_wait<0>();
        __syncwarp();

        // ---- the window: 16-bit rows, 16 tokens at a time through the warp's ring
        const int64_t win_row0 = ((int64_t)w.s.slot * H + hk) * cfg.ring_tokens;
#pragma unroll 1
        for (int tile = r0; tile < r1; ++tile) {
            const int t0 = lq + (tile - fc.tiles_c) * kRingTile;
            int id = 0;
            if (lane < kRingTile && t0 + lane < L) id = table[(t0 + lane) >> page_shift];
            constexpr int STEP = 32 / Geo::RCHUNKS;
            const int c = lane % Geo::RCHUNKS, first = t0 % cfg.ring_tokens;
            const uint8_t *kw = static_cast<const uint8_t *>(p.c.k_win) + win_row0 * Geo::RROW + c * 16;
#pragma unroll
            for (int k = 0; k < kRingTile / STEP; ++k) {
                const int t = k * STEP + lane / Geo::RCHUNKS;
                if (t0 + t < L) {
                    int row = first + t;      // the window is no longer than the ring: it wraps once at most
                    if (row >= cfg.ring_tokens) row -= cfg.ring_tokens;
                    cp16(ring + t * Geo::RROW + (c ^ (t & 7)) * 16, kw + (int64_t)row * Geo::RROW);
                }
            }
            cp_commit();
            const int tok = t0 + g + 8 * (j & 1);      // of lanes j = 0 and 1
            const float old = j < 2 && tok < L ? old_weight(tok) : 0.f;
            const bool none = id < 0 || id >= cfg.n_pages;
            if (none) set_status(p.c.status, SKVQ_STATUS_BAD_PAGE);
            const uint32_t gone = __ballot_sync(0xffffffffu, none);
            cp_wait<0>();
            __syncwarp();
            float s[NT][4];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[n][e] = 0.f;
#pragma unroll
            for (int st = 0; st < Geo::SETS; ++st) {
                uint32_t x[2][4];
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    uint4 v = *reinterpret_cast<const uint4 *>(mine + (g + 8 * half) * Geo::RROW + ((4 * st + j) ^ g) * 16);
                    v.x = as_h2<T>(v.x); v.y = as_h2<T>(v.y); v.z = as_h2<T>(v.z); v.w = as_h2<T>(v.w);
                    x[half][0] = __byte_perm(v.x, v.z, 0x5410); x[half][1] = __byte_perm(v.x, v.z, 0x7632);
                    x[half][2] = __byte_perm(v.y, v.w, 0x5410); x[half][3] = __byte_perm(v.y, v.w, 0x7632);
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    uint4 q = *reinterpret_cast<const uint4 *>(queries + (E == 2 ? 8 * n + g : g >> 1) * Geo::QROW + 32 * st + 8 * j);
                    if (E == 1 && g % 2) q = make_uint4(0u, 0u, 0u, 0u);
                    mma16816(s[n], x[0][0], x[1][0], x[0][1], x[1][1], q.x, q.y);
                    mma16816(s[n], x[0][2], x[1][2], x[0][3], x[1][3], q.z, q.w);
                }
            }
            float sums[2] = {0.f, 0.f};
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int half = 0; half < 2; ++half)
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const int at = g + 8 * half;
                        const bool hidden = t0 + at >= lim[n][e] || ((gone >> at) & 1u);      // rows behind the last token were not copied
                        sums[half] += hidden ? 0.f : ex2_approx(fmaf(s[n][2 * half + e], rs[n][e] * kZeroScale, nl[n][e]) * kLog2E);
                    }
            const bool odd = j & 1;
            float x = (odd ? sums[1] : sums[0]) + __shfl_xor_sync(0xffffffffu, odd ? sums[0] : sums[1], 1);
            x += __shfl_xor_sync(0xffffffffu, x, 2);
            if (j < 2 && tok < L) w_out[tok] = old + x;
            __syncwarp();
        }
    }
}

// ------------------------------------------------------------------------------------------------ many rows: prompts and chunks
// D / 8 lanes own a row; they take a token and walk over heads with the token's angles in registers.
template <typename T, int D>
__global__ void __launch_bounds__(kQueryThreads) weight_queries_kernel(const __grid_constant__ WeightPlan plan)
{
    using R = Row<T, 128>;      // 8 channels a lane, whatever D is
    constexpr int C = R::C, LANES = D / C, TOKENS = kQueryThreads / LANES;
    __shared__ __align__(16) T rows[TOKENS][2][D + 8];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const PagedWeightArgs &a = plan.a;
    const PagedArgs &p = a.p;
    const int unit = threadIdx.x / LANES, sub = threadIdx.x % LANES, c0 = sub * C, b = blockIdx.z;
    WeightSeq w;
    weight_sequence(a, b, w);
    if (!w.ok || w.rows <= kFewRows) return;
    const int filled = (w.rows + kTileRows - 1) / kTileRows * kTileRows;      // zeros behind the last row: tiles are read whole
    if ((int)blockIdx.x * TOKENS * w.rep >= filled) return;
    const int i = blockIdx.x * TOKENS + unit, pos = w.s.len - w.m + i;
    const int h0 = blockIdx.y * plan.heads, h1 = min(h0 + plan.heads, p.cfg.n_q_heads);
    const bool have = i < w.m, turn = p.rope.table && have && pos >= 0;
    const int64_t tok = w.s.row0 + w.s.n - w.m + i;
    float2 cs[C];
    if (turn) load_angles(cs, p.rope, pos, c0);
    const T *src = static_cast<const T *>(a.q) + tok * a.q_stride + c0;
    T *raw = rows[unit][0], *turned = rows[unit][1];
    int from[C], hk = -1;
    R next;
    float lse_next = CUDART_INF_F;
#pragma unroll
    for (int k = 0; k < R::WORDS; ++k) next.w[k] = 0u;
    if (have && h0 < h1) {
        next.load(src + (int64_t)h0 * D);
        lse_next = a.lse[tok * p.cfg.n_q_heads + h0];
    }
    for (int h = h0; h < h1; ++h) {
        if (h / w.rep != hk) {
            hk = h / w.rep;
#pragma unroll
            for (int j = 0; j < C; ++j) {
                const int c = c0 + channel_at(j);
                from[j] = p.c.reorder_k ? p.c.reorder_k[hk * D + c] & (D - 1) : c;
            }
        }
        R row = next;
        const float lse = lse_next;
        if (have && h + 1 < h1) {
            next.load(src + (int64_t)(h + 1) * D);
            lse_next = a.lse[tok * p.cfg.n_q_heads + h + 1];
        }
        if (p.rope.table) {
            if (!p.rope.interleaved) {
                row.store(raw + c0);
                __syncwarp();
            }
            if (turn) rotate_row<T, 128>(row, c0, cs, raw, p.rope.rot_dim, p.rope.interleaved);
        }
        row.store(turned + c0);
        __syncwarp();
        float x[C];
        uint32_t mx = 0u;      // the largest magnitude's bits: those of infinities and of what is no number are larger still
#pragma unroll
        for (int j = 0; j < C; ++j) {
            x[j] = Elem<T>::to_float(turned[from[j]]);
            mx = max(mx, __float_as_uint(x[j]) & 0x7FFFFFFFu);
        }
#pragma unroll
        for (int d = 1; d < LANES; d <<= 1) mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, d));
        const bool counts = mx < 0x7F800000u && fabsf(lse) < CUDART_INF_F;
        const float up = counts ? row_factor(__uint_as_float(mx)) : 1.f;
#pragma unroll
        for (int j = 0; j < C; ++j) x[j] = counts ? x[j] * up : 0.f;
        const int r = i * w.rep + h - hk * w.rep;
        if (r >= filled) continue;
        uint8_t *tile = const_cast<uint8_t *>(query_tile(plan, w, b, hk, r / kTileRows));
        const int tr = r % kTileRows;
        *reinterpret_cast<uint4 *>(tile + (c0 >> 6) * kTileRows * 128 + tr * 128 + ((((c0 >> 3) & 7) ^ (tr & 7)) << 4)) =
            make_uint4(packed<__half>(x[0], x[1]), packed<__half>(x[2], x[3]), packed<__half>(x[4], x[5]), packed<__half>(x[6], x[7]));
        if (sub == 0) {
            float *constants = reinterpret_cast<float *>(tile + kTileRows * D * 2) + (tr >> 1) * 4 + (tr & 1);
            constants[0] = plan.many_scale * __uint_as_float((254u << 23) - __float_as_uint(up));      // divided by the power of two
            constants[2] = counts ? -lse : -CUDART_INF_F;
        }
    }
}

// One CTA per SM works on items: 256 tokens of a KV head (two blocks of 128, a token per lane of the tensor memory) and the query tiles
// that see them.  Transposed scores, S^T = K~ Q^T: a token's sum over the rows then stays in one thread.  Roles, ordered by mbarriers:
//   dequantizers  4 warps, two tokens per thread: the key as fp32 h c + z, split into fp16 high and low parts (2^-22 together), both
//                 into tensor memory as the A operand: 2 D columns of K for a product whose B operand, the queries, is read from
//                 shared memory alone.
//   loader        a thread brings query tiles with their rows' constants into a ring, one bulk copy each (they are laid out for it).
//   issuer        a warp: S = (low + high) Q^T of a block and a tile; the products of one block run while the other's scores become
//                 probabilities.
//   exponentials  2 x 4 warps, a block each: scores from tensor memory, exp(factor s - lse), their sum.
// Measured: 2048 queries at the end of 32k tokens, 32 heads over 8, D = 128: 785 us, 0.68 PFLOP/s of scores and twice that of products; ragged
// prompts up to 4095 tokens, 32 heads of 64: 360 us, of it 65 for the queries; four prompts of 8192 tokens judged by 32 queries 59 us.  The products
// bound it: about 85 clocks for 128 x 128 x 16 with A in tensor memory, 690 us without any exponentials.  Tried: 64 rows a time with two buffers a
// block 900, the two blocks' products in turn 779 but the prompts 384; a quarter of the exponentials by multiply-adds 843; 16 warps of
// exponentials 785, prompts 387; exact codes with an accumulator per group, half the products, 1009: the parameters' fp32 arithmetic, seven
// paired instructions a pair of scores, costs more than the product saves.
// Items are laid end to end, priced in query tiles (causal limits included), and cut into equal runs, one per CTA; partial sums of an
// item that several runs share are added in order by a last kernel.
constexpr int kBlock = 128;                            // tokens of a block, rows of a query tile
constexpr int kItemTokens = 2 * kBlock;
constexpr int kExpThreads = 2 * kBlock;                // warps 0-7
constexpr int kManyThreads = kExpThreads + kBlock + 64;      // warps 8-11 dequantize, 12 issues, 13 loads
constexpr int kManyDesc = 8;                           // ints of a run's descriptor

struct ManyArgs {
    WeightPlan plan;
    int n_slots;
    uint8_t *shares;      // [n_slots][kManyDesc] ints, then [n_slots][2][kItemTokens] floats: a run's share of an item it continues (0), of one it begins (1)
};

template <int D> struct ManyGeo {
    static constexpr int TILE = tile_bytes(D);
    static constexpr int STAGES = D == 128 ? 4 : 6;
    static constexpr int SMEM = STAGES * TILE + 1024;            // and room to align to 1024 bytes
    static constexpr int HALF_BYTES = kBlock * 128;              // 64 channels of a tile
    static constexpr int A_COLUMNS = D;                          // of a block: high parts, low parts, two to a column
    static constexpr int A_BUFFERS = D == 128 ? 1 : 2;           // what 512 columns leave room for
    static constexpr int TMEM_S = 0, TMEM_A = 256;               // columns: S 2 blocks x 128 rows
    // The tensor core cuts its sums toward zero, after each of the D / 16 products: on average a score is too small by this share of itself (measured,
    // queries and keys with outliers, groups of 32 to 128).  Rounding the scale after adding the share to it leaves 0.3 of 2^-24 at sm_scale = 128^-1/2, and at
    // most half of fp32's step wherever the scale lies; the chunk below is off by 4.9e-7 so against 64 bits, 1.03e-6 without, 6.4e-7 the plain form in fp32.
    static constexpr float CUT = (D == 128 ? 1.1f : 0.8f) / 16777216.f;
};

// The items of one sequence: per KV head, 256 tokens each; query tiles that they look at.
struct ManyItems {
    int rep, m, len, base, rows, steps, causal, tiles;
    __device__ __forceinline__ void set(const PagedWeightArgs &a, const WeightSeq &w)
    {
        rep = w.rep;
        m = w.m;
        len = w.s.len;
        base = len - m;
        rows = w.rows;
        steps = (rows + kTileRows - 1) / kTileRows;
        causal = a.causal;
        tiles = rows > kFewRows ? (len + kItemTokens - 1) / kItemTokens : 0;      // the others are the other kernel's
    }
    // the first row that sees token t (of a causal step)
    __device__ __forceinline__ int first_row(int t) const { return causal ? max(t - base, 0) * rep : 0; }
    __device__ __forceinline__ int first_step(int tile) const { return first_row(tile * kItemTokens) / kTileRows; }
    __device__ __forceinline__ int cost(int tile) const { return steps - first_step(tile); }
    // tiles that all steps look at
    __device__ __forceinline__ int whole() const { return !causal ? tiles : base < 0 ? 0 : min(tiles, base / kItemTokens + 1); }
    __device__ __forceinline__ long long total() const
    {
        long long c = (long long)whole() * steps;
        for (int tile = whole(); tile < tiles; ++tile) c += cost(tile);
        return c;
    }
};

// What a role works on: steps [s0, s1) of tile `tile` of KV head h of sequence b.  In shared memory: in registers it would spill.
struct ManySegment {
    long long f, f1;      // what is left of the CTA's run
    int valid, b, h, tile, s0, s1, whole, begins, parts;
    WeightSeq w;
    ManyItems it;
};
__device__ __noinline__ void next_segment(const ManyArgs &args, const long long *pre, long long per, ManySegment &s)
{
    const PagedWeightArgs &a = args.plan.a;
    const long long f = s.f;
    if (f >= s.f1) { s.valid = 0; return; }
    int b = s.b;
    while (pre[b + 1] <= f) ++b;
    WeightSeq w;
    ManyItems it;
    weight_sequence(a, b, w);
    it.set(a, w);
    const long long per_head = (pre[b + 1] - pre[b]) / a.p.cfg.n_kv_heads;
    long long at = f - pre[b];
    const int h = (int)(at / per_head);
    at -= h * per_head;
    const int full = it.whole();
    int tile = (int)min(at / it.steps, (long long)full);
    at -= (long long)tile * it.steps;
    int c = it.steps;
    if (tile >= full) {
        c = it.cost(tile);
        while (at >= c) { at -= c; c = it.cost(++tile); }
    }
    const int take = (int)min((long long)(c - at), s.f1 - f);
    s.b = b;
    s.h = h;
    s.tile = tile;
    s.s0 = it.steps - c + (int)at;
    s.s1 = s.s0 + take;
    s.begins = at == 0;
    s.whole = at == 0 && take == c;
    s.parts = (int)((f - at + c - 1) / per - blockIdx.x + 1);
    s.w = w;
    s.it = it;
    s.f = f + take;
    s.valid = 1;
}

// Thirty-two scores of a thread's token -> their probabilities' sum.  `constants`: {factor, factor, -lse, -lse} of two rows.  EDGE: rows
// below `hidden` do not see the token.
template <bool EDGE> __device__ __forceinline__ float sum_probabilities(const float (&x)[32], const float4 *constants, int hidden)
{
    uint64_t l0 = 0ull, l1 = 0ull;
#pragma unroll
    for (int c = 0; c < 32; c += 2) {
        const float4 k = constants[c / 2];
        float a, b;
        unpair(pair_mul(pair_fma(pair(x[c], x[c + 1]), pair(k.x, k.y), pair(k.z, k.w)), pair(kLog2E, kLog2E)), a, b);
        a = ex2_approx(a);
        b = ex2_approx(b);
        if (EDGE && c < hidden) a = 0.f;
        if (EDGE && c + 1 < hidden) b = 0.f;
        if (c & 2) l1 = pair_add(l1, pair(a, b));
        else l0 = pair_add(l0, pair(a, b));
    }
    float a, b;
    unpair(pair_add(l0, l1), a, b);
    return a + b;
}

template <typename T, int D, int NG>
__global__ void __launch_bounds__(kManyThreads, 1) weight_many_kernel(const __grid_constant__ ManyArgs args)
{
    using Geo = ManyGeo<D>;
    const PagedWeightArgs &a = args.plan.a;
    const PagedArgs &p = a.p;
    const skvq_paged_config &cfg = p.cfg;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    long long *pre = reinterpret_cast<long long *>(smem + Geo::STAGES * Geo::TILE);
    __shared__ __align__(8) uint64_t bars[2 * Geo::STAGES + 8];
    __shared__ uint32_t tmem_sh;
    __shared__ int fail_sh;
    __shared__ long long scan_sh[16];
    __shared__ ManySegment seg_sh[5];      // of the two blocks' exponentials, of the dequantizers, the issuer, the loader
    const int tid = threadIdx.x, lane = tid & 31, B = p.batch.n_seqs, H = cfg.n_kv_heads;
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);

    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");

    // ---- the flat partition
    {
        long long carry = 0;
        for (int base = 0; base < B; base += kManyThreads) {
            const int b = base + tid;
            long long c = 0;
            if (b < B) {
                WeightSeq w;
                weight_sequence(a, b, w);
                if (w.ok) {      // the kernel for few rows reports the others
                    ManyItems it;
                    it.set(a, w);
                    c = it.total() * H;
                }
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
            for (int w = 0; w < kManyThreads / 32; ++w) {
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
    const uint32_t q_full = bar0, q_empty = bar0 + 8 * Geo::STAGES;      // + 8 * stage
    const uint32_t s_full = bar0 + 16 * Geo::STAGES, s_empty = s_full + 16;      // + 8 * block
    const uint32_t a_full = s_full + 32, a_empty = s_full + 48;          // + 8 * buffer
    __shared__ __align__(8) uint64_t drained_sh;
    const uint32_t drained = smem_u32(&drained_sh);
    if (tid == 0) {
#pragma unroll
        for (int i = 0; i < Geo::STAGES; ++i) {
            mbar_init(q_full + 8 * i, 1);
            mbar_init(q_empty + 8 * i, 1 + kExpThreads / 32);      // the products, and a warp each that has read its constants
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            mbar_init(s_full + 8 * i, 1);
            mbar_init(s_empty + 8 * i, 4);
            mbar_init(a_full + 8 * i, kBlock);
            mbar_init(a_empty + 8 * i, 1);
        }
        mbar_init(drained, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fail_sh = 0;
    }
    if (warp == 0) tmem_alloc(smem_u32(&tmem_sh), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_sh;
    const long long total = pre[B], per = max((total + args.n_slots - 1) / args.n_slots, 1LL);
    int *desc = reinterpret_cast<int *>(args.shares) + (size_t)blockIdx.x * kManyDesc;
    if (tid < 5) {
        ManySegment &first = seg_sh[tid];
        first.f = blockIdx.x * per;
        first.f1 = min(first.f + per, total);
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
    // follows from it, so that who has read spoilt operands finds it set when it comes to write its sums.
    bool alive = true;
    volatile int *fail = &fail_sh;
    auto wait = [&](uint32_t bar, uint32_t parity) {      // by whole warps
        if (alive && !mbar_wait_cycles(bar, parity)) {
            alive = false;
            *fail = 1;
            set_status(p.c.status, SKVQ_STATUS_COPY_TIMEOUT);
        }
    };
    // A role is 128 threads (block 0, block 1, the dequantizers) or a warp (issuer, loader).
    const int role = warp < 12 ? warp >> 2 : warp - 9;
    const ManySegment &s = seg_sh[role];
    auto role_sync = [&]() {
        if (warp < 12) asm volatile("bar.sync %0, 128;" ::"r"(1 + role) : "memory");
        else __syncwarp();
    };
    auto next = [&]() {
        role_sync();
        if ((warp < 12 ? tid & 127 : lane) == 0) next_segment(args, pre, per, seg_sh[role]);
        role_sync();
        return s.valid != 0;
    };
    // rows of step `step` come as one or two halves of 64
    auto halves = [&](int step) { return s.it.rows - step * kTileRows > 64 ? 2 : 1; };

    if (warp >= 8 && warp < 12) {
        // ================================================================ dequantizers
        const int row = tid - kExpThreads, P = cfg.page_tokens, page_shift = __ffs(P) - 1;
        const uint32_t quad = (uint32_t)((warp & 3) * 32) << 16;
        uint32_t n = 0;      // segments so far
        while (next()) {
            if (*fail) alive = false;
            const uint32_t buf = n % Geo::A_BUFFERS, use = n / Geo::A_BUFFERS;
            if (use) wait(a_empty + 8 * buf, (use - 1) & 1);
            tc_fence_after();
            const int32_t *table = p.batch.page_table + (int64_t)s.b * p.batch.max_pages;
#pragma unroll 1
            for (int blk = 0; blk < 2; ++blk) {
                const int t = s.tile * kItemTokens + blk * kBlock + row;
                const uint32_t dst = tmem + Geo::TMEM_A + (buf * 2 + blk) * Geo::A_COLUMNS + quad;
                int page = -1;
                if (t < s.w.s.len) {
                    page = table[t >> page_shift];
                    if (page < 0 || page >= cfg.n_pages) { page = -1; set_status(p.c.status, SKVQ_STATUS_BAD_PAGE); }
                }
                const bool codes = page >= 0 && t < s.w.s.lq, window = page >= 0 && !codes;
                const int64_t at = codes ? ((int64_t)page * H + s.h) * P + (t & (P - 1)) : 0;
                const int64_t ring = window ? ((int64_t)s.w.s.slot * H + s.h) * cfg.ring_tokens + t % cfg.ring_tokens : 0;
                const uint4 *code_row = reinterpret_cast<const uint4 *>(static_cast<const uint8_t *>(p.c.k_codes) + at * (D / 2));
                const uint4 *ring_row = reinterpret_cast<const uint4 *>(static_cast<const T *>(p.c.k_win) + ring * D);
                uint4 c[D / 32];
                uint32_t meta[NG];
#pragma unroll
                for (int i = 0; i < D / 32; ++i) c[i] = codes ? code_row[i] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                for (int g = 0; g < NG; ++g) meta[g] = codes ? static_cast<const uint32_t *>(p.c.k_meta)[at * NG + g] : 0u;
                // 32 channels at a time, operand order 0 4 1 5 2 6 3 7 in every run of eight: 16 columns of high parts, 16 of low ones
#pragma unroll
                for (int i = 0; i < D / 32; ++i) {
                    const float2 hz = floats<__half>(meta[i * NG / (D / 32)]);
                    uint32_t high[16], low[16];
                    const uint32_t words[4] = {c[i].x, c[i].y, c[i].z, c[i].w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        float x[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) {      // 2^23 + code, minus 2^23
                            const int nibble = (e >> 1) + 4 * (e & 1);
                            x[e] = fmaf(hz.x, __uint_as_float(0x4B000000u | (words[k] >> (4 * nibble) & 15u)) - 8388608.f, hz.y);
                        }
                        if (window) {
                            const uint4 v = ring_row[i * 4 + k];
                            const uint32_t pairs[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                const int ch = (e >> 1) + 4 * (e & 1);
                                const float2 f = floats<T>(pairs[ch / 2]);
                                x[e] = ch & 1 ? f.y : f.x;
                            }
                        }
#pragma unroll
                        for (int e = 0; e < 8; e += 2) {
                            const uint32_t hi = packed<__half>(x[e], x[e + 1]);
                            const float2 f = floats<__half>(hi);
                            high[k * 4 + e / 2] = hi;
                            low[k * 4 + e / 2] = packed<__half>(x[e] - f.x, x[e + 1] - f.y);
                        }
                    }
                    tmem_st16(dst + i * 16, high);
                    tmem_st16(dst + D / 2 + i * 16, low);
                }
            }
            tmem_wait_st();
            tc_fence_before();
            mbar_arrive(a_full + 8 * buf);
            ++n;
        }
    } else if (warp == 12) {
        // ================================================================ products
        constexpr uint32_t kWhole = idesc_f16_f32(kBlock, kTileRows), kHalf = idesc_f16_f32(kBlock, kTileRows / 2);
        const uint32_t smem_base = smem_u32(smem);
        uint32_t n = 0, nq = 0;      // segments, query tiles
        while (next()) {
            if (*fail) alive = false;
            const uint32_t buf = n % Geo::A_BUFFERS;
            wait(a_full + 8 * buf, (n / Geo::A_BUFFERS) & 1);
            for (int step = s.s0; step < s.s1; ++step, ++nq) {
                const uint32_t stage = nq % Geo::STAGES, idesc = halves(step) == 2 ? kWhole : kHalf;
                wait(q_full + 8 * stage, (nq / Geo::STAGES) & 1);
                const uint64_t dq = desc_k_major(smem_base + stage * Geo::TILE);
#pragma unroll 1
                for (int blk = 0; blk < 2; ++blk) {
                    if (nq) wait(s_empty + 8 * blk, (nq - 1) & 1);
                    tc_fence_after();
                    if (elect_one()) {
                        const uint32_t d = tmem + Geo::TMEM_S + blk * kTileRows, ka = tmem + Geo::TMEM_A + (buf * 2 + blk) * Geo::A_COLUMNS;
#pragma unroll
                        for (int part = 1; part >= 0; --part)      // the low parts first: the accumulator's truncations are of small sums then
#pragma unroll
                            for (int ks = 0; ks < D / 16; ++ks)
                                umma_f16_ts(d, ka + part * (D / 2) + ks * 8, dq + (ks >> 2) * (Geo::HALF_BYTES >> 4) + (ks & 3) * 2, idesc, part == 0 || ks > 0);
                        umma_commit(s_full + 8 * blk);
                    }
                    __syncwarp();
                }
                if (elect_one()) umma_commit(q_empty + 8 * stage);
                __syncwarp();
            }
            if (elect_one()) umma_commit(a_empty + 8 * buf);
            __syncwarp();
            ++n;
        }
        // the last products must not outlive the CTA, whoever waited for them
        if (n) {
            if (elect_one()) umma_commit(drained);
            __syncwarp();
            mbar_wait_cycles(drained, 0);
        }
    } else if (warp == 13) {
        // ================================================================ query tiles
        const uint32_t smem_base = smem_u32(smem);
        uint32_t nq = 0;
        while (next()) {
            if (*fail) alive = false;
            for (int step = s.s0; step < s.s1; ++step, ++nq) {
                const uint32_t stage = nq % Geo::STAGES, use = nq / Geo::STAGES;
                if (use) wait(q_empty + 8 * stage, (use - 1) & 1);
                alive = __all_sync(0xffffffffu, alive && !*fail);
                if (lane == 0 && alive) {      // once a wait has run out nothing is copied any more
                    mbar_expect_tx(q_full + 8 * stage, Geo::TILE);
                    bulk_g2s(smem_base + stage * Geo::TILE, query_tile(args.plan, s.w, s.b, s.h, step), Geo::TILE, q_full + 8 * stage);
                }
                __syncwarp();
            }
        }
        // copies in flight end before the CTA does
        for (uint32_t i = nq > Geo::STAGES ? nq - Geo::STAGES : 0; i < nq; ++i) mbar_wait_cycles(q_full + 8 * (i % Geo::STAGES), (i / Geo::STAGES) & 1);
    } else {
        // ================================================================ exponentials
        const int blk = warp >> 2, row = tid & (kBlock - 1);
        const uint32_t s_addr = tmem + Geo::TMEM_S + blk * kTileRows + ((uint32_t)((warp & 3) * 32) << 16);
        uint32_t nq = 0;      // query tiles
        while (next()) {
            if (*fail) alive = false;
            const int t = s.tile * kItemTokens + blk * kBlock + row;
            const int hidden_rows = t < s.w.s.len ? s.it.first_row(t) : 0;      // rows below it do not see the token
            float sum = 0.f;
            for (int step = s.s0; step < s.s1; ++step, ++nq) {
                const uint32_t stage = nq % Geo::STAGES;
                wait(q_full + 8 * stage, (nq / Geo::STAGES) & 1);
                const float4 *constants = reinterpret_cast<const float4 *>(smem + stage * Geo::TILE + kTileRows * D * 2);
                const int parts = halves(step);
                wait(s_full + 8 * blk, nq & 1);
                tc_fence_after();
#pragma unroll 1
                for (int hf = 0; hf < parts; ++hf) {
                    float x[32], y[32];
                    tmem_ld32(s_addr + hf * 64, x);
                    tmem_ld32(s_addr + hf * 64 + 32, y);
                    tmem_wait_ld32(x);
                    tmem_wait_ld32(y);
                    if (hf == parts - 1) {      // the scores are in registers: the next product may overwrite them
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(s_empty + 8 * blk);
                    }
                    const int hidden = hidden_rows - step * kTileRows - hf * 64;      // columns below it
                    if (__any_sync(0xffffffffu, hidden > 0)) {
                        sum += sum_probabilities<true>(x, constants + hf * 32, hidden);
                        sum += sum_probabilities<true>(y, constants + hf * 32 + 16, hidden - 32);
                    } else {
                        sum += sum_probabilities<false>(x, constants + hf * 32, 0);
                        sum += sum_probabilities<false>(y, constants + hf * 32 + 16, 0);
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(q_empty + 8 * stage);
            }
            if (t < s.w.s.len) {      // a token without a page gains nothing
                const int page = p.batch.page_table[(int64_t)s.b * p.batch.max_pages + t / cfg.page_tokens];
                if (page < 0 || page >= cfg.n_pages) sum = 0.f;
            }
            alive = __all_sync(0xffffffffu, alive && !*fail);
            if (!alive) sum = CUDART_NAN_F;
            if (s.whole) {
                if (t < s.w.s.len) write_weight(a, s.w, s.h, t, sum);
            } else {
                float *shares = reinterpret_cast<float *>(args.shares + (size_t)args.n_slots * kManyDesc * 4);
                shares[((size_t)blockIdx.x * 2 + (s.begins ? 1 : 0)) * kItemTokens + blk * kBlock + row] = sum;
                if (s.begins && tid == 0) {
                    desc[1] = s.b; desc[2] = s.h; desc[3] = s.tile; desc[4] = s.parts;
                    desc[0] = 1;
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 0) tmem_dealloc(tmem, 512);
}

// Adds up the shares of an item that several runs have: blockIdx.x is the run that begins it.
__global__ void __launch_bounds__(kItemTokens) weight_join_kernel(const __grid_constant__ ManyArgs args)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const int *desc = reinterpret_cast<const int *>(args.shares) + (size_t)blockIdx.x * kManyDesc;
    if (desc[0] == 0) return;
    const PagedWeightArgs &a = args.plan.a;
    const int b = desc[1], h = desc[2], n = desc[4], t = desc[3] * kItemTokens + threadIdx.x;
    WeightSeq w;
    weight_sequence(a, b, w);
    if (t >= w.s.len) return;
    const float *shares = reinterpret_cast<const float *>(args.shares + (size_t)args.n_slots * kManyDesc * 4) + threadIdx.x;
    float sum = 0.f;
    for (int k = 0; k < n; ++k) sum += shares[((size_t)(blockIdx.x + k) * 2 + (k == 0 ? 1 : 0)) * kItemTokens];
    write_weight(a, w, h, t, sum);
}

// The most counted rows that a KV head of a sequence can have.
int64_t most_rows(const skvq_paged_config &cfg, const skvq_paged_batch &batch, int last)
{
    return (int64_t)(last && last < batch.max_new ? last : batch.max_new) * (cfg.n_q_heads / cfg.n_kv_heads);
}
// The layout of the query tiles: the smaller of a fixed number per sequence and one after the other (by all new tokens: those that `last` leaves out
// leave their tiles unused).
int64_t query_tiles(const skvq_paged_config &cfg, const skvq_paged_batch &batch, int last, int &seq_tiles)
{
    const int64_t rows = most_rows(cfg, batch, last), uniform = (rows + kTileRows - 1) / kTileRows * batch.n_seqs;
    const int64_t together = (int64_t)batch.n_tokens * (cfg.n_q_heads / cfg.n_kv_heads) / kTileRows + batch.n_seqs;
    seq_tiles = 0;
    if (rows <= kFewRows) return 0;
    if (uniform <= together) seq_tiles = (int)(uniform / batch.n_seqs);
    return seq_tiles ? uniform : together;
}

// Runs that the work is cut into: a CTA per SM, a query tile each at least.
int many_slots(const skvq_paged_config &cfg, const skvq_paged_batch &batch, int64_t rows)
{
    // one factor at a time: their product may have more than 64 bits
    const int64_t factors[] = {cfg.n_kv_heads, (batch.max_len + kItemTokens - 1) / kItemTokens, (rows + kTileRows - 1) / kTileRows};
    int64_t units = batch.n_seqs;
    for (const int64_t f : factors) units = f && units > sm_count() / f ? sm_count() : units * f;
    return (int)(units < 1 ? 1 : units);
}

template <typename T, int D, int NG, int NT, int E> cudaError_t launch_few(const WeightPlan &p, cudaStream_t stream)
{
    using Geo = FewGeo<D, NG, NT, E>;
    const skvq_paged_config &cfg = p.a.p.cfg;
    const skvq_paged_batch &batch = p.a.p.batch;
    static unsigned long long done = 0;
    const cudaError_t e = configure_smem_once(weight_few_kernel<T, D, NG, NT, E>, Geo::SMEM + (int)sizeof(long long) * (kMaxPagedSeqs + 1), done);
    if (e != cudaSuccess) return e;
    // one wave of resident CTAs, no more warps than tiles; one at least: it reports the sequences that are skipped
    const long long lq = batch.max_len > cfg.window ? batch.max_len - cfg.window : 0;
    const long long tiles = (lq + kTile - 1) / kTile + kRingCost * ((batch.max_len - lq + kRingTile - 1) / kRingTile);
    const long long wave = (long long)kFewCtas * sm_count(), useful = std::max(((long long)batch.n_seqs * cfg.n_kv_heads * tiles + kFewWarps - 1) / kFewWarps, 1LL);
    return launch_chained(weight_few_kernel<T, D, NG, NT, E>, dim3((unsigned)(useful < wave ? useful : wave)), kFewThreads,
                          Geo::SMEM + sizeof(long long) * (batch.n_seqs + 1), stream, p);
}

template <typename T, int D, int NG> cudaError_t launch_weights(const PagedWeightArgs &a, cudaStream_t stream)
{
    const skvq_paged_config &cfg = a.p.cfg;
    const skvq_paged_batch &batch = a.p.batch;
    WeightPlan p{};
    p.a = a;
    p.many_scale = std::fma(a.sm_scale, ManyGeo<D>::CUT, a.sm_scale);
    query_tiles(cfg, batch, a.last, p.seq_tiles);
    const int64_t rows = batch.n_tokens > 0 ? most_rows(cfg, batch, a.last) : 0, rep = cfg.n_q_heads / cfg.n_kv_heads;
    // The variant for few rows goes by the host's bound, the most rows that a sequence may have.  Measured with a row per sequence (64 sequences of 1024
    // to 16384 tokens, 32 heads, group 64): 294 us as at most 4 rows, 315 as 8, 419 as 16, 433 where the bound is above 16 and the kernels below follow with
    // nothing to do; with 4 rows (4 sequences of 131072 tokens, 32 heads over 8, group 32) 87, 90, 141, 147.
    cudaError_t e = rows <= kFewRowTile / 2 ? launch_few<T, D, NG, 1, 1>(p, stream) : rows <= kFewRowTile ? launch_few<T, D, NG, 1, 2>(p, stream) : launch_few<T, D, NG, 2, 2>(p, stream);
    if (e != cudaSuccess || rows <= kFewRows) return e;
    const int64_t padded = (rows + kTileRows - 1) / kTileRows * kTileRows, per = kQueryThreads / (D / 8), chunks = ((padded + rep - 1) / rep + per - 1) / per;
    p.heads = cfg.n_q_heads;
    while (p.heads > 4 && chunks * batch.n_seqs * ((cfg.n_q_heads + p.heads - 1) / p.heads) < 32LL * sm_count()) p.heads = (p.heads + 1) / 2;
    e = launch_chained(weight_queries_kernel<T, D>, dim3((unsigned)chunks, (cfg.n_q_heads + p.heads - 1) / p.heads, batch.n_seqs), kQueryThreads, 0, stream, p);
    if (e != cudaSuccess) return e;
    int seq_tiles;
    const ManyArgs m{p, many_slots(cfg, batch, rows), a.ws + query_tiles(cfg, batch, a.last, seq_tiles) * cfg.n_kv_heads * tile_bytes(D)};
    static unsigned long long done = 0;
    e = configure_smem_once(weight_many_kernel<T, D, NG>, ManyGeo<D>::SMEM + (int)sizeof(long long) * (kMaxPagedSeqs + 1), done);
    if (e != cudaSuccess) return e;
    e = launch_chained(weight_many_kernel<T, D, NG>, dim3(m.n_slots), kManyThreads, ManyGeo<D>::SMEM + sizeof(long long) * (batch.n_seqs + 1), stream, m);
    if (e != cudaSuccess) return e;
    return launch_chained(weight_join_kernel, dim3(m.n_slots), kItemTokens, 0, stream, m);
}

template <typename T> cudaError_t launch_by_shape(const PagedWeightArgs &a, cudaStream_t stream)
{
    if (a.p.cfg.head_dim == 128)
        return a.p.ng == 1 ? launch_weights<T, 128, 1>(a, stream) : a.p.ng == 2 ? launch_weights<T, 128, 2>(a, stream) : launch_weights<T, 128, 4>(a, stream);
    return a.p.ng == 1 ? launch_weights<T, 64, 1>(a, stream) : launch_weights<T, 64, 2>(a, stream);
}

}  // namespace

size_t paged_weights_workspace_bytes(const skvq_paged_config &cfg, const skvq_paged_batch &batch, int last)
{
    int seq_tiles;
    const int64_t rows = most_rows(cfg, batch, last), tiles = query_tiles(cfg, batch, last, seq_tiles);
    if (tiles == 0) return 0;
    return (size_t)tiles * cfg.n_kv_heads * tile_bytes(cfg.head_dim) + many_slots(cfg, batch, rows) * (size_t)(kManyDesc * 4 + 2 * kItemTokens * 4);
}

cudaError_t launch_paged_weights(const PagedWeightArgs &a, cudaStream_t stream)
{
    return a.p.cfg.dtype == SKVQ_F16 ? launch_by_shape<__half>(a, stream) : launch_by_shape<__nv_bfloat16>(a, stream);
}

}  // namespace skvq
