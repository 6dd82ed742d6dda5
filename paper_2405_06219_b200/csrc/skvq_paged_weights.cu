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

#include "skvq_mma_common.cuh"
#include "skvq_paged.cuh"
#include "skvq_paged_split.cuh"

namespace skvq {
namespace {

using mmak::ex2_approx;
using mmak::mma16816;
using mmak::smem_u32;

constexpr float kSubnormal = 1.f / 16777216.f;      // 2^-24: the least fp16 subnormal, what a code's lowest bit stands for as an operand
constexpr float kZeroScale = 1.f / 1024.f;           // brings a sum of 128 operands below 2^14 into fp16's range
constexpr int kQueryThreads = 128;
constexpr int kQueryTokens = kQueryThreads / 16;
constexpr int kTileRows = 128;      // rows of a query tile

// A query tile: kTileRows rows of D fp16, 64-channel halves one after the other, a half's rows 128 bytes each with 16-byte piece c of row r
// at c ^ (r & 7) (the 128-byte swizzle of the tensor core's operands); then floats [kTileRows] factor of a score in units of log2,
// [kTileRows] minus the lse in units of log2 (minus infinity: the row adds nothing), [NG][kTileRows] sums of the row over a group's channels.
struct WeightPlan {
    PagedWeightArgs a;
    int seq_tiles;        // > 0: sequence b's tiles begin at b * seq_tiles; 0: at starts[b] * Hq/Hkv / kTileRows + b
    int heads;            // query heads that a CTA of the first kernel walks over
};
__host__ __device__ constexpr int tile_bytes(int D, int ng) { return kTileRows * (D * 2 + (2 + ng) * 4); }

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
    return p.a.ws + ((base + tile) * p.a.p.cfg.n_kv_heads + h) * tile_bytes(p.a.p.cfg.head_dim, p.a.p.ng);
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
// operand of mma.m16n8k16, 8 rows the B operand, one accumulator per group.  A nibble under zeros is an fp16 subnormal, c 2^-24 (or
// 16 c 2^-24, against q/16), so codes enter the product as they are, exactly.  The zero points' share, the sum over groups of z sum q',
// is one more product: the parameters' words {h, z} are its A operand as they lie in memory, {0, sum q'} in two fp16 parts (22 bits)
// the B operand.  With at most 4 rows they take every other column, and a lane has one row instead of two.
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

template <typename T, int D, int NG, int NT, int E>
__global__ void __launch_bounds__(kFewThreads, NT == 1 ? 5 : 4) weight_few_kernel(const __grid_constant__ WeightPlan plan)
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
                    constants[r * (2 + NG)] = counts ? a.sm_scale * 1.4426950408889634f / up : 0.f;
                    constants[r * (2 + NG) + 1] = counts ? lse * -1.4426950408889634f : -CUDART_INF_F;
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
                        const uint32_t x = c[2 * h2], y = c[2 * h2 + 1], xs = x >> 8, ys = y >> 8;
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            float (&d)[4] = acc[n][st / PER];
                            const uint32_t x0 = x & 0x000F000Fu, y0 = y & 0x000F000Fu, x1 = x & 0x00F000F0u, y1 = y & 0x00F000F0u;
                            if (st % PER == 0) mma16816_from(d, x0, y0, x1, y1, bq[n][2 * st][0], bq[n][2 * st][1], 0.f, 0.f, 0.f, 0.f);
                            else mma16816(d, x0, y0, x1, y1, bq[n][2 * st][0], bq[n][2 * st][1]);
                            mma16816(d, xs & 0x000F000Fu, ys & 0x000F000Fu, xs & 0x00F000F0u, ys & 0x00F000F0u, bq[n][2 * st + 1][0], bq[n][2 * st + 1][1]);
                        }
                    }
                }
                float s[2][NT][E];
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    float h[NG];
#pragma unroll
                    for (int k = 0; k < NG; ++k) h[k] = floats<__half>(km[(16 * u + 8 * half + g) * NG + k]).x;
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < E; ++e) {
                            float x = h[0] * acc[n][0][2 * half + e];
#pragma unroll
                            for (int k = 1; k < NG; ++k) x = fmaf(h[k], acc[n][k][2 * half + e], x);
                            s[half][n][e] = fmaf(fmaf(x, kZeroScale / kSubnormal, zero[n][2 * half + e]), rs[n][e], nl[n][e]);
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
                        sums[half] += hidden ? 0.f : ex2_approx(fmaf(s[n][2 * half + e], rs[n][e] * kZeroScale, nl[n][e]));
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
// Sixteen lanes own a row; a half-warp takes a token and walks over heads with the token's angles in registers.
template <typename T, int D, int NG>
__global__ void __launch_bounds__(kQueryThreads) weight_queries_kernel(const __grid_constant__ WeightPlan plan)
{
    using R = Row<T, D>;
    constexpr int C = R::C;
    __shared__ __align__(16) T rows[kQueryTokens][2][D + 8];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const PagedWeightArgs &a = plan.a;
    const PagedArgs &p = a.p;
    const int unit = threadIdx.x >> 4, sub = threadIdx.x & 15, c0 = sub * C, b = blockIdx.z;
    WeightSeq w;
    weight_sequence(a, b, w);
    if (!w.ok || w.rows <= kFewRows) return;
    const int filled = (w.rows + kTileRows - 1) / kTileRows * kTileRows;      // zeros behind the last row: tiles are read whole
    if ((int)blockIdx.x * kQueryTokens * w.rep >= filled) return;
    const int i = blockIdx.x * kQueryTokens + unit, pos = w.s.len - w.m + i;
    const int h0 = blockIdx.y * plan.heads, h1 = min(h0 + plan.heads, p.cfg.n_q_heads);
    const bool have = i < w.m, turn = p.rope.table && have && pos >= 0;
    const int64_t tok = w.s.row0 + w.s.n - w.m + i;
    float2 cs[C];
    if (turn) load_angles(cs, p.rope, pos, c0);
    const T *src = static_cast<const T *>(a.q) + tok * a.q_stride + c0;
    T *raw = rows[unit][0], *turned = rows[unit][1];
    int from[C], hk = -1;
    R next;
#pragma unroll
    for (int k = 0; k < R::WORDS; ++k) next.w[k] = 0u;
    if (have && h0 < h1) next.load(src + (int64_t)h0 * D);
    for (int h = h0; h < h1; ++h) {
        if (h / w.rep != hk) {
            hk = h / w.rep;
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
        bool finite = true;
#pragma unroll
        for (int j = 0; j < C; ++j) {
            x[j] = Elem<T>::to_float(turned[from[j]]);
            mx = fmaxf(mx, fabsf(x[j]));
            finite = finite && fabsf(x[j]) < CUDART_INF_F;
        }
        const float lse = have ? a.lse[tok * p.cfg.n_q_heads + h] : CUDART_INF_F;
        const uint32_t odd = __ballot_sync(0xffffffffu, !finite) & (0xFFFFu << (threadIdx.x & 16));
        const bool counts = odd == 0u && fabsf(lse) < CUDART_INF_F;
#pragma unroll
        for (int d = 1; d < 16; d <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
        const float up = counts ? row_factor(mx) : 1.f;
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < C; ++j) {
            x[j] = counts ? x[j] * up : 0.f;
            sum += __half2float(__float2half_rn(x[j]));
        }
        // sums of a group's channels: a group is the channels of 16 / NG lanes
#pragma unroll
        for (int d = 1; d < 16 / NG; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        const int r = i * w.rep + h - hk * w.rep;
        if (r >= filled) continue;
        uint8_t *tile = const_cast<uint8_t *>(query_tile(plan, w, b, hk, r / kTileRows));
        const int tr = r % kTileRows;
        uint8_t *dst = tile + (c0 >> 6) * kTileRows * 128 + tr * 128 + (((((c0 >> 3) & 7) ^ (tr & 7)) << 4)) + (c0 & 7) * 2;
        if constexpr (C == 8)
            *reinterpret_cast<uint4 *>(dst) = make_uint4(packed<__half>(x[0], x[1]), packed<__half>(x[2], x[3]), packed<__half>(x[4], x[5]), packed<__half>(x[6], x[7]));
        else *reinterpret_cast<uint2 *>(dst) = make_uint2(packed<__half>(x[0], x[1]), packed<__half>(x[2], x[3]));
        float *constants = reinterpret_cast<float *>(tile + kTileRows * D * 2) + tr;
        if (sub == 0) {
            constants[0] = a.sm_scale * 1.4426950408889634f / up;
            constants[kTileRows] = counts ? lse * -1.4426950408889634f : -CUDART_INF_F;
        }
        if (sub % (16 / NG) == 0) constants[(2 + sub / (16 / NG)) * kTileRows] = sum;
    }
}

// A CTA per 64 tokens of a KV head: its keys in shared memory as fp32, a token and a quarter of the rows per thread.
constexpr int kTokens = 64;
constexpr int kThreads = 256;
template <typename T, int D, int NG>
__global__ void __launch_bounds__(kThreads) weight_tokens_kernel(const __grid_constant__ WeightPlan plan)
{
    __shared__ float key[kTokens][D + 1];
    __shared__ float zero[kTokens][NG];
    __shared__ float query[8][D], constants[8][2 + NG], part[4][kTokens];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const PagedWeightArgs &a = plan.a;
    const skvq_paged_config &cfg = a.p.cfg;
    const int b = blockIdx.z, h = blockIdx.y, token = threadIdx.x % kTokens, quarter = threadIdx.x / kTokens, t = blockIdx.x * kTokens + token;
    WeightSeq w;
    weight_sequence(a, b, w);
    if (!w.ok || w.rows <= kFewRows || (int)blockIdx.x * kTokens >= w.s.len) return;
    const int P = cfg.page_tokens;
    bool have = t < w.s.len;
    if (have) {
        const int page = a.p.batch.page_table[(int64_t)b * a.p.batch.max_pages + t / P];
        if (page < 0 || page >= cfg.n_pages) {
            set_status(a.p.c.status, SKVQ_STATUS_BAD_PAGE);
            have = false;
        } else if (t < w.s.lq) {
            const int64_t at = ((int64_t)page * cfg.n_kv_heads + h) * P + t % P;
            for (int c = quarter * (D / 4); c < (quarter + 1) * (D / 4); ++c) {
                const int code = static_cast<const uint8_t *>(a.p.c.k_codes)[at * (D / 2) + c / 2] >> (c % 2 * 4) & 15;
                const __half2 m = static_cast<const __half2 *>(a.p.c.k_meta)[at * NG + c / (D / NG)];
                key[token][c] = __low2float(m) * code;
                zero[token][c / (D / NG)] = __high2float(m);
            }
        } else {
            const int64_t row = ((int64_t)w.s.slot * cfg.n_kv_heads + h) * cfg.ring_tokens + t % cfg.ring_tokens;
            for (int c = quarter * (D / 4); c < (quarter + 1) * (D / 4); ++c) {
                key[token][c] = Elem<T>::to_float(static_cast<const T *>(a.p.c.k_win)[row * D + c]);
                zero[token][c / (D / NG)] = 0.f;
            }
        }
    }
    // rows below it do not see the token
    const int64_t first_row = a.causal ? (int64_t)max(t - (w.s.len - w.m), 0) * w.rep : 0;
    float sum = 0.f;
    for (int r0 = 0; r0 < w.rows; r0 += 8) {
        __syncthreads();
        for (int e = threadIdx.x; e < 8 * D; e += kThreads) {
            const int r = r0 + e / D, c = e % D, tr = r % kTileRows;
            if (r >= w.rows) break;
            const uint8_t *tile = query_tile(plan, w, b, h, r / kTileRows);
            query[e / D][(c & ~7) + channel_at(c & 7)] = __half2float(*reinterpret_cast<const __half *>(
                tile + (c >> 6) * kTileRows * 128 + tr * 128 + ((((c >> 3) & 7) ^ (tr & 7)) << 4) + (c & 7) * 2));
            if (c < 2 + NG) constants[e / D][c] = reinterpret_cast<const float *>(tile + kTileRows * D * 2)[c * kTileRows + tr];
        }
        __syncthreads();
        for (int k = quarter; k < min(8, w.rows - r0); k += 4) {
            if (!have || r0 + k < first_row) continue;
            float s = 0.f;
            for (int c = 0; c < D; ++c) s = fmaf(query[k][c], key[token][c], s);
            for (int g = 0; g < NG; ++g) s = fmaf(constants[k][2 + g], zero[token][g], s);
            sum += exp2f(fmaf(s, constants[k][0], constants[k][1]));
        }
    }
    part[quarter][token] = sum;
    __syncthreads();
    if (quarter == 0 && t < w.s.len) {
        const int64_t at = ((int64_t)w.s.slot * cfg.n_kv_heads + h) * a.capacity + t;
        const float old = a.w_in && t < w.s.len - w.s.n ? a.w_in[at] : 0.f;
        a.w_out[at] = old + ((part[0][token] + part[1][token]) + (part[2][token] + part[3][token]));
    }
}

// The most counted rows that a KV head of a sequence can have.
int64_t most_rows(const skvq_paged_config &cfg, const skvq_paged_batch &batch, int last)
{
    return (int64_t)(last && last < batch.max_new ? last : batch.max_new) * (cfg.n_q_heads / cfg.n_kv_heads);
}
// The layout of the query tiles: the smaller of a fixed number per sequence and one after the other.
int64_t query_tiles(const skvq_paged_config &cfg, const skvq_paged_batch &batch, int last, int &seq_tiles)
{
    const int64_t rows = most_rows(cfg, batch, last), uniform = (rows + kTileRows - 1) / kTileRows * batch.n_seqs;
    const int64_t together = (int64_t)batch.n_tokens * (cfg.n_q_heads / cfg.n_kv_heads) / kTileRows + batch.n_seqs;
    seq_tiles = 0;
    if (rows <= kFewRows) return 0;
    if (uniform <= together || (last && last < batch.max_new)) seq_tiles = (int)(uniform / batch.n_seqs);
    return seq_tiles ? uniform : together;
}

template <typename T, int D, int NG, int NT, int E> cudaError_t launch_few(const WeightPlan &p, cudaStream_t stream)
{
    using Geo = FewGeo<D, NG, NT, E>;
    const skvq_paged_config &cfg = p.a.p.cfg;
    const skvq_paged_batch &batch = p.a.p.batch;
    static unsigned long long done = 0;
    const cudaError_t e = configure_smem_once(weight_few_kernel<T, D, NG, NT, E>, Geo::SMEM + (int)sizeof(long long) * (kMaxPagedSeqs + 1), done);
    if (e != cudaSuccess) return e;
    // one wave of resident CTAs, no more warps than tiles
    const long long lq = batch.max_len > cfg.window ? batch.max_len - cfg.window : 0;
    const long long tiles = (lq + kTile - 1) / kTile + kRingCost * ((batch.max_len - lq + kRingTile - 1) / kRingTile);
    const long long wave = (NT == 1 ? 5LL : 4LL) * sm_count(), useful = ((long long)batch.n_seqs * cfg.n_kv_heads * tiles + kFewWarps - 1) / kFewWarps;
    return launch_chained(weight_few_kernel<T, D, NG, NT, E>, dim3((unsigned)(useful < wave ? useful : wave)), kFewThreads,
                          Geo::SMEM + sizeof(long long) * (batch.n_seqs + 1), stream, p);
}

template <typename T, int D, int NG> cudaError_t launch_weights(const PagedWeightArgs &a, cudaStream_t stream)
{
    const skvq_paged_config &cfg = a.p.cfg;
    const skvq_paged_batch &batch = a.p.batch;
    WeightPlan p{};
    p.a = a;
    query_tiles(cfg, batch, a.last, p.seq_tiles);
    const int64_t rows = batch.n_tokens > 0 ? most_rows(cfg, batch, a.last) : 0, rep = cfg.n_q_heads / cfg.n_kv_heads;
    cudaError_t e = rows <= kFewRowTile / 2 ? launch_few<T, D, NG, 1, 1>(p, stream) : rows <= kFewRowTile ? launch_few<T, D, NG, 1, 2>(p, stream) : launch_few<T, D, NG, 2, 2>(p, stream);
    if (e != cudaSuccess || rows <= kFewRows) return e;
    const int64_t padded = (rows + kTileRows - 1) / kTileRows * kTileRows, chunks = ((padded + rep - 1) / rep + kQueryTokens - 1) / kQueryTokens;
    p.heads = cfg.n_q_heads;
    while (p.heads > 4 && chunks * batch.n_seqs * ((cfg.n_q_heads + p.heads - 1) / p.heads) < 32LL * sm_count()) p.heads = (p.heads + 1) / 2;
    e = launch_chained(weight_queries_kernel<T, D, NG>, dim3((unsigned)chunks, (cfg.n_q_heads + p.heads - 1) / p.heads, batch.n_seqs), kQueryThreads, 0, stream, p);
    if (e != cudaSuccess) return e;
    return launch_chained(weight_tokens_kernel<T, D, NG>, dim3((batch.max_len + kTokens - 1) / kTokens, cfg.n_kv_heads, batch.n_seqs), kThreads, 0, stream, p);
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
    return (size_t)query_tiles(cfg, batch, last, seq_tiles) * cfg.n_kv_heads * tile_bytes(cfg.head_dim, cfg.head_dim / cfg.group_size);
}

cudaError_t launch_paged_weights(const PagedWeightArgs &a, cudaStream_t stream)
{
    if (a.p.batch.max_len == 0) return cudaSuccess;
    return a.p.cfg.dtype == SKVQ_F16 ? launch_by_shape<__half>(a, stream) : launch_by_shape<__nv_bfloat16>(a, stream);
}

}  // namespace skvq
