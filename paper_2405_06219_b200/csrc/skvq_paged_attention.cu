// skvq_paged_attention for few query rows per (sequence, KV head): single-token decode, drafted tokens.
//
// The rows of a KV head are packed: row = new token * (Hq/Hkv) + query head, 16 rows per item.  Items of the whole batch are
// laid end to end, priced in 32-token tiles (a tile of the unquantized window costs kRingCost), and cut into equal
// runs, one per CTA: ragged batches and long single sequences load the GPU alike.  The four warps of a CTA take quarters of
// a run, stream their tiles through private shared-memory rings, and join their softmax states at the end; an item that
// several CTAs share is joined by the merge kernel.
//
// With q' the rotated, reordered query, the scores of a quantized token are formed without dequantizing the key:
//   q'.K~_t = sum_g h_{t,g} (sum_{j in g} q'_j c_{t,j}) + sum_g z_{t,g} (sum_{j in g} q'_j)
// the inner sums on mma.m16n8k16 with the codes (exact in fp16) as B operand, fp32 accumulators, one per group.  Values are
// formed as fp16(h c + z) in registers (one rounding, 2^-11 relative at most, against 2^-9 for bf16 outputs and 2^-12 for fp16) and
// multiplied by the probabilities in fp16.  A probability is held times 2^14 relative to the running maximum: fp16 then
// resolves 2^-38 of the largest, so a million small ones still add up; their sum is kept in fp32.
// Fragments: the channels of a k-step and the tokens of a column are free to choose as long as both operands agree.  A lane's
// B registers of the score product are the nibble pairs (i, i+4) of one 32-bit word, a word of every lane inside one
// 32-channel granule; of the value product they pair one channel of tokens j and j+4, so neither operand is ever transposed
// through shared memory.
#include <math_constants.h>

#include "skvq_mma_common.cuh"
#include "skvq_paged.cuh"

namespace skvq {
namespace {

using mmak::and_or;
using mmak::ex2_approx;
using mmak::mma16816;
using mmak::smem_u32;

constexpr int kSplitWarps = 4;
constexpr int kSplitThreads = kSplitWarps * 32;
constexpr int kRowsPerItem = 16;
constexpr int kTile = 32;             // tokens per warp tile
constexpr int kRingCost = 4;          // a window tile moves 16-bit rows: about four times the bytes
constexpr int kStages = 3;
constexpr float kPScaleLog2 = 14.0f;

struct SplitArgs {
    PagedAttnArgs a;
    int n_slots;
};

// Workspace: descriptor [n_slots][8] ints, then partials [n_slots][2][16 rows][D + 4] floats {o[D], m, l, pad}.  A run holds at
// most one item that it continues (partial 0) and one that it begins and does not finish (partial 1).
constexpr int kDescInts = 8;
__host__ __device__ constexpr int partial_stride(int D) { return D + 4; }

template <int D, int NG>
struct Geometry {
    static constexpr int ROW = D / 2;                  // bytes of a code row
    static constexpr int CHUNKS = ROW / 16;
    static constexpr int CODES = kTile * ROW;
    static constexpr int META = kTile * NG * 4;
    static constexpr int STAGE = 2 * CODES + 2 * META;
    static constexpr int SETS = D / 32;                // 32-channel granules
    static constexpr int CPT = D / 8;                  // value channels per lane
    static constexpr int QROW = D + 8;                 // halves per query row in shared memory
    static constexpr int RINGS = kSplitWarps * kStages * STAGE;
    static constexpr int JOIN = 2 * kRowsPerItem * D * 4;      // two warps' accumulators
    static constexpr int POOL = RINGS > JOIN ? RINGS : JOIN;
    static constexpr int SMEM = POOL + kRowsPerItem * QROW * 2;
};

// Position of 16-byte piece c of row t inside the tile: rows that one load instruction touches fall into different banks.
template <int D> __device__ __forceinline__ int piece_at(int t, int c)
{
    if (D == 128) return c ^ ((t & 2) | ((t >> 2) & 1));
    return c ^ ((t >> 2) & 1);
}

__device__ __forceinline__ void cp16(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

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
// Four nibble pairs (i, i + 4) of a word as exact fp16 pairs.  1024 + c is fp16 0x6400 | c, 1024 + 16 c is 0x6400 | c << 4.
__device__ __forceinline__ void nibble_pairs(uint32_t w, uint32_t (&r)[4])
{
    constexpr uint32_t M = 0x64006400u, SIXTEENTH = 0x2C002C00u, MINUS64 = 0xD400D400u;
    const uint32_t u = w >> 8;
    r[0] = h2_sub(and_or(w, 0x000F000Fu, M), M);
    r[1] = h2_fma(and_or(w, 0x00F000F0u, M), SIXTEENTH, MINUS64);
    r[2] = h2_sub(and_or(u, 0x000F000Fu, M), M);
    r[3] = h2_fma(and_or(u, 0x00F000F0u, M), SIXTEENTH, MINUS64);
}
__device__ __forceinline__ uint32_t pack_h2(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// A pair of elements of the cache's type as fp16 (bf16: exact between 2^-14 and 65504, off by 2^-25 at most below).
template <typename T> __device__ __forceinline__ uint32_t as_h2(uint32_t v);
template <> __device__ __forceinline__ uint32_t as_h2<__half>(uint32_t v) { return v; }
template <> __device__ __forceinline__ uint32_t as_h2<__nv_bfloat16>(uint32_t v)
{
    return pack_h2(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u));
}

// What a sequence contributes to the flat partition.
struct SeqCost {
    int tiles_c, tiles_r;      // 32-token tiles of quantized tokens, of the window
    int cost;                  // of one item, at least 1
    int m_tiles;               // 16-row items per KV head
};
__device__ __forceinline__ SeqCost seq_cost(const PagedArgs &p, const PagedSeq &s)
{
    SeqCost c;
    const int rep = p.cfg.n_q_heads / p.cfg.n_kv_heads;
    const int lq = max(s.len - p.cfg.window, 0);
    c.tiles_c = (lq + kTile - 1) / kTile;
    c.tiles_r = (s.len - lq + kTile - 1) / kTile;
    c.cost = max(c.tiles_c + kRingCost * c.tiles_r, 1);
    c.m_tiles = (s.n * rep + kRowsPerItem - 1) / kRowsPerItem;
    return c;
}

template <typename T, int D, int NG>
__global__ void __launch_bounds__(kSplitThreads) paged_split_kernel(const __grid_constant__ SplitArgs args)
{
    using Geo = Geometry<D, NG>;
    const PagedAttnArgs &a = args.a;
    const PagedArgs &p = a.p;
    const skvq_paged_config &cfg = p.cfg;
    extern __shared__ __align__(128) uint8_t smem[];
    long long *pre = reinterpret_cast<long long *>(smem + Geo::SMEM);      // [n_seqs + 1] cost of the sequences before b
    __half *qs = reinterpret_cast<__half *>(smem + Geo::POOL);
    __shared__ long long scan_sh[kSplitWarps];
    __shared__ float row_scale[kRowsPerItem], q_sum[kRowsPerItem][4];
    __shared__ float ml_sh[kSplitWarps][kRowsPerItem][2];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, j = lane & 3;
    const int rep = cfg.n_q_heads / cfg.n_kv_heads, B = p.batch.n_seqs;

    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");

    // ---- the flat partition: exclusive prefix of the sequences' costs
    {
        long long carry = 0;
        for (int base = 0; base < B; base += kSplitThreads) {
            const int b = base + tid;
            long long c = 0;
            if (b < B) {
                PagedSeq s;
                if (paged_sequence(p, b, false, s)) {
                    const SeqCost sc = seq_cost(p, s);
                    c = (long long)sc.cost * sc.m_tiles * cfg.n_kv_heads;
                } else if (blockIdx.x == 0) {
                    set_status(p.c.status, SKVQ_STATUS_BAD_BATCH);
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
            for (int w = 0; w < kSplitWarps; ++w) {
                if (w < warp) before += scan_sh[w];
                carry += scan_sh[w];
            }
            if (b < B) pre[b] = before + incl - c;
            __syncthreads();
        }
        if (tid == 0) pre[B] = carry;
        __syncthreads();
    }
    const long long total = pre[B], ups = max((total + args.n_slots - 1) / args.n_slots, 1LL);
    long long f = blockIdx.x * ups;
    const long long f1 = min(f + ups, total);
    int *desc = reinterpret_cast<int *>(a.ws) + (size_t)blockIdx.x * kDescInts;
    if (tid == 0) desc[0] = 0;
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
    float *partials = a.ws + (size_t)args.n_slots * kDescInts;

    while (f < f1) {
        while (pre[b + 1] <= f) ++b;
        PagedSeq seq;
        paged_sequence(p, b, false, seq);
        const SeqCost sc = seq_cost(p, seq);
        const long long item = (f - pre[b]) / sc.cost;
        const int off = (int)((f - pre[b]) - item * sc.cost);
        const int take = (int)min((long long)(sc.cost - off), f1 - f);
        const int hk = (int)(item / sc.m_tiles), mt = (int)(item - (long long)hk * sc.m_tiles);
        const int row_base = mt * kRowsPerItem, R = min(kRowsPerItem, seq.n * rep - row_base);
        const int L = seq.len, lq = max(L - cfg.window, 0);
        // rows see tokens below their limit
        auto row_limit = [&](int r) { return a.causal ? min(L, L - seq.n + (row_base + min(r, R - 1)) / rep + 1) : L; };
        const int limit_lo = row_limit(0), limit_hi = row_limit(R - 1);
        const int lim0 = row_limit(g), lim1 = row_limit(g + 8);

        // ---- queries: rotate, round to T, reorder; fp16 rows (bf16 rows times a power of two), group sums
        {
            const int r = tid >> 3, part = tid & 7;      // 8 threads per row, CPT channels each
            T *raw = reinterpret_cast<T *>(smem);        // [16][D], before the rings are in use
            const int i = (row_base + r) / rep, head = hk * rep + (row_base + r) % rep;
            const int pos = L - seq.n + i;
            const T *src = static_cast<const T *>(a.q) + (int64_t)(seq.row0 + i) * a.q_stride + (int64_t)head * D;
            if (r < R) {
                const float2 *table = static_cast<const float2 *>(p.rope.table);
                const int half = p.rope.rot_dim / 2;
                for (int k = 0; k < Geo::CPT; ++k) {
                    const int c = part * Geo::CPT + k;
                    T x = src[c];
                    if (table && pos >= 0 && c < p.rope.rot_dim) {
                        const bool second = p.rope.interleaved ? c & 1 : c >= half;
                        const int pair = p.rope.interleaved ? c >> 1 : (second ? c - half : c);
                        const int partner = p.rope.interleaved ? c ^ 1 : (second ? c - half : c + half);
                        const float2 cs = table[(int64_t)pos * half + pair];
                        const float own = Elem<T>::to_float(x), other = Elem<T>::to_float(src[partner]);
                        x = Elem<T>::from_float(second ? rotate_second(other, own, cs.x, cs.y) : rotate_first(own, other, cs.x, cs.y));
                    }
                    raw[r * D + c] = x;
                }
            }
            __syncwarp();
            float x[Geo::CPT], mx = 0.f, sum = 0.f;
            for (int k = 0; k < Geo::CPT; ++k) {
                const int c = part * Geo::CPT + k;
                const int s = p.c.reorder_k ? p.c.reorder_k[hk * D + c] & (D - 1) : c;
                x[k] = r < R ? Elem<T>::to_float(raw[r * D + s]) : 0.f;
                mx = fmaxf(mx, fabsf(x[k]));
            }
            float up = 1.f;
            if (sizeof(T) == 2 && !__is_same(T, __half)) {
                // bf16 has more range than fp16: bring the row's largest to [2^13, 2^14), exactly
#pragma unroll
                for (int m = 1; m < 8; m <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, m));
                if (mx > 0.f && mx < CUDART_INF_F) {
                    int e;
                    frexpf(mx, &e);
                    up = ldexpf(1.f, min(14 - e, 126));
                }
            }
            __syncwarp();
            for (int k = 0; k < Geo::CPT; ++k) {
                const __half v = __float2half_rn(x[k] * up);
                sum += __half2float(v);
                qs[r * Geo::QROW + part * Geo::CPT + k] = v;
            }
            const int per_group = 8 / NG;
            for (int m = 1; m < per_group; m <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, m);
            if (part % per_group == 0) q_sum[r][part / per_group] = sum;
            if (part == 0) row_scale[r] = a.sm_scale * 1.4426950408889634f / up;
        }
        __syncthreads();
        uint32_t aq[Geo::SETS * 2][4];
#pragma unroll
        for (int s = 0; s < Geo::SETS; ++s) {
            const uint4 x = *reinterpret_cast<const uint4 *>(qs + g * Geo::QROW + 32 * s + 8 * j);
            const uint4 y = *reinterpret_cast<const uint4 *>(qs + (g + 8) * Geo::QROW + 32 * s + 8 * j);
            aq[2 * s][0] = __byte_perm(x.x, x.z, 0x5410); aq[2 * s][1] = __byte_perm(y.x, y.z, 0x5410);
            aq[2 * s][2] = __byte_perm(x.x, x.z, 0x7632); aq[2 * s][3] = __byte_perm(y.x, y.z, 0x7632);
            aq[2 * s + 1][0] = __byte_perm(x.y, x.w, 0x5410); aq[2 * s + 1][1] = __byte_perm(y.y, y.w, 0x5410);
            aq[2 * s + 1][2] = __byte_perm(x.y, x.w, 0x7632); aq[2 * s + 1][3] = __byte_perm(y.y, y.w, 0x7632);
        }
        const float rs0 = row_scale[g], rs1 = row_scale[g + 8];
        float qsum0[NG], qsum1[NG];
#pragma unroll
        for (int n = 0; n < NG; ++n) { qsum0[n] = q_sum[g][n]; qsum1[n] = q_sum[g + 8][n]; }

        // ---- this warp's quarter of the run
        auto tile_of = [&](int x) { return x <= sc.tiles_c ? x : sc.tiles_c + (x - sc.tiles_c + kRingCost - 1) / kRingCost; };
        const int seg0 = tile_of(off), seg1 = tile_of(off + take);
        const int c0 = min(seg0, sc.tiles_c), c1 = max(min(min(seg1, sc.tiles_c), (limit_hi + kTile - 1) / kTile), c0);
        const int q0 = c0 + (int)((long long)(c1 - c0) * warp / kSplitWarps), q1 = c0 + (int)((long long)(c1 - c0) * (warp + 1) / kSplitWarps);

        float o[Geo::CPT][4];
#pragma unroll
        for (int n = 0; n < Geo::CPT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[n][e] = 0.f;
        float m0 = -CUDART_INF_F, m1 = -CUDART_INF_F, l0 = 0.f, l1 = 0.f;

        // Scores (log2 domain) of 32 tokens -> probabilities as A fragments; s[n] = columns of 8-token block n.
        auto softmax_tile = [&](float (&s)[4][4], uint32_t (&pa)[2][4]) {
            float x0 = fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[1][0], s[1][1])), x1 = fmaxf(fmaxf(s[0][2], s[0][3]), fmaxf(s[1][2], s[1][3]));
            x0 = fmaxf(x0, fmaxf(fmaxf(s[2][0], s[2][1]), fmaxf(s[3][0], s[3][1])));
            x1 = fmaxf(x1, fmaxf(fmaxf(s[2][2], s[2][3]), fmaxf(s[3][2], s[3][3])));
#pragma unroll
            for (int d = 1; d < 4; d <<= 1) {
                x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, d));
                x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, d));
            }
            const float n0 = fmaxf(m0, x0), n1 = fmaxf(m1, x1);
            if (__any_sync(0xffffffffu, n0 > m0 || n1 > m1)) {
                const float f0 = n0 > m0 ? ex2_approx(m0 - n0) : 1.f, f1 = n1 > m1 ? ex2_approx(m1 - n1) : 1.f;
                l0 *= f0;
                l1 *= f1;
#pragma unroll
                for (int n = 0; n < Geo::CPT; ++n) { o[n][0] *= f0; o[n][1] *= f0; o[n][2] *= f1; o[n][3] *= f1; }
                m0 = n0;
                m1 = n1;
            }
            const float b0 = (m0 == -CUDART_INF_F ? 0.f : m0) - kPScaleLog2, b1 = (m1 == -CUDART_INF_F ? 0.f : m1) - kPScaleLog2;
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const float e0 = ex2_approx(s[n][0] - b0), e1 = ex2_approx(s[n][1] - b0), e2 = ex2_approx(s[n][2] - b1), e3 = ex2_approx(s[n][3] - b1);
                l0 += e0 + e1;
                l1 += e2 + e3;
                pa[n >> 1][2 * (n & 1)] = pack_h2(e0, e1);
                pa[n >> 1][2 * (n & 1) + 1] = pack_h2(e2, e3);
            }
        };

        // ---- quantized tokens
        const uint32_t ring = smem_u32(smem) + warp * kStages * Geo::STAGE;
        const uint8_t *ring_ptr = smem + warp * kStages * Geo::STAGE;
        const int P = cfg.page_tokens;
        const int32_t *table = p.batch.page_table + (int64_t)b * p.batch.max_pages;
        // Page ids of 32 consecutive 16-token blocks, one per lane; -1 past the quantized tokens, -2 for an id outside the pool.
        auto load_pages = [&](int block) {
            const int t = (block + lane) * 16;
            int id = -1;
            if (t < lq) {
                id = table[t / P];
                if (id < 0 || id >= cfg.n_pages) { id = -2; set_status(p.c.status, SKVQ_STATUS_BAD_PAGE); }
            }
            return id;
        };
        int pages_base = q0 * 2, pages = q0 < q1 ? load_pages(pages_base) : -1, pages_next = q0 < q1 ? load_pages(pages_base + 32) : -1;
        uint32_t bad = 0;      // bit 2 * stage + block: the block has no page
        auto fetch = [&](int tile, int stage) {
            if (tile < q1) {
                if (tile * 2 >= pages_base + 32) {
                    pages_base += 32;
                    pages = pages_next;
                    pages_next = load_pages(pages_base + 32);
                }
                const int ida = __shfl_sync(0xffffffffu, pages, tile * 2 - pages_base), idb = __shfl_sync(0xffffffffu, pages, tile * 2 + 1 - pages_base);
                bad = (bad & ~(3u << (2 * stage))) | ((ida < 0 ? 1u : 0u) | (idb < 0 ? 2u : 0u)) << (2 * stage);
                const uint32_t base = ring + stage * Geo::STAGE;
                // first row of the two 16-token blocks in the pool
                const int64_t ra = ((int64_t)ida * cfg.n_kv_heads + hk) * P + (tile * kTile) % P;
                const int64_t rb = ((int64_t)idb * cfg.n_kv_heads + hk) * P + (tile * kTile + 16) % P;
#pragma unroll
                for (int k = 0; k < Geo::CHUNKS; ++k) {
                    const int q = k * 32 + lane, t = q / Geo::CHUNKS, c = q % Geo::CHUNKS;
                    if ((t < 16 ? ida : idb) >= 0) {
                        const int64_t row = (t < 16 ? ra : rb) + (t & 15);
                        const uint32_t dst = base + t * Geo::ROW + piece_at<D>(t, c) * 16;
                        cp16(dst, static_cast<const uint8_t *>(p.c.k_codes) + row * Geo::ROW + c * 16);
                        cp16(dst + Geo::CODES, static_cast<const uint8_t *>(p.c.v_codes) + row * Geo::ROW + c * 16);
                    }
                }
                constexpr int PIECES = kTile * NG / 4;      // 16-byte pieces of one tensor's parameters
#pragma unroll
                for (int k = 0; k < (2 * PIECES + 31) / 32; ++k) {
                    const int q = k * 32 + lane, side = q >= PIECES, piece = q - side * PIECES;
                    const int t = piece * 4 / NG;
                    if (q < 2 * PIECES && (t < 16 ? ida : idb) >= 0) {
                        const int64_t row = t < 16 ? ra : rb;
                        const uint8_t *src = static_cast<const uint8_t *>(side ? p.c.v_meta : p.c.k_meta) + row * (NG * 4) + (piece - (t < 16 ? 0 : PIECES / 2)) * 16;
                        cp16(base + 2 * Geo::CODES + side * Geo::META + piece * 16, src);
                    }
                }
            }
            cp_commit();
        };
#pragma unroll
        for (int k = 0; k < kStages - 1; ++k) fetch(q0 + k, k);
        int stage = 0;
        for (int tile = q0; tile < q1; ++tile) {
            cp_wait<kStages - 2>();
            __syncwarp();
            const uint8_t *buf = ring_ptr + stage * Geo::STAGE;
            const uint32_t bad_here = (bad >> (2 * stage)) & 3u;
            const int t0 = tile * kTile;
            const __half2 *km = reinterpret_cast<const __half2 *>(buf + 2 * Geo::CODES), *vm = reinterpret_cast<const __half2 *>(buf + 2 * Geo::CODES + Geo::META);
            float s[4][4];
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const int t = 8 * n + (g >> 1) + 4 * (g & 1);      // the token of column g
                float acc[NG][4];
#pragma unroll
                for (int k = 0; k < NG; ++k)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[k][e] = 0.f;
#pragma unroll
                for (int st = 0; st < Geo::SETS; ++st) {
                    const uint32_t w = *reinterpret_cast<const uint32_t *>(buf + t * Geo::ROW + piece_at<D>(t, st) * 16 + j * 4);
                    uint32_t c[4];
                    nibble_pairs(w, c);
                    float (&d)[4] = acc[st * NG / Geo::SETS];
                    mma16816(d, aq[2 * st][0], aq[2 * st][1], aq[2 * st][2], aq[2 * st][3], c[0], c[1]);
                    mma16816(d, aq[2 * st + 1][0], aq[2 * st + 1][1], aq[2 * st + 1][2], aq[2 * st + 1][3], c[2], c[3]);
                }
                float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < NG; ++k) {
                    const float2 ha = __half22float2(km[(8 * n + j) * NG + k]), hb = __half22float2(km[(8 * n + j + 4) * NG + k]);
                    x[0] = fmaf(ha.x, acc[k][0], fmaf(ha.y, qsum0[k], x[0]));
                    x[1] = fmaf(hb.x, acc[k][1], fmaf(hb.y, qsum0[k], x[1]));
                    x[2] = fmaf(ha.x, acc[k][2], fmaf(ha.y, qsum1[k], x[2]));
                    x[3] = fmaf(hb.x, acc[k][3], fmaf(hb.y, qsum1[k], x[3]));
                }
                s[n][0] = x[0] * rs0;
                s[n][1] = x[1] * rs0;
                s[n][2] = x[2] * rs1;
                s[n][3] = x[3] * rs1;
            }
            const int end = min(lq, limit_lo);
            const bool edge = t0 + kTile > end || bad_here;      // some row or some token of the tile is masked
            if (edge) {
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    const int ta = t0 + 8 * n + j, tb = ta + 4;
                    const bool gone = (bad_here >> (n >> 1)) & 1u;
                    if (gone || ta >= min(lq, lim0)) s[n][0] = -CUDART_INF_F;
                    if (gone || tb >= min(lq, lim0)) s[n][1] = -CUDART_INF_F;
                    if (gone || ta >= min(lq, lim1)) s[n][2] = -CUDART_INF_F;
                    if (gone || tb >= min(lq, lim1)) s[n][3] = -CUDART_INF_F;
                }
            }
            uint32_t pa[2][4];
            softmax_tile(s, pa);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int ta = 16 * u + j;      // value rows ta, ta + 4 (first register), ta + 8, ta + 12 (second)
                uint32_t hz[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    hz[k] = *reinterpret_cast<const uint32_t *>(&vm[(ta + 4 * k) * NG + g * NG / 8]);
                    // a row that holds nothing must not reach the product: 0 times what lies there need not be 0
                    if (edge && (t0 + ta + 4 * k >= lq || ((bad_here >> u) & 1u))) hz[k] = 0u;
                }
                const uint32_t h_a = __byte_perm(hz[0], hz[1], 0x5410), z_a = __byte_perm(hz[0], hz[1], 0x7632);
                const uint32_t h_b = __byte_perm(hz[2], hz[3], 0x5410), z_b = __byte_perm(hz[2], hz[3], 0x7632);
                uint32_t w[4][D / 64];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int t = ta + 4 * k, byte = g * (D / 16);
                    const uint8_t *src = buf + Geo::CODES + t * Geo::ROW + piece_at<D>(t, byte / 16) * 16 + byte % 16;
                    if constexpr (D == 128) {
                        const uint2 v = *reinterpret_cast<const uint2 *>(src);
                        w[k][0] = v.x;
                        w[k][1] = v.y;
                    } else {
                        w[k][0] = *reinterpret_cast<const uint32_t *>(src);
                    }
                }
#pragma unroll
                for (int q = 0; q < D / 64; ++q) {
#pragma unroll
                    for (int hf = 0; hf < 2; ++hf) {
                        const uint32_t sel = hf ? 0x7632 : 0x5410;
                        uint32_t x[4], y[4];      // channels 4 hf .. 4 hf + 3 of the word, two tokens each
                        // nibble k of both halves: pairs (token, token + 4) of channel 4 hf + k
                        nibble_pairs(__byte_perm(w[0][q], w[1][q], sel), x);
                        nibble_pairs(__byte_perm(w[2][q], w[3][q], sel), y);
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            mma16816(o[8 * q + 4 * hf + k], pa[u][0], pa[u][1], pa[u][2], pa[u][3], h2_fma(h_a, x[k], z_a), h2_fma(h_b, y[k], z_b));
                    }
                }
            }
            __syncwarp();
            fetch(tile + kStages - 1, stage == 0 ? kStages - 1 : stage - 1);
            stage = stage + 1 == kStages ? 0 : stage + 1;
        }
        cp_wait<0>();

        // ---- the window: 16-bit rows straight from the ring; the warps take its tiles in turn
        const int r0 = max(seg0, sc.tiles_c), r1 = max(min(seg1, sc.tiles_c + sc.tiles_r), r0);
        const int64_t win_row0 = ((int64_t)seq.slot * cfg.n_kv_heads + hk) * cfg.ring_tokens;
        for (int tile = r0 + warp; tile < r1; tile += kSplitWarps) {
            const int t0 = lq + (tile - sc.tiles_c) * kTile;
            if (t0 >= limit_hi) break;
            const T *kw = static_cast<const T *>(p.c.k_win), *vw = static_cast<const T *>(p.c.v_win);
            float s[4][4];
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const int t = min(t0 + 8 * n + (g >> 1) + 4 * (g & 1), L - 1);
                const T *src = kw + (win_row0 + t % cfg.ring_tokens) * D + 8 * j;
                float d[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int st = 0; st < Geo::SETS; ++st) {
                    uint4 x = *reinterpret_cast<const uint4 *>(src + 32 * st);
                    x.x = as_h2<T>(x.x); x.y = as_h2<T>(x.y); x.z = as_h2<T>(x.z); x.w = as_h2<T>(x.w);
                    mma16816(d, aq[2 * st][0], aq[2 * st][1], aq[2 * st][2], aq[2 * st][3], __byte_perm(x.x, x.z, 0x5410), __byte_perm(x.x, x.z, 0x7632));
                    mma16816(d, aq[2 * st + 1][0], aq[2 * st + 1][1], aq[2 * st + 1][2], aq[2 * st + 1][3], __byte_perm(x.y, x.w, 0x5410), __byte_perm(x.y, x.w, 0x7632));
                }
                const int ta = t0 + 8 * n + j, tb = ta + 4;
                s[n][0] = ta < lim0 ? d[0] * rs0 : -CUDART_INF_F;
                s[n][1] = tb < lim0 ? d[1] * rs0 : -CUDART_INF_F;
                s[n][2] = ta < lim1 ? d[2] * rs1 : -CUDART_INF_F;
                s[n][3] = tb < lim1 ? d[3] * rs1 : -CUDART_INF_F;
            }
            uint32_t pa[2][4];
            softmax_tile(s, pa);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                uint4 x[4][D / 64];      // rows ta, ta + 4, ta + 8, ta + 12, this lane's CPT channels
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int t = t0 + 16 * u + j + 4 * k;
                    const T *src = vw + (win_row0 + min(t, L - 1) % cfg.ring_tokens) * D + g * Geo::CPT;
#pragma unroll
                    for (int q = 0; q < D / 64; ++q) {
                        x[k][q] = t < L ? *reinterpret_cast<const uint4 *>(src + 8 * q) : make_uint4(0u, 0u, 0u, 0u);
                        x[k][q].x = as_h2<T>(x[k][q].x); x[k][q].y = as_h2<T>(x[k][q].y);
                        x[k][q].z = as_h2<T>(x[k][q].z); x[k][q].w = as_h2<T>(x[k][q].w);
                    }
                }
#pragma unroll
                for (int q = 0; q < D / 64; ++q) {
                    const uint32_t *e0 = &x[0][q].x, *e1 = &x[1][q].x, *e2 = &x[2][q].x, *e3 = &x[3][q].x;
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const uint32_t sel = k & 1 ? 0x7632 : 0x5410;
                        mma16816(o[8 * q + k], pa[u][0], pa[u][1], pa[u][2], pa[u][3], __byte_perm(e0[k >> 1], e1[k >> 1], sel), __byte_perm(e2[k >> 1], e3[k >> 1], sel));
                    }
                }
            }
        }

        // ---- join the four warps, in a fixed order
#pragma unroll
        for (int d = 1; d < 4; d <<= 1) {
            l0 += __shfl_xor_sync(0xffffffffu, l0, d);
            l1 += __shfl_xor_sync(0xffffffffu, l1, d);
        }
        if (j == 0) {
            ml_sh[warp][g][0] = m0; ml_sh[warp][g][1] = l0;
            ml_sh[warp][g + 8][0] = m1; ml_sh[warp][g + 8][1] = l1;
        }
        __syncthreads();      // also: no warp reads its ring any more
        float M0 = -CUDART_INF_F, M1 = -CUDART_INF_F, S0 = 0.f, S1 = 0.f;
#pragma unroll
        for (int w = 0; w < kSplitWarps; ++w) { M0 = fmaxf(M0, ml_sh[w][g][0]); M1 = fmaxf(M1, ml_sh[w][g + 8][0]); }
#pragma unroll
        for (int w = 0; w < kSplitWarps; ++w) {
            if (M0 != -CUDART_INF_F) S0 += ml_sh[w][g][1] * ex2_approx(ml_sh[w][g][0] - M0);
            if (M1 != -CUDART_INF_F) S1 += ml_sh[w][g + 8][1] * ex2_approx(ml_sh[w][g + 8][0] - M1);
        }
        {
            const float f0 = m0 == -CUDART_INF_F ? 0.f : ex2_approx(m0 - M0), fb = m1 == -CUDART_INF_F ? 0.f : ex2_approx(m1 - M1);
#pragma unroll
            for (int n = 0; n < Geo::CPT; ++n) { o[n][0] *= f0; o[n][1] *= f0; o[n][2] *= fb; o[n][3] *= fb; }
        }
        float *join = reinterpret_cast<float *>(smem);      // [2][CPT * 4][32 lanes]
#pragma unroll
        for (int round = 0; round < 2; ++round) {
            const int givers = round == 0 ? 2 : 1;      // warps givers .. 2*givers-1 hand over to 0 .. givers-1
            if (warp >= givers && warp < 2 * givers) {
#pragma unroll
                for (int n = 0; n < Geo::CPT; ++n)
                    *reinterpret_cast<float4 *>(join + (((warp - givers) * Geo::CPT + n) * 32 + lane) * 4) = make_float4(o[n][0], o[n][1], o[n][2], o[n][3]);
            }
            __syncthreads();
            if (warp < givers) {
#pragma unroll
                for (int n = 0; n < Geo::CPT; ++n) {
                    const float4 v = *reinterpret_cast<const float4 *>(join + ((warp * Geo::CPT + n) * 32 + lane) * 4);
                    o[n][0] += v.x; o[n][1] += v.y; o[n][2] += v.z; o[n][3] += v.w;
                }
            }
            __syncthreads();
        }
        const bool whole = off == 0 && take == sc.cost;
        float *rows = join;                      // [16][D], then written out by all threads
        float *part = partials + ((size_t)blockIdx.x * 2 + (off == 0 ? 1 : 0)) * kRowsPerItem * partial_stride(D);
        if (warp == 0) {
            const float i0 = S0 > 0.f || S0 != S0 ? 1.f / S0 : 0.f, i1 = S1 > 0.f || S1 != S1 ? 1.f / S1 : 0.f;
            const int32_t *rv = p.c.reorder_v ? p.c.reorder_v + hk * D : nullptr;
#pragma unroll
            for (int n = 0; n < Geo::CPT; ++n) {
                const int ca = 2 * j * Geo::CPT + n, cb = ca + Geo::CPT;      // stored channels of columns 2j, 2j + 1
                if (whole) {
                    const int da = rv ? rv[ca] & (D - 1) : ca, db = rv ? rv[cb] & (D - 1) : cb;
                    rows[g * D + da] = o[n][0] * i0; rows[g * D + db] = o[n][1] * i0;
                    rows[(g + 8) * D + da] = o[n][2] * i1; rows[(g + 8) * D + db] = o[n][3] * i1;
                } else {
                    rows[g * D + ca] = o[n][0]; rows[g * D + cb] = o[n][1];
                    rows[(g + 8) * D + ca] = o[n][2]; rows[(g + 8) * D + cb] = o[n][3];
                }
            }
            if (j == 0) {
                ml_sh[0][g][0] = M0; ml_sh[0][g][1] = S0;
                ml_sh[0][g + 8][0] = M1; ml_sh[0][g + 8][1] = S1;
            }
        }
        __syncthreads();
        for (int e = tid; e < R * D; e += kSplitThreads) {
            const int r = e / D, c = e % D;
            if (whole) {
                const int i = (row_base + r) / rep, head = hk * rep + (row_base + r) % rep;
                static_cast<T *>(a.out)[(int64_t)(seq.row0 + i) * a.out_stride + head * D + c] = Elem<T>::from_float(rows[r * D + c]);
            } else {
                part[r * partial_stride(D) + c] = rows[r * D + c];
            }
        }
        if (tid < R) {
            const float m = ml_sh[0][tid][0], l = ml_sh[0][tid][1];
            if (!whole) {
                part[tid * partial_stride(D) + D] = m;
                part[tid * partial_stride(D) + D + 1] = l;
            } else if (a.lse) {
                const int i = (row_base + tid) / rep, head = hk * rep + (row_base + tid) % rep;
                a.lse[(int64_t)(seq.row0 + i) * cfg.n_q_heads + head] = m == -CUDART_INF_F ? m : (m + log2f(l) - kPScaleLog2) * 0.6931471805599453f;
            }
        }
        if (!whole && off == 0 && tid == 0) {
            const long long last = (pre[b] + (item + 1) * sc.cost - 1) / ups;
            desc[1] = seq.row0; desc[2] = seq.n; desc[3] = hk; desc[4] = mt; desc[5] = (int)(last - blockIdx.x + 1);
            desc[0] = 1;
        }
        f += take;
        __syncthreads();      // the pool is reused by the next segment
    }
}

// Joins the partials of an item that several runs share: one CTA per (run that begins the item, row).
template <typename T, int D>
__global__ void __launch_bounds__(D) paged_merge_kernel(const __grid_constant__ SplitArgs args)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const PagedAttnArgs &a = args.a;
    const skvq_paged_config &cfg = a.p.cfg;
    const int slot = blockIdx.x, r = blockIdx.y, c = threadIdx.x;
    const int *desc = reinterpret_cast<const int *>(a.ws) + (size_t)slot * kDescInts;
    if (desc[0] == 0) return;
    const int rep = cfg.n_q_heads / cfg.n_kv_heads, row = desc[4] * kRowsPerItem + r;
    if (row >= desc[2] * rep) return;
    const int n = desc[5], hk = desc[3];
    constexpr int PS = partial_stride(D);
    const float *base = a.ws + (size_t)args.n_slots * kDescInts + ((size_t)slot * 2 * kRowsPerItem + r) * PS;
    auto partial = [&](int k) { return base + (size_t)(2 * k + (k == 0 ? 1 : 0)) * kRowsPerItem * PS; };
    float m = -CUDART_INF_F;
    for (int k = 0; k < n; ++k) m = fmaxf(m, partial(k)[D]);
    float o = 0.f, l = 0.f;
    if (m != -CUDART_INF_F) {
#pragma unroll 4
        for (int k = 0; k < n; ++k) {
            const float *q = partial(k);
            const float f = ex2_approx(q[D] - m);
            l = fmaf(q[D + 1], f, l);
            o = fmaf(q[c], f, o);
        }
    }
    const int i = row / rep, head = hk * rep + row % rep;
    const int dst = a.p.c.reorder_v ? a.p.c.reorder_v[hk * D + c] & (D - 1) : c;
    static_cast<T *>(a.out)[(int64_t)(desc[1] + i) * a.out_stride + head * D + dst] = Elem<T>::from_float(l > 0.f || l != l ? o / l : 0.f);
    if (a.lse && c == 0)
        a.lse[(int64_t)(desc[1] + i) * cfg.n_q_heads + head] = m == -CUDART_INF_F ? m : (m + log2f(l) - kPScaleLog2) * 0.6931471805599453f;
}

int split_slots(const skvq_paged_config &cfg, const skvq_paged_batch &batch, int n_splits)
{
    const long long rep = cfg.n_q_heads / cfg.n_kv_heads, m_tiles = (batch.max_new * rep + kRowsPerItem - 1) / kRowsPerItem;
    const long long lq = batch.max_len > cfg.window ? batch.max_len - cfg.window : 0;
    const long long cost = (lq + kTile - 1) / kTile + kRingCost * ((batch.max_len - lq + kTile - 1) / kTile) + 1;
    const long long items = (long long)batch.n_seqs * cfg.n_kv_heads * m_tiles;
    long long slots;
    if (n_splits > 0) slots = (long long)n_splits * items;
    else {
        // one wave of resident CTAs, each with two tiles per warp at least: a shorter run costs more to join than it saves
        slots = 3LL * sm_count();
        if (slots > items * cost / 8) slots = items * cost / 8;
    }
    if (slots > items * cost) slots = items * cost;
    if (slots > 16384) slots = 16384;
    return slots < 1 ? 1 : (int)slots;
}

template <typename Kern, typename Args>
cudaError_t launch_chained(Kern kern, dim3 grid, int threads, size_t smem, cudaStream_t stream, const Args &args)
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

template <typename T, int D, int NG>
cudaError_t launch_split(const PagedAttnArgs &a, cudaStream_t stream)
{
    SplitArgs s{a, split_slots(a.p.cfg, a.p.batch, a.n_splits)};
    const size_t smem = Geometry<D, NG>::SMEM + sizeof(long long) * (a.p.batch.n_seqs + 1);
    static unsigned long long done = 0;
    cudaError_t e = configure_smem_once(paged_split_kernel<T, D, NG>, Geometry<D, NG>::SMEM + (int)sizeof(long long) * (kMaxPagedSeqs + 1), done);
    if (e != cudaSuccess) return e;
    e = launch_chained(paged_split_kernel<T, D, NG>, dim3(s.n_slots), kSplitThreads, smem, stream, s);
    if (e != cudaSuccess) return e;
    return launch_chained(paged_merge_kernel<T, D>, dim3(s.n_slots, kRowsPerItem), D, 0, stream, s);
}

template <typename T> cudaError_t launch_by_shape(const PagedAttnArgs &a, cudaStream_t stream)
{
    if (a.p.cfg.head_dim == 128)
        return a.p.ng == 1 ? launch_split<T, 128, 1>(a, stream) : a.p.ng == 2 ? launch_split<T, 128, 2>(a, stream) : launch_split<T, 128, 4>(a, stream);
    return a.p.ng == 1 ? launch_split<T, 64, 1>(a, stream) : launch_split<T, 64, 2>(a, stream);
}

}  // namespace

size_t paged_workspace_bytes(const skvq_paged_config &cfg, const skvq_paged_batch &batch, int n_splits)
{
    const size_t slots = split_slots(cfg, batch, n_splits);
    return slots * kDescInts * 4 + slots * 2 * kRowsPerItem * partial_stride(cfg.head_dim) * 4;
}

cudaError_t launch_paged_attention(const PagedAttnArgs &a, cudaStream_t stream)
{
    return a.p.cfg.dtype == SKVQ_F16 ? launch_by_shape<__half>(a, stream) : launch_by_shape<__nv_bfloat16>(a, stream);
}

}  // namespace skvq
