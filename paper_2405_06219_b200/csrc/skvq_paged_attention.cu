// skvq_paged_attention for few query rows per (sequence, KV head): single-token decode, drafted tokens.
//
// The rows of a KV head are packed: row = new token * (Hq/Hkv) + query head, 8 NT rows per item (NT = 1, 2 or 4).  Items of
// the whole batch are laid end to end, priced in 32-token tiles (a tile of the unquantized window costs kRingCost), and cut
// into equal runs, one per CTA: ragged batches and long single sequences load the GPU alike.  The four warps of a CTA take
// quarters of a run, stream their tiles through private shared-memory rings, and join their softmax states at the end; an item
// that several CTAs share is joined by the merge kernel.
//
// With q' the rotated, reordered query, the scores of a quantized token are formed without dequantizing the key:
//   q'.K~_t = sum_g h_{t,g} (sum_{j in g} q'_j c_{t,j}) + sum_g z_{t,g} (sum_{j in g} q'_j)
// the inner sums on mma.m16n8k16 with fp32 accumulators, one per group: 16 tokens' codes (exact in fp16) are the A operand, 8
// query rows the B operand, so that what costs instructions -- unpacking codes -- is shared by all rows and a single query
// wastes no more than the 8 columns.  Values are formed as fp16(h c + z) in registers (one rounding, 2^-11 at most) as the A
// operand of the transposed product (V~^T P^T) and multiplied by the probabilities in fp16.  A probability is held times 2^14
// relative to the running maximum: fp16 then resolves 2^-38 of the largest, so a million small ones still add up; their
// sum is kept in fp32.
// Fragments: the channels of a k-step and the tokens of a row are free to choose as long as both operands agree.  A lane's
// registers of the score product are the nibble pairs (i, i+4) of one 32-bit word, a word of every lane inside one
// 32-channel granule; of the value product they pair one channel of tokens j and j+4.  Neither operand passes through shared
// memory a second time; only the 16 x 8 probabilities are transposed (movmatrix).
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
constexpr int kTile = 32;             // tokens per warp tile
constexpr int kRingCost = 4;          // a window tile moves 16-bit rows: about four times the bytes
constexpr int kStages = 2;
constexpr float kPScaleLog2 = 14.0f;

struct SplitArgs {
    PagedAttnArgs a;
    int n_slots;
    int rows;      // rows per item: 8 NT
};

// Workspace: descriptor [n_slots][8] ints, then partials [n_slots][2][rows][D + 4] floats {o[D], m, l, pad}.  A run holds at
// most one item that it continues (partial 0) and one that it begins and does not finish (partial 1).
constexpr int kDescInts = 8;
__host__ __device__ constexpr int partial_stride(int D) { return D + 4; }

template <int D, int NG, int NT>
struct Geometry {
    static constexpr int ROW = D / 2;                  // bytes of a code row
    static constexpr int CHUNKS = ROW / 16;
    static constexpr int CODES = kTile * ROW;
    static constexpr int META = kTile * NG * 4;
    static constexpr int STAGE = 2 * CODES + 2 * META;
    static constexpr int SETS = D / 32;                // 32-channel granules
    static constexpr int CPT = D / 8;                  // value channels per lane
    static constexpr int MT = D / 16;                  // 16-channel tiles of the value product
    static constexpr int ROWS = 8 * NT;
    static constexpr int QROW = D + 8;                 // halves per query row in shared memory
    static constexpr int JROW = D + 4;                 // floats per row of a warp's accumulators in shared memory
    static constexpr int RINGS = kSplitWarps * kStages * STAGE;
    static constexpr int JOIN = kSplitWarps * ROWS * JROW * 4;
    static constexpr int POOL = RINGS > JOIN ? RINGS : JOIN;      // both hold, at other times, the raw queries too
    static constexpr int SMEM = POOL + ROWS * QROW * 2;
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
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v)      // of 16-bit elements; lane 4r + c holds columns 2c, 2c + 1 of row r
{
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
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
    int m_tiles;               // items per KV head
};
__device__ __forceinline__ SeqCost seq_cost(const PagedArgs &p, const PagedSeq &s, int rows)
{
    SeqCost c;
    const int rep = p.cfg.n_q_heads / p.cfg.n_kv_heads;
    const int lq = max(s.len - p.cfg.window, 0);
    c.tiles_c = (lq + kTile - 1) / kTile;
    c.tiles_r = (s.len - lq + kTile - 1) / kTile;
    c.cost = max(c.tiles_c + kRingCost * c.tiles_r, 1);
    c.m_tiles = (s.n * rep + rows - 1) / rows;
    return c;
}

template <typename T, int D, int NG, int NT>
__global__ void __launch_bounds__(kSplitThreads, NT == 4 ? 2 : (NT == 2 ? 3 : 4)) paged_split_kernel(const __grid_constant__ SplitArgs args)
{
    using Geo = Geometry<D, NG, NT>;
    constexpr int ROWS = Geo::ROWS;
    const PagedAttnArgs &a = args.a;
    const PagedArgs &p = a.p;
    const skvq_paged_config &cfg = p.cfg;
    extern __shared__ __align__(128) uint8_t smem[];
    long long *pre = reinterpret_cast<long long *>(smem + Geo::SMEM);      // [n_seqs + 1] cost of the sequences before b
    __half *qs = reinterpret_cast<__half *>(smem + Geo::POOL);
    __shared__ long long scan_sh[kSplitWarps];
    __shared__ float row_scale[ROWS], q_sum[ROWS][4];
    __shared__ float ml_sh[kSplitWarps][ROWS][2];
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
                    const SeqCost sc = seq_cost(p, s, ROWS);
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
        const SeqCost sc = seq_cost(p, seq, ROWS);
        const long long item = (f - pre[b]) / sc.cost;
        const int off = (int)((f - pre[b]) - item * sc.cost);
        const int take = (int)min((long long)(sc.cost - off), f1 - f);
        const int hk = (int)(item / sc.m_tiles), mt = (int)(item - (long long)hk * sc.m_tiles);
        const int row_base = mt * ROWS, R = min(ROWS, seq.n * rep - row_base);
        const int L = seq.len, lq = max(L - cfg.window, 0);
        // rows see tokens below their limit
        auto row_limit = [&](int r) { return a.causal ? min(L, L - seq.n + (row_base + min(r, R - 1)) / rep + 1) : L; };
        const int limit_lo = row_limit(0), limit_hi = row_limit(R - 1);
        int lim[NT][2];      // of this lane's columns of the score product: rows 8 n + 2 j, 8 n + 2 j + 1
#pragma unroll
        for (int n = 0; n < NT; ++n) { lim[n][0] = row_limit(8 * n + 2 * j); lim[n][1] = row_limit(8 * n + 2 * j + 1); }

        // ---- this warp's quarter of the run; its first pages are on their way while the queries are prepared
        auto tile_of = [&](int x) { return x <= sc.tiles_c ? x : sc.tiles_c + (x - sc.tiles_c + kRingCost - 1) / kRingCost; };
        const int seg0 = tile_of(off), seg1 = tile_of(off + take);
        const int c0 = min(seg0, sc.tiles_c), c1 = max(min(min(seg1, sc.tiles_c), (limit_hi + kTile - 1) / kTile), c0);
        const int q0 = c0 + (int)((long long)(c1 - c0) * warp / kSplitWarps), q1 = c0 + (int)((long long)(c1 - c0) * (warp + 1) / kSplitWarps);
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

        // ---- queries: rotate, round to T, reorder; fp16 rows (bf16 rows times a power of two), group sums
        for (int r = tid >> 3; r < ROWS; r += kSplitThreads / 8) {
            const int part = tid & 7;      // 8 threads per row, CPT channels each
            T *raw = reinterpret_cast<T *>(smem);        // [ROWS][D], before the rings are in use
            const int i = (row_base + r) / rep, head = hk * rep + (row_base + r) % rep;
            const int pos = L - seq.n + i;
            const T *src = static_cast<const T *>(a.q) + (int64_t)(seq.row0 + i) * a.q_stride + (int64_t)head * D;
            if (r < R) {
                const float2 *rope = static_cast<const float2 *>(p.rope.table);
                const int half = p.rope.rot_dim / 2;
#pragma unroll 4
                for (int k = 0; k < Geo::CPT; ++k) {
                    const int c = part + 8 * k;
                    T x = src[c];
                    if (rope && pos >= 0 && c < p.rope.rot_dim) {
                        const bool second = p.rope.interleaved ? c & 1 : c >= half;
                        const int pair = p.rope.interleaved ? c >> 1 : (second ? c - half : c);
                        const int partner = p.rope.interleaved ? c ^ 1 : (second ? c - half : c + half);
                        const float2 cs = rope[(int64_t)pos * half + pair];
                        const float own = Elem<T>::to_float(x), other = Elem<T>::to_float(src[partner]);
                        x = Elem<T>::from_float(second ? rotate_second(other, own, cs.x, cs.y) : rotate_first(own, other, cs.x, cs.y));
                    }
                    raw[r * D + c] = x;
                }
            }
            __syncwarp();
            float x[Geo::CPT], mx = 0.f, sum = 0.f;
#pragma unroll
            for (int k = 0; k < Geo::CPT; ++k) {
                const int c = part * Geo::CPT + k;
                const int s = p.c.reorder_k ? p.c.reorder_k[hk * D + c] & (D - 1) : c;
                x[k] = r < R ? Elem<T>::to_float(raw[r * D + s]) : 0.f;
                mx = fmaxf(mx, fabsf(x[k]));
            }
            float up = 1.f;
            if (!__is_same(T, __half)) {
                // bf16 has more range than fp16: bring the row's largest to [2^13, 2^14), exactly
#pragma unroll
                for (int m = 1; m < 8; m <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, m));
                if (mx > 0.f && mx < CUDART_INF_F) {
                    int e;
                    frexpf(mx, &e);
                    up = ldexpf(1.f, min(14 - e, 126));
                }
            }
#pragma unroll
            for (int k = 0; k < Geo::CPT; ++k) {
                const __half v = __float2half_rn(x[k] * up);
                sum += __half2float(v);
                qs[r * Geo::QROW + part * Geo::CPT + k] = v;
            }
            const int per_group = 8 / NG;
#pragma unroll
            for (int m = 1; m < per_group; m <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, m);
            if (part % per_group == 0) q_sum[r][part / per_group] = sum;
            if (part == 0) row_scale[r] = a.sm_scale * 1.4426950408889634f / up;
        }
        __syncthreads();
        uint32_t bq[NT][Geo::SETS * 2][2];
        float rs[NT][2], qsum[NT][2][NG];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int s = 0; s < Geo::SETS; ++s) {
                const uint4 x = *reinterpret_cast<const uint4 *>(qs + (8 * n + g) * Geo::QROW + 32 * s + 8 * j);
                bq[n][2 * s][0] = __byte_perm(x.x, x.z, 0x5410);
                bq[n][2 * s][1] = __byte_perm(x.x, x.z, 0x7632);
                bq[n][2 * s + 1][0] = __byte_perm(x.y, x.w, 0x5410);
                bq[n][2 * s + 1][1] = __byte_perm(x.y, x.w, 0x7632);
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                rs[n][e] = row_scale[8 * n + 2 * j + e];
#pragma unroll
                for (int k = 0; k < NG; ++k) qsum[n][e][k] = q_sum[8 * n + 2 * j + e][k];
            }
        }

        float o[NT][Geo::MT][4];      // [.][channel pair][{first, second channel} x {row 2j, row 2j + 1}]
        float m_run[NT][2], l_run[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int m = 0; m < Geo::MT; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[n][m][e] = 0.f;
#pragma unroll
            for (int e = 0; e < 2; ++e) { m_run[n][e] = -CUDART_INF_F; l_run[n][e] = 0.f; }
        }

        // Scores (log2 domain) of 32 tokens -> probabilities as B fragments.  s[u][n] = {token a: rows 2j, 2j+1; token a + 8: the
        // same}, token a = 16 u + (g >> 1) + 4 (g & 1).
        auto softmax_tile = [&](float (&s)[2][NT][4], uint32_t (&pb)[2][NT][2]) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float x[2], base[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    x[e] = fmaxf(fmaxf(s[0][n][e], s[0][n][2 + e]), fmaxf(s[1][n][e], s[1][n][2 + e]));
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) x[e] = fmaxf(x[e], __shfl_xor_sync(0xffffffffu, x[e], d));
                    x[e] = fmaxf(x[e], m_run[n][e]);
                }
                if (__any_sync(0xffffffffu, x[0] > m_run[n][0] || x[1] > m_run[n][1])) {
                    float down[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        down[e] = x[e] > m_run[n][e] ? ex2_approx(m_run[n][e] - x[e]) : 1.f;
                        l_run[n][e] *= down[e];
                        m_run[n][e] = x[e];
                    }
#pragma unroll
                    for (int m = 0; m < Geo::MT; ++m) { o[n][m][0] *= down[0]; o[n][m][1] *= down[1]; o[n][m][2] *= down[0]; o[n][m][3] *= down[1]; }
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) base[e] = (m_run[n][e] == -CUDART_INF_F ? 0.f : m_run[n][e]) - kPScaleLog2;
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    float v[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = ex2_approx(s[u][n][e] - base[e & 1]);
                    l_run[n][0] += v[0] + v[2];
                    l_run[n][1] += v[1] + v[3];
                    pb[u][n][0] = transpose8x8(pack_h2(v[0], v[1]));
                    pb[u][n][1] = transpose8x8(pack_h2(v[2], v[3]));
                }
            }
        };

        // ---- quantized tokens
        const uint32_t ring = smem_u32(smem) + warp * kStages * Geo::STAGE;
        const uint8_t *ring_ptr = smem + warp * kStages * Geo::STAGE;
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
                const int64_t ra = ((int64_t)ida * cfg.n_kv_heads + hk) * P + ((tile * kTile) & (P - 1));
                const int64_t rb = ((int64_t)idb * cfg.n_kv_heads + hk) * P + ((tile * kTile + 16) & (P - 1));
#pragma unroll
                for (int k = 0; k < Geo::CHUNKS; ++k) {
                    const int q = k * 32 + lane, t = q / Geo::CHUNKS, c = q % Geo::CHUNKS;
                    const bool first = k < Geo::CHUNKS / 2;      // rows 0-15
                    if ((first ? ida : idb) >= 0) {
                        const int64_t at = ((first ? ra : rb) + (t & 15)) * Geo::ROW + c * 16;
                        const uint32_t dst = base + t * Geo::ROW + piece_at<D>(t, c) * 16;
                        cp16(dst, static_cast<const uint8_t *>(p.c.k_codes) + at);
                        cp16(dst + Geo::CODES, static_cast<const uint8_t *>(p.c.v_codes) + at);
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
        const int tok = (g >> 1) + 4 * (g & 1);      // the token of row g of the score product, inside its 8
        const int end = min(lq, limit_lo);
#pragma unroll 1
        for (int tile = q0; tile < q1; ++tile) {
            fetch(tile + kStages - 1, stage == 0 ? kStages - 1 : stage - 1);
            cp_wait<kStages - 1>();
            __syncwarp();
            const uint8_t *buf = ring_ptr + stage * Geo::STAGE;
            const uint32_t bad_here = (bad >> (2 * stage)) & 3u;
            const int t0 = tile * kTile;
            const uint32_t *km = reinterpret_cast<const uint32_t *>(buf + 2 * Geo::CODES), *vm = reinterpret_cast<const uint32_t *>(buf + 2 * Geo::CODES + Geo::META);
            float s[2][NT][4];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int t = 16 * u + tok;
                float acc[NT][NG][4];
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int k = 0; k < NG; ++k)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[n][k][e] = 0.f;
#pragma unroll
                for (int st = 0; st < Geo::SETS; ++st) {
                    uint32_t x[4], y[4];
                    nibble_pairs(*reinterpret_cast<const uint32_t *>(buf + t * Geo::ROW + piece_at<D>(t, st) * 16 + j * 4), x);
                    nibble_pairs(*reinterpret_cast<const uint32_t *>(buf + (t + 8) * Geo::ROW + piece_at<D>(t, st) * 16 + j * 4), y);
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        float (&d)[4] = acc[n][st * NG / Geo::SETS];
                        mma16816(d, x[0], y[0], x[1], y[1], bq[n][2 * st][0], bq[n][2 * st][1]);
                        mma16816(d, x[2], y[2], x[3], y[3], bq[n][2 * st + 1][0], bq[n][2 * st + 1][1]);
                    }
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[u][n][e] = 0.f;
#pragma unroll
                for (int k = 0; k < NG; ++k) {
                    const uint32_t ma = km[t * NG + k], mb = km[(t + 8) * NG + k];
                    const float2 ha = __half22float2(*reinterpret_cast<const __half2 *>(&ma)), hb = __half22float2(*reinterpret_cast<const __half2 *>(&mb));
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            s[u][n][e] = fmaf(ha.x, acc[n][k][e], fmaf(ha.y, qsum[n][e][k], s[u][n][e]));
                            s[u][n][2 + e] = fmaf(hb.x, acc[n][k][2 + e], fmaf(hb.y, qsum[n][e][k], s[u][n][2 + e]));
                        }
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[u][n][e] *= rs[n][e & 1];
            }
            const bool edge = t0 + kTile > end || bad_here;      // some row or some token of the tile is masked
            if (edge) {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int ta = t0 + 16 * u + tok;
                    const bool gone = (bad_here >> u) & 1u;
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (gone || ta + 8 * (e >> 1) >= min(lq, lim[n][e & 1])) s[u][n][e] = -CUDART_INF_F;
                }
            }
            uint32_t pb[2][NT][2];
            softmax_tile(s, pb);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int ta = 16 * u + j;      // value rows ta, ta + 4 (first k half), ta + 8, ta + 12 (second)
                uint32_t hz[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    hz[k] = vm[(ta + 4 * k) * NG + g * NG / 8];
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
                        uint32_t x[4], y[4];      // channels 4 hf .. 4 hf + 3 of the word, pairs (token, token + 4)
                        nibble_pairs(__byte_perm(w[0][q], w[1][q], sel), x);
                        nibble_pairs(__byte_perm(w[2][q], w[3][q], sel), y);
#pragma unroll
                        for (int k = 0; k < 4; ++k) { x[k] = h2_fma(h_a, x[k], z_a); y[k] = h2_fma(h_b, y[k], z_b); }
#pragma unroll
                        for (int k = 0; k < 2; ++k)
#pragma unroll
                            for (int n = 0; n < NT; ++n)
                                mma16816(o[n][4 * q + 2 * hf + k], x[2 * k], x[2 * k + 1], y[2 * k], y[2 * k + 1], pb[u][n][0], pb[u][n][1]);
                    }
                }
            }
            __syncwarp();
            stage = stage + 1 == kStages ? 0 : stage + 1;
        }
        cp_wait<0>();

        // ---- the window: 16-bit rows straight from the ring; the warps take its tiles in turn
        const int r0 = max(seg0, sc.tiles_c), r1 = max(min(seg1, sc.tiles_c + sc.tiles_r), r0);
        const int64_t win_row0 = ((int64_t)seq.slot * cfg.n_kv_heads + hk) * cfg.ring_tokens;
        auto ring_row = [&](int t) { return win_row0 + min(t, L - 1) % cfg.ring_tokens; };
#pragma unroll 1
        for (int tile = r0 + warp; tile < r1; tile += kSplitWarps) {
            const int t0 = lq + (tile - sc.tiles_c) * kTile;
            if (t0 >= limit_hi) break;
            const T *kw = static_cast<const T *>(p.c.k_win), *vw = static_cast<const T *>(p.c.v_win);
            float s[2][NT][4];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int ta = t0 + 16 * u + tok;
                const T *src_a = kw + ring_row(ta) * D + 8 * j, *src_b = kw + ring_row(ta + 8) * D + 8 * j;
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[u][n][e] = 0.f;
#pragma unroll
                for (int st = 0; st < Geo::SETS; ++st) {
                    uint4 x = *reinterpret_cast<const uint4 *>(src_a + 32 * st), y = *reinterpret_cast<const uint4 *>(src_b + 32 * st);
                    x.x = as_h2<T>(x.x); x.y = as_h2<T>(x.y); x.z = as_h2<T>(x.z); x.w = as_h2<T>(x.w);
                    y.x = as_h2<T>(y.x); y.y = as_h2<T>(y.y); y.z = as_h2<T>(y.z); y.w = as_h2<T>(y.w);
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        mma16816(s[u][n], __byte_perm(x.x, x.z, 0x5410), __byte_perm(y.x, y.z, 0x5410), __byte_perm(x.x, x.z, 0x7632),
                                 __byte_perm(y.x, y.z, 0x7632), bq[n][2 * st][0], bq[n][2 * st][1]);
                        mma16816(s[u][n], __byte_perm(x.y, x.w, 0x5410), __byte_perm(y.y, y.w, 0x5410), __byte_perm(x.y, x.w, 0x7632),
                                 __byte_perm(y.y, y.w, 0x7632), bq[n][2 * st + 1][0], bq[n][2 * st + 1][1]);
                    }
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[u][n][e] = ta + 8 * (e >> 1) < lim[n][e & 1] ? s[u][n][e] * rs[n][e & 1] : -CUDART_INF_F;
            }
            uint32_t pb[2][NT][2];
            softmax_tile(s, pb);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
#pragma unroll
                for (int q = 0; q < D / 64; ++q) {
                    uint32_t e[4][4];      // rows ta, ta + 4, ta + 8, ta + 12, eight of this lane's channels
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int t = t0 + 16 * u + j + 4 * k;
                        uint4 x = make_uint4(0u, 0u, 0u, 0u);
                        if (t < L) x = *reinterpret_cast<const uint4 *>(vw + ring_row(t) * D + g * Geo::CPT + 8 * q);
                        e[k][0] = as_h2<T>(x.x); e[k][1] = as_h2<T>(x.y); e[k][2] = as_h2<T>(x.z); e[k][3] = as_h2<T>(x.w);
                    }
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int n = 0; n < NT; ++n)
                            mma16816(o[n][4 * q + k], __byte_perm(e[0][k], e[1][k], 0x5410), __byte_perm(e[0][k], e[1][k], 0x7632),
                                     __byte_perm(e[2][k], e[3][k], 0x5410), __byte_perm(e[2][k], e[3][k], 0x7632), pb[u][n][0], pb[u][n][1]);
                }
            }
        }

        // ---- join the four warps, in a fixed order
        __syncthreads();      // no warp reads its ring any more
        float *join = reinterpret_cast<float *>(smem);      // [warp][row][D]: channel c at (c % CPT) * 8 + c / CPT, so lanes write side by side
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = 8 * n + 2 * j + e;
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) l_run[n][e] += __shfl_xor_sync(0xffffffffu, l_run[n][e], d);
                if (g == 0) { ml_sh[warp][r][0] = m_run[n][e]; ml_sh[warp][r][1] = l_run[n][e]; }
                if (r < R) {
                    float *row = join + (warp * ROWS + r) * Geo::JROW + g;
#pragma unroll
                    for (int m = 0; m < Geo::MT; ++m) { row[16 * m] = o[n][m][e]; row[16 * m + 8] = o[n][m][2 + e]; }
                }
            }
        }
        __syncthreads();
        const bool whole = off == 0 && take == sc.cost;
        float *part = partials + ((size_t)blockIdx.x * 2 + (off == 0 ? 1 : 0)) * ROWS * partial_stride(D);
        const int32_t *rv = p.c.reorder_v ? p.c.reorder_v + hk * D : nullptr;
        constexpr int LANES = kSplitThreads / D;      // rows side by side
        const int c = tid % D, dst = rv ? rv[c] & (D - 1) : c;
        for (int r = tid / D; r < R; r += LANES) {
            float M = -CUDART_INF_F, l = 0.f, v = 0.f;
#pragma unroll
            for (int w = 0; w < kSplitWarps; ++w) M = fmaxf(M, ml_sh[w][r][0]);
            if (M != -CUDART_INF_F) {
#pragma unroll
                for (int w = 0; w < kSplitWarps; ++w) {
                    const float k = ex2_approx(ml_sh[w][r][0] - M);
                    l = fmaf(ml_sh[w][r][1], k, l);
                    v = fmaf(join[(w * ROWS + r) * Geo::JROW + (c % Geo::CPT) * 8 + c / Geo::CPT], k, v);
                }
            }
            if (whole) {
                const int i = (row_base + r) / rep, head = hk * rep + (row_base + r) % rep;
                static_cast<T *>(a.out)[(int64_t)(seq.row0 + i) * a.out_stride + head * D + dst] = Elem<T>::from_float(M == -CUDART_INF_F ? 0.f : v / l);
                if (a.lse && c == 0)
                    a.lse[(int64_t)(seq.row0 + i) * cfg.n_q_heads + head] = M == -CUDART_INF_F ? M : (M + log2f(l) - kPScaleLog2) * 0.6931471805599453f;
            } else {
                part[r * partial_stride(D) + c] = v;
                if (c == 0) { part[r * partial_stride(D) + D] = M; part[r * partial_stride(D) + D + 1] = l; }
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
    const int rep = cfg.n_q_heads / cfg.n_kv_heads, row = desc[4] * args.rows + r;
    if (row >= desc[2] * rep) return;
    const int n = desc[5], hk = desc[3];
    constexpr int PS = partial_stride(D);
    const float *base = a.ws + (size_t)args.n_slots * kDescInts + ((size_t)slot * 2 * args.rows + r) * PS;
    auto partial = [&](int k) { return base + (size_t)(2 * k + (k == 0 ? 1 : 0)) * args.rows * PS; };
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
    static_cast<T *>(a.out)[(int64_t)(desc[1] + i) * a.out_stride + head * D + dst] = Elem<T>::from_float(m == -CUDART_INF_F ? 0.f : o / l);
    if (a.lse && c == 0)
        a.lse[(int64_t)(desc[1] + i) * cfg.n_q_heads + head] = m == -CUDART_INF_F ? m : (m + log2f(l) - kPScaleLog2) * 0.6931471805599453f;
}

// Rows per item: 8, 16 or 32, by the most rows a KV head can have.
int item_rows(const skvq_paged_config &cfg, const skvq_paged_batch &batch)
{
    const long long rows = (long long)batch.max_new * (cfg.n_q_heads / cfg.n_kv_heads);
    return rows <= 8 ? 8 : (rows <= 16 ? 16 : 32);
}

int split_slots(const skvq_paged_config &cfg, const skvq_paged_batch &batch, int n_splits)
{
    const int per = item_rows(cfg, batch);
    const long long rep = cfg.n_q_heads / cfg.n_kv_heads, m_tiles = (batch.max_new * rep + per - 1) / per;
    const long long lq = batch.max_len > cfg.window ? batch.max_len - cfg.window : 0;
    const long long cost = (lq + kTile - 1) / kTile + kRingCost * ((batch.max_len - lq + kTile - 1) / kTile) + 1;
    const long long items = (long long)batch.n_seqs * cfg.n_kv_heads * m_tiles;
    long long slots;
    if (n_splits > 0) slots = (long long)n_splits * items;
    else {
        // one wave of resident CTAs, each with two tiles per warp at least: a shorter run costs more to join than it saves
        slots = (per == 8 ? 4LL : (per == 16 ? 3LL : 2LL)) * sm_count();
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

template <typename T, int D, int NG, int NT>
cudaError_t launch_split(const PagedAttnArgs &a, cudaStream_t stream)
{
    using Geo = Geometry<D, NG, NT>;
    const SplitArgs s{a, split_slots(a.p.cfg, a.p.batch, a.n_splits), Geo::ROWS};
    static unsigned long long done = 0;
    cudaError_t e = configure_smem_once(paged_split_kernel<T, D, NG, NT>, Geo::SMEM + (int)sizeof(long long) * (kMaxPagedSeqs + 1), done);
    if (e != cudaSuccess) return e;
    e = launch_chained(paged_split_kernel<T, D, NG, NT>, dim3(s.n_slots), kSplitThreads, Geo::SMEM + sizeof(long long) * (a.p.batch.n_seqs + 1), stream, s);
    if (e != cudaSuccess) return e;
    return launch_chained(paged_merge_kernel<T, D>, dim3(s.n_slots, Geo::ROWS), D, 0, stream, s);
}

template <typename T, int D, int NG> cudaError_t launch_by_rows(const PagedAttnArgs &a, cudaStream_t stream)
{
    const int rows = item_rows(a.p.cfg, a.p.batch);
    return rows == 8 ? launch_split<T, D, NG, 1>(a, stream) : rows == 16 ? launch_split<T, D, NG, 2>(a, stream) : launch_split<T, D, NG, 4>(a, stream);
}

template <typename T> cudaError_t launch_by_shape(const PagedAttnArgs &a, cudaStream_t stream)
{
    if (a.p.cfg.head_dim == 128)
        return a.p.ng == 1 ? launch_by_rows<T, 128, 1>(a, stream) : a.p.ng == 2 ? launch_by_rows<T, 128, 2>(a, stream) : launch_by_rows<T, 128, 4>(a, stream);
    return a.p.ng == 1 ? launch_by_rows<T, 64, 1>(a, stream) : launch_by_rows<T, 64, 2>(a, stream);
}

}  // namespace

size_t paged_workspace_bytes(const skvq_paged_config &cfg, const skvq_paged_batch &batch, int n_splits)
{
    const size_t slots = split_slots(cfg, batch, n_splits);
    return slots * kDescInts * 4 + slots * 2 * item_rows(cfg, batch) * partial_stride(cfg.head_dim) * 4;
}

cudaError_t launch_paged_attention(const PagedAttnArgs &a, cudaStream_t stream)
{
    return a.p.cfg.dtype == SKVQ_F16 ? launch_by_shape<__half>(a, stream) : launch_by_shape<__nv_bfloat16>(a, stream);
}

}  // namespace skvq
