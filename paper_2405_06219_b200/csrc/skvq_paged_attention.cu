// skvq_paged_attention for few query rows per (sequence, KV head): single-token decode, drafted tokens.
//
// The rows of a KV head are packed: row = new token * (Hq/Hkv) + query head, 8 NT rows per item (NT = 1 or 2).  Items of
// the whole batch are laid end to end, priced in 32-token tiles (a tile of the unquantized window costs kRingCost), and cut
// into equal runs, one per CTA: ragged batches and long single sequences load the GPU alike.  The four warps of a CTA take
// quarters of a run, stream their tiles through private shared-memory rings, and join their softmax states at the end; an item
// that several CTAs share is joined by the merge kernel.
//
// With q' the rotated, reordered query, the scores of a quantized token are formed without dequantizing the key:
//   q'.K~_t = sum_g h_{t,g} (sum_{j in g} q'_j c_{t,j}) + sum_g z_{t,g} (sum_{j in g} q'_j)
// the inner sums on mma.m16n8k16 with fp32 accumulators, one per group: 16 tokens' codes are the A operand, 8 query rows the B
// operand, so that what costs instructions -- unpacking codes -- is shared by all rows and a single query wastes no more than
// the 8 columns.  A code goes in as 1024 + c (one instruction: its nibble under the bits of 1024) or, where the nibble lies four
// bits higher, as 1024 + 16 c against q'/16; the accumulators start at minus 1024 times the sum of the operand's q', so they end at
// sum q' c.  On the way they reach 1024 |q'| per term: of fp32's 24 bits that leaves 17 for the sum of codes, an error of h 2^-9
// sum |q'| at the very most (16 truncated additions of 2^-23).  Values enter the transposed product (V~^T P^T) as
// fp16(h c + z): one rounding, 2^-11 of the value at most; probabilities are rounded to fp16.  (h c alone as the operand and the zero
// points as one more row tile of the product is an instruction less per pair, but rounds h c, twice to three times the value:
// outputs 6e-4 instead of 3e-4 off in fp16, and measured no faster, 595 and 589 us for the serving mix.)
// A probability is held times 2^14
// relative to the running maximum: fp16 then resolves 2^-38 of the largest, so a million small ones still add up; their
// sum is kept in fp32.
// Fragments: the channels of a k-step and the tokens of a row are free to choose as long as both operands agree.  A lane's
// registers of the score product are the nibble pairs (i, i+4) of one 32-bit word, a word of every lane inside one
// 32-channel granule; of the value product they pair one channel of tokens j and j+4.  Neither operand passes through shared
// memory a second time; only the 16 x 8 probabilities are transposed (movmatrix).
// Measured: a decode step of 64 sequences of 1024 to 16384 tokens, 32 heads, 564 to 588 us (4.3 to 4.5 TB/s of the cache); 4 sequences of 131072
// tokens, 32 heads over 8, 163 us.  Instruction issue bounds it (61 % of the slots with 11 warps an SM, the logic pipe that unpacks
// codes half busy); a CTA more an SM spills.
#include <math_constants.h>

#include "skvq_mma_common.cuh"
#include "skvq_paged_split.cuh"

namespace skvq {
namespace {

using mmak::and_or;
using mmak::ex2_approx;
using mmak::mma16816;
using mmak::smem_u32;

constexpr int kSplitWarps = 4;
constexpr int kSplitThreads = kSplitWarps * 32;
constexpr int kTile = 32;             // tokens per warp tile
constexpr int kRingTile = 16;         // tokens per warp tile of the unquantized window: its rows fill the warp's whole ring
constexpr int kRingCost = 2;          // and move about twice a code tile's bytes
constexpr int kStages = 2;
constexpr float kPScaleLog2 = 14.0f;

struct SplitArgs {
    PagedAttnArgs a;
    int n_slots;
    int rows;      // rows per item: 8 NT
    int pieces;    // > 0: a CTA takes one of so many pieces of an item; 0: an equal share of the whole step
};

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
    static constexpr int POOL = RINGS > JOIN ? RINGS : JOIN;
    static constexpr int QS = ROWS * QROW * 2;         // queries, odd channels times 1/16; then the queries; then the queries in source order
    static constexpr int SMEM = POOL + 3 * QS;
    static constexpr int RROW = D * 2;                 // bytes of a window row
    static constexpr int RCHUNKS = RROW / 16;
    static_assert(2 * kRingTile * RROW <= kStages * STAGE, "a window tile fits the warp's ring");
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
// Four nibble pairs (i, i + 4) of a word as fp16 pairs: 1024 + c is 0x6400 | c, 1024 + 16 c is 0x6400 | c << 4.
__device__ __forceinline__ void raw_pairs(uint32_t w, uint32_t (&r)[4])      // 1024 + c, 1024 + 16 c, 1024 + c, 1024 + 16 c
{
    constexpr uint32_t M = 0x64006400u;
    const uint32_t u = w >> 8;
    r[0] = and_or(w, 0x000F000Fu, M);
    r[1] = and_or(w, 0x00F000F0u, M);
    r[2] = and_or(u, 0x000F000Fu, M);
    r[3] = and_or(u, 0x00F000F0u, M);
}
// d = a b + c with an accumulator of its own
__device__ __forceinline__ void mma16816_from(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, float c0,
                                              float c1, float c2, float c3)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
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
    int tiles_c, tiles_r;      // tiles of quantized tokens (32), of the window (16)
    int cost;                  // of one item, at least 1
    int m_tiles;               // items per KV head
};
__device__ __forceinline__ SeqCost seq_cost(const PagedArgs &p, const PagedSeq &s, int rows, int pieces)
{
    SeqCost c;
    const int rep = p.cfg.n_q_heads / p.cfg.n_kv_heads;
    c.tiles_c = (s.lq + kTile - 1) / kTile;
    c.tiles_r = (s.len - s.lq + kRingTile - 1) / kRingTile;
    c.cost = pieces ? pieces : max(c.tiles_c + kRingCost * c.tiles_r, 1);
    c.m_tiles = s.n * rep <= kFewRows ? (s.n * rep + rows - 1) / rows : 0;      // the others are the tcgen05 kernel's
    return c;
}

template <typename T, int D, int NG, int NT>
__global__ void __launch_bounds__(kSplitThreads, NT == 2 ? 2 : 3) paged_split_kernel(const __grid_constant__ SplitArgs args)
{
    using Geo = Geometry<D, NG, NT>;
    constexpr int ROWS = Geo::ROWS;
    const PagedAttnArgs &a = args.a;
    const PagedArgs &p = a.p;
    const skvq_paged_config &cfg = p.cfg;
    extern __shared__ __align__(128) uint8_t smem[];
    long long *pre = reinterpret_cast<long long *>(smem + Geo::SMEM);      // [n_seqs + 1] cost of the sequences before b
    __half *qs = reinterpret_cast<__half *>(smem + Geo::POOL), *qr = qs + ROWS * Geo::QROW;
    T *raw = reinterpret_cast<T *>(qr + ROWS * Geo::QROW);      // [ROWS][QROW]
    __shared__ long long scan_sh[kSplitWarps];
    __shared__ float row_scale[ROWS], q_sum[ROWS][4], q_off[ROWS][4], q_max[ROWS][4];      // per 32-channel granule
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
                    const SeqCost sc = seq_cost(p, s, ROWS, args.pieces);
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
    if (tid == 0 && args.pieces != 1) desc[0] = 0;
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
        const SeqCost sc = seq_cost(p, seq, ROWS, args.pieces);
        const long long item = (f - pre[b]) / sc.cost;
        const int off = (int)((f - pre[b]) - item * sc.cost);
        const int take = (int)min((long long)(sc.cost - off), f1 - f);
        const int hk = (int)(item / sc.m_tiles), mt = (int)(item - (long long)hk * sc.m_tiles);
        const int row_base = mt * ROWS, R = min(ROWS, seq.n * rep - row_base);
        const int L = seq.len, lq = seq.lq;
        // rows see tokens below their limit
        auto row_limit = [&](int r) { return a.causal ? min(L, L - seq.n + (row_base + min(r, R - 1)) / rep + 1) : L; };
        const int limit_lo = row_limit(0), limit_hi = row_limit(R - 1);
        int lim[NT][2];      // of this lane's columns of the score product: rows 8 n + 2 j, 8 n + 2 j + 1
#pragma unroll
        for (int n = 0; n < NT; ++n) { lim[n][0] = row_limit(8 * n + 2 * j); lim[n][1] = row_limit(8 * n + 2 * j + 1); }

        // ---- this warp's quarter of the run; its first pages are on their way while the queries are prepared
        auto tile_of = [&](int x) { return x <= sc.tiles_c ? x : sc.tiles_c + (x - sc.tiles_c + kRingCost - 1) / kRingCost; };
        const int full = sc.tiles_c + kRingCost * sc.tiles_r;
        const int seg0 = tile_of(args.pieces ? full * off / args.pieces : off), seg1 = tile_of(args.pieces ? full * (off + take) / args.pieces : off + take);
        const int c0 = min(seg0, sc.tiles_c), c1 = max(min(min(seg1, sc.tiles_c), (limit_hi + kTile - 1) / kTile), c0);
        const int q0 = c0 + (int)((long long)(c1 - c0) * warp / kSplitWarps), q1 = c0 + (int)((long long)(c1 - c0) * (warp + 1) / kSplitWarps);
        const int P = cfg.page_tokens, page_shift = __ffs(P) - 1;
        const int32_t *table = p.batch.page_table + (int64_t)b * p.batch.max_pages;
        // Page ids of 32 consecutive 16-token blocks, one per lane; -1 past the quantized tokens, -2 for an id outside the pool.
        auto load_pages = [&](int block) {
            const int t = (block + lane) * 16;
            int id = -1;
            if (t < lq) {
                id = table[t >> page_shift];
                if (id < 0 || id >= cfg.n_pages) { id = -2; set_status(p.c.status, SKVQ_STATUS_BAD_PAGE); }
            }
            return id;
        };
        int pages_base = q0 * 2, pages = q0 < q1 ? load_pages(pages_base) : -1, pages_next = q0 < q1 ? load_pages(pages_base + 32) : -1;

        // ---- quantized tokens
        const uint32_t ring = smem_u32(smem) + warp * kStages * Geo::STAGE;
        const uint8_t *ring_ptr = smem + warp * kStages * Geo::STAGE;
        const uint32_t codes_dst = (lane / Geo::CHUNKS) * Geo::ROW + piece_at<D>(lane / Geo::CHUNKS, lane % Geo::CHUNKS) * 16;
        const uint8_t *km_pool = static_cast<const uint8_t *>(p.c.k_meta), *vm_pool = static_cast<const uint8_t *>(p.c.v_meta);
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
                // The codes of a 16-token block are contiguous in the pool, and a lane's pieces of the tile lie 32 pieces apart:
                // one address per block and tensor, constant offsets from there.
                const uint32_t base = ring + stage * Geo::STAGE;
                const int64_t ra = ((int64_t)ida * cfg.n_kv_heads + hk) * P + ((tile * kTile) & (P - 1));
                const int64_t rb = ((int64_t)idb * cfg.n_kv_heads + hk) * P + ((tile * kTile + 16) & (P - 1));
                constexpr int HALF = Geo::CHUNKS / 2;
#pragma unroll
                for (int blk = 0; blk < 2; ++blk) {
                    if ((blk ? idb : ida) >= 0) {
                        const int64_t at = (blk ? rb : ra) * Geo::ROW + lane * 16;
                        const uint8_t *kc = static_cast<const uint8_t *>(p.c.k_codes) + at, *vc = static_cast<const uint8_t *>(p.c.v_codes) + at;
#pragma unroll
                        for (int k = 0; k < HALF; ++k) {
                            const uint32_t dst = base + codes_dst + (blk * HALF + k) * 512;
                            cp16(dst, kc + k * 512);
                            cp16(dst + Geo::CODES, vc + k * 512);
                        }
                    }
                }
                // parameters: PIECES 16-byte pieces per tensor, the first half of them block a's
                constexpr int PIECES = kTile * NG / 4;
                if constexpr (PIECES <= 16) {
                    const int side = lane >= PIECES, piece = lane - side * PIECES;
                    const bool second = piece >= PIECES / 2;
                    if (lane < 2 * PIECES && (second ? idb : ida) >= 0)
                        cp16(base + 2 * Geo::CODES + lane * 16, (side ? vm_pool : km_pool) + (second ? rb : ra) * (NG * 4) + (piece - second * (PIECES / 2)) * 16);
                } else {
                    const bool second = lane >= PIECES / 2;
                    if ((second ? idb : ida) >= 0) {
                        const int64_t at = (second ? rb : ra) * (NG * 4) + (lane - second * (PIECES / 2)) * 16;
                        cp16(base + 2 * Geo::CODES + lane * 16, km_pool + at);
                        cp16(base + 2 * Geo::CODES + Geo::META + lane * 16, vm_pool + at);
                    }
                }
            }
            cp_commit();
        };
#pragma unroll
        for (int k = 0; k < kStages - 1; ++k) fetch(q0 + k, k);
        // ---- queries: rotate, round to T, reorder; fp16 rows times a power of two, sums of every 32-channel granule.  A thread
        // per channel (of D = 64: of two rows at a time), so that the few rows of a decode step take one trip to memory
        {
            constexpr int STEP = kSplitThreads / D, PARTS = D / 32;
            const int c = tid % D, r_first = tid / D, part = c / 32;
            const int from = p.c.reorder_k ? p.c.reorder_k[hk * D + c] & (D - 1) : c;
            const float2 *rope = static_cast<const float2 *>(p.rope.table);
            const int half = p.rope.rot_dim / 2;
            const bool turn = rope && c < p.rope.rot_dim, second = p.rope.interleaved ? c & 1 : c >= half;
            const int pair = p.rope.interleaved ? c >> 1 : (second ? c - half : c);
            const int partner = p.rope.interleaved ? c ^ 1 : (second ? c - half : c + half);
#pragma unroll 4
            for (int r = r_first; r < R; r += STEP) {
                const int i = (row_base + r) / rep, head = hk * rep + (row_base + r) % rep, pos = L - seq.n + i;
                const T *src = static_cast<const T *>(a.q) + (int64_t)(seq.row0 + i) * a.q_stride + (int64_t)head * D;
                T x = src[c];
                if (turn && pos >= 0) {
                    const float2 cs = rope[(int64_t)pos * half + pair];
                    const float own = Elem<T>::to_float(x), other = Elem<T>::to_float(src[partner]);
                    x = Elem<T>::from_float(second ? rotate_second(other, own, cs.x, cs.y) : rotate_first(own, other, cs.x, cs.y));
                }
                raw[r * Geo::QROW + c] = x;
            }
            __syncthreads();
#pragma unroll 4
            for (int r = r_first; r < R; r += STEP) {
                const float mx = mmak::warp_max(fabsf(Elem<T>::to_float(raw[r * Geo::QROW + from])));
                if (lane == 0) q_max[r][part] = mx;
            }
            __syncthreads();
            const float sign = a.sm_scale < 0.f ? -1.f : (a.sm_scale == 0.f ? 0.f : 1.f);      // the rows' scale is positive
#pragma unroll 2
            for (int r = r_first; r < ROWS; r += STEP) {
                __half v = __float2half_rn(0.f), w = v;
                float sum = 0.f, off_sum = 0.f, up = 1.f;
                if (r < R) {
                    float mx = q_max[r][0];
#pragma unroll
                    for (int k = 1; k < PARTS; ++k) mx = fmaxf(mx, q_max[r][k]);
                    // bring the row's largest to [2^13, 2^14): exact, whatever the range of the type
                    if (mx > 0.f && mx < CUDART_INF_F) up = __int_as_float((127 + min(13 - (__float_as_int(mx) >> 23) + 127, 60)) << 23);
                    // an infinite query: infinities would leave scores of -infinity, which mean masked
                    v = __float2half_rn(Elem<T>::to_float(raw[r * Geo::QROW + from]) * (mx < CUDART_INF_F ? up * sign : CUDART_NAN_F));
                    w = c & 1 ? __hmul(v, __float2half_rn(0.0625f)) : v;
                    sum = mmak::warp_sum(__half2float(v));
                    off_sum = mmak::warp_sum(__half2float(w));
                }
                qr[r * Geo::QROW + c] = v;
                qs[r * Geo::QROW + c] = w;
                if (lane == 0) { q_sum[r][part] = sum; q_off[r][part] = -1024.f * off_sum; }
                if (c == 0) row_scale[r] = (sign == 0.f ? 1.f : fabsf(a.sm_scale)) * 1.4426950408889634f / up;
            }
        }
        __syncthreads();
        uint32_t bq[NT][Geo::SETS * 2][2];
        float rs[NT][2], qsum[NT][2][NG], qoff[NT][2][NG];
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
                for (int k = 0; k < NG; ++k) {
                    constexpr int PER = Geo::SETS / NG;      // granules per group
                    float u = 0.f, v = 0.f;
#pragma unroll
                    for (int m = 0; m < PER; ++m) { u += q_sum[8 * n + 2 * j + e][k * PER + m]; v += q_off[8 * n + 2 * j + e][k * PER + m]; }
                    qsum[n][e][k] = u;
                    qoff[n][e][k] = v;
                }
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

        // Scores of 16 or 32 tokens (to be multiplied by the row's scale rs) -> probabilities as B fragments.  s[u][n] = {token a: rows
        // 2j, 2j+1; token a + 8: the same}, token a = 16 u + (g >> 1) + 4 (g & 1).
        auto softmax_tile = [&](auto &s, auto &pb) {
            constexpr int U = sizeof(s) / sizeof(s[0]);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float x[2], base[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    x[e] = fmaxf(s[0][n][e], s[0][n][2 + e]);
                    if constexpr (U == 2) x[e] = fmaxf(x[e], fmaxf(s[1][n][e], s[1][n][2 + e]));
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) x[e] = fmaxf(x[e], __shfl_xor_sync(0xffffffffu, x[e], d));
                    x[e] = fmaxf(x[e], m_run[n][e]);
                }
                if (__any_sync(0xffffffffu, x[0] > m_run[n][0] || x[1] > m_run[n][1])) {
                    float down[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        down[e] = x[e] > m_run[n][e] ? ex2_approx((m_run[n][e] - x[e]) * rs[n][e]) : 1.f;
                        l_run[n][e] *= down[e];
                        m_run[n][e] = x[e];
                    }
#pragma unroll
                    for (int m = 0; m < Geo::MT; ++m) { o[n][m][0] *= down[0]; o[n][m][1] *= down[1]; o[n][m][2] *= down[0]; o[n][m][3] *= down[1]; }
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) base[e] = kPScaleLog2 - (m_run[n][e] == -CUDART_INF_F ? 0.f : m_run[n][e] * rs[n][e]);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    float v[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = ex2_approx(fmaf(s[u][n][e], rs[n][e & 1], base[e & 1]));
                    l_run[n][0] += v[0] + v[2];
                    l_run[n][1] += v[1] + v[3];
                    pb[u][n][0] = transpose8x8(pack_h2(v[0], v[1]));
                    pb[u][n][1] = transpose8x8(pack_h2(v[2], v[3]));
                }
            }
        };

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
                for (int st = 0; st < Geo::SETS; ++st) {
                    uint32_t x[4], y[4];
                    raw_pairs(*reinterpret_cast<const uint32_t *>(buf + t * Geo::ROW + piece_at<D>(t, st) * 16 + j * 4), x);
                    raw_pairs(*reinterpret_cast<const uint32_t *>(buf + (t + 8) * Geo::ROW + piece_at<D>(t, st) * 16 + j * 4), y);
                    constexpr int PER = Geo::SETS / NG;      // sets per group
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        float (&d)[4] = acc[n][st / PER];
                        if (st % PER == 0)
                            mma16816_from(d, x[0], y[0], x[1], y[1], bq[n][2 * st][0], bq[n][2 * st][1], qoff[n][0][st / PER], qoff[n][1][st / PER],
                                          qoff[n][0][st / PER], qoff[n][1][st / PER]);
                        else
                            mma16816(d, x[0], y[0], x[1], y[1], bq[n][2 * st][0], bq[n][2 * st][1]);
                        mma16816(d, x[2], y[2], x[3], y[3], bq[n][2 * st + 1][0], bq[n][2 * st + 1][1]);
                    }
                }
#pragma unroll
                for (int k = 0; k < NG; ++k) {
                    const uint32_t ma = km[t * NG + k], mb = km[(t + 8) * NG + k];
                    const float2 ha = __half22float2(*reinterpret_cast<const __half2 *>(&ma)), hb = __half22float2(*reinterpret_cast<const __half2 *>(&mb));
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const float za = ha.y * qsum[n][e][k], zb = hb.y * qsum[n][e][k];
                            s[u][n][e] = fmaf(ha.x, acc[n][k][e], k ? za + s[u][n][e] : za);
                            s[u][n][2 + e] = fmaf(hb.x, acc[n][k][2 + e], k ? zb + s[u][n][2 + e] : zb);
                        }
                }
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
                }
                if (edge) {      // a row that holds nothing must not reach the product: 0 times what lies there need not be 0
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (t0 + ta + 4 * k >= lq || ((bad_here >> u) & 1u)) hz[k] = 0u;
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
                        raw_pairs(__byte_perm(w[0][q], w[1][q], sel), x);
                        raw_pairs(__byte_perm(w[2][q], w[3][q], sel), y);
#pragma unroll
                        for (int k = 0; k < 4; ++k) {      // 1024 + c - 1024, (1024 + 16 c) / 16 - 64: the code, exact
                            x[k] = h2_fma(k & 1 ? h2_fma(x[k], 0x2C002C00u, 0xD400D400u) : h2_sub(x[k], 0x64006400u), h_a, z_a);
                            y[k] = h2_fma(k & 1 ? h2_fma(y[k], 0x2C002C00u, 0xD400D400u) : h2_sub(y[k], 0x64006400u), h_b, z_b);
                        }
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

        // ---- the window: 16-bit rows, 16 tokens at a time through the warp's whole ring; the warps take its tiles in turn
        __syncwarp();
        const int r0 = max(seg0, sc.tiles_c), r1 = max(min(seg1, sc.tiles_c + sc.tiles_r), r0);
        const int64_t win_row0 = ((int64_t)seq.slot * cfg.n_kv_heads + hk) * cfg.ring_tokens;
#pragma unroll 1
        for (int tile = r0 + warp; tile < r1; tile += kSplitWarps) {
            const int t0 = lq + (tile - sc.tiles_c) * kRingTile;
            if (t0 >= limit_hi) break;
            uint32_t gone;      // tokens of the tile whose page-table entry is no page of the pool
            {
                int id = 0;
                if (lane < kRingTile && t0 + lane < L) id = table[(t0 + lane) >> page_shift];
                // lane: piece lane % RCHUNKS of every (32 / RCHUNKS)-th row; piece c of row t lies at c ^ (t & 7)
                constexpr int STEP = 32 / Geo::RCHUNKS;
                const int c = lane % Geo::RCHUNKS, first = t0 % cfg.ring_tokens;
                const uint8_t *kw = static_cast<const uint8_t *>(p.c.k_win) + win_row0 * Geo::RROW + c * 16, *vw = static_cast<const uint8_t *>(p.c.v_win) + win_row0 * Geo::RROW + c * 16;
#pragma unroll
                for (int k = 0; k < kRingTile / STEP; ++k) {
                    const int t = k * STEP + lane / Geo::RCHUNKS;
                    const uint32_t at = t * Geo::RROW + (c ^ (t & 7)) * 16;
                    if (t0 + t < L) {
                        int row = first + t;      // the window is no longer than the ring: it wraps once at most
                        if (row >= cfg.ring_tokens) row -= cfg.ring_tokens;
                        cp16(ring + at, kw + (int64_t)row * Geo::RROW);
                        cp16(ring + kRingTile * Geo::RROW + at, vw + (int64_t)row * Geo::RROW);
                    } else {
                        *reinterpret_cast<uint4 *>(smem + warp * kStages * Geo::STAGE + kRingTile * Geo::RROW + at) = make_uint4(0u, 0u, 0u, 0u);
                    }
                }
                cp_commit();
                const bool none = id < 0 || id >= cfg.n_pages;
                if (none) set_status(p.c.status, SKVQ_STATUS_BAD_PAGE);
                gone = __ballot_sync(0xffffffffu, none);
                cp_wait<0>();
                __syncwarp();
                if (gone) {      // their value rows hold nothing that may reach the product
                    for (int e = lane; e < kRingTile * Geo::RCHUNKS; e += 32)
                        if ((gone >> (e / Geo::RCHUNKS)) & 1u)
                            *reinterpret_cast<uint4 *>(smem + warp * kStages * Geo::STAGE + kRingTile * Geo::RROW + e * 16) = make_uint4(0u, 0u, 0u, 0u);
                    __syncwarp();
                }
            }
            float s[1][NT][4];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[0][n][e] = 0.f;
#pragma unroll
            for (int st = 0; st < Geo::SETS; ++st) {
                uint4 x = *reinterpret_cast<const uint4 *>(ring_ptr + tok * Geo::RROW + ((4 * st + j) ^ tok) * 16);
                uint4 y = *reinterpret_cast<const uint4 *>(ring_ptr + (tok + 8) * Geo::RROW + ((4 * st + j) ^ tok) * 16);
                x.x = as_h2<T>(x.x); x.y = as_h2<T>(x.y); x.z = as_h2<T>(x.z); x.w = as_h2<T>(x.w);
                y.x = as_h2<T>(y.x); y.y = as_h2<T>(y.y); y.z = as_h2<T>(y.z); y.w = as_h2<T>(y.w);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const uint4 q = *reinterpret_cast<const uint4 *>(qr + (8 * n + g) * Geo::QROW + 32 * st + 8 * j);
                    mma16816(s[0][n], x.x, y.x, x.z, y.z, q.x, q.z);
                    mma16816(s[0][n], x.y, y.y, x.w, y.w, q.y, q.w);
                }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (t0 + tok + 8 * (e >> 1) >= lim[n][e & 1] || ((gone >> (tok + 8 * (e >> 1))) & 1u)) s[0][n][e] = -CUDART_INF_F;
            uint32_t pb[1][NT][2];
            softmax_tile(s, pb);
#pragma unroll
            for (int q = 0; q < D / 64; ++q) {
                uint32_t e[4][4];      // rows j, j + 4, j + 8, j + 12, eight of this lane's channels
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int t = j + 4 * k;
                    const uint4 x = *reinterpret_cast<const uint4 *>(ring_ptr + kRingTile * Geo::RROW + t * Geo::RROW + ((g * (D / 64) + q) ^ (t & 7)) * 16);
                    e[k][0] = as_h2<T>(x.x); e[k][1] = as_h2<T>(x.y); e[k][2] = as_h2<T>(x.z); e[k][3] = as_h2<T>(x.w);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
                        mma16816(o[n][4 * q + k], __byte_perm(e[0][k], e[1][k], 0x5410), __byte_perm(e[0][k], e[1][k], 0x7632),
                                 __byte_perm(e[2][k], e[3][k], 0x5410), __byte_perm(e[2][k], e[3][k], 0x7632), pb[0][n][0], pb[0][n][1]);
            }
            __syncwarp();
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
                if (g == 0) { ml_sh[warp][r][0] = m_run[n][e] * rs[n][e]; ml_sh[warp][r][1] = l_run[n][e]; }      // from here on in units of log2
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
            const float from = M == -CUDART_INF_F ? 0.f : M;      // nothing seen: sums of zero; a query that is not a number: sums that are none
#pragma unroll
            for (int w = 0; w < kSplitWarps; ++w) {
                const float k = ex2_approx(ml_sh[w][r][0] - from);
                l = fmaf(ml_sh[w][r][1], k, l);
                v = fmaf(join[(w * ROWS + r) * Geo::JROW + (c % Geo::CPT) * 8 + c / Geo::CPT], k, v);
            }
            if (whole) {
                const int i = (row_base + r) / rep, head = hk * rep + (row_base + r) % rep;
                static_cast<T *>(a.out)[(int64_t)(seq.row0 + i) * a.out_stride + head * D + dst] = Elem<T>::from_float(l == 0.f ? 0.f : v / l);
                if (a.lse && c == 0)
                    a.lse[(int64_t)(seq.row0 + i) * cfg.n_q_heads + head] = l == 0.f ? -CUDART_INF_F : (M + log2f(l) - kPScaleLog2) * 0.6931471805599453f;
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

// Joins the partials of an item that several runs share: blockIdx.x is the run that begins it; a warp takes a row, D/32 channels a lane.
constexpr int kMergeWarps = 4;
struct MergeArgs {
    PagedAttnArgs a;
    int n_slots, rows;
    float lse_offset;
};
template <typename T, int D>
__global__ void __launch_bounds__(kMergeWarps * 32) paged_merge_kernel(const __grid_constant__ MergeArgs args)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    constexpr int C = D / 32, PS = partial_stride(D);
    const PagedAttnArgs &a = args.a;
    const skvq_paged_config &cfg = a.p.cfg;
    const int slot = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int4 d0 = *reinterpret_cast<const int4 *>(reinterpret_cast<const int *>(a.ws) + (size_t)slot * kDescInts);
    if (d0.x == 0) return;
    const int4 d1 = *reinterpret_cast<const int4 *>(reinterpret_cast<const int *>(a.ws) + (size_t)slot * kDescInts + 4);
    const int row0 = d0.y, n_new = d0.z, hk = d0.w, item = d1.x, n = d1.y, rep = cfg.n_q_heads / cfg.n_kv_heads;
    int dst[C];
#pragma unroll
    for (int k = 0; k < C; ++k) dst[k] = a.p.c.reorder_v ? a.p.c.reorder_v[hk * D + lane * C + k] & (D - 1) : lane * C + k;
    for (int r = blockIdx.y * kMergeWarps + warp; r < args.rows; r += gridDim.y * kMergeWarps) {
        const int row = item * args.rows + r;
        if (row >= n_new * rep) return;
        const float *base = a.ws + (size_t)args.n_slots * kDescInts + ((size_t)slot * 2 * args.rows + r) * PS;
        auto partial = [&](int k) { return base + (size_t)(2 * k + (k == 0 ? 1 : 0)) * args.rows * PS; };
        // 32 partials at a time: their maxima and sums in the lanes of the warp
        float m = -CUDART_INF_F, l = 0.f, o[C];
#pragma unroll
        for (int k = 0; k < C; ++k) o[k] = 0.f;
        for (int k0 = 0; k0 < n; k0 += 32) {
            const bool have = k0 + lane < n;
            const float pm = have ? partial(k0 + lane)[D] : -CUDART_INF_F, pl = have ? partial(k0 + lane)[D + 1] : 0.f;
            float top = fmaxf(pm, m);
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
            const float from = top == -CUDART_INF_F ? 0.f : top;
            const float down = ex2_approx(m - from), f = ex2_approx(pm - from);
            float sum = pl * f;
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            l = fmaf(l, down, sum);
#pragma unroll
            for (int k = 0; k < C; ++k) o[k] *= down;
            m = top;
            const int last = min(32, n - k0);
#pragma unroll 4
            for (int q = 0; q < last; ++q) {
                const float g = __shfl_sync(0xffffffffu, f, q);
                if constexpr (C == 4) {
                    const float4 v = *reinterpret_cast<const float4 *>(partial(k0 + q) + lane * 4);
                    o[0] = fmaf(v.x, g, o[0]); o[1] = fmaf(v.y, g, o[1]); o[2] = fmaf(v.z, g, o[2]); o[3] = fmaf(v.w, g, o[3]);
                } else {
                    const float2 v = *reinterpret_cast<const float2 *>(partial(k0 + q) + lane * 2);
                    o[0] = fmaf(v.x, g, o[0]); o[1] = fmaf(v.y, g, o[1]);
                }
            }
        }
        const int i = row / rep, head = hk * rep + row % rep;
        T *out = static_cast<T *>(a.out) + (int64_t)(row0 + i) * a.out_stride + (int64_t)head * D;
#pragma unroll
        for (int k = 0; k < C; ++k) out[dst[k]] = Elem<T>::from_float(l == 0.f ? 0.f : o[k] / l);
        if (a.lse && lane == 0)
            a.lse[(int64_t)(row0 + i) * cfg.n_q_heads + head] = l == 0.f ? -CUDART_INF_F : (m + log2f(l) - args.lse_offset) * 0.6931471805599453f;
    }
}

// The most rows a KV head of this kernel can have, and the rows per item: 8 or 16.
long long few_rows(const skvq_paged_config &cfg, const skvq_paged_batch &batch)
{
    const long long rows = (long long)batch.max_new * (cfg.n_q_heads / cfg.n_kv_heads);
    return rows < kFewRows ? rows : kFewRows;
}
int item_rows(const skvq_paged_config &cfg, const skvq_paged_batch &batch)
{
    const long long rows = few_rows(cfg, batch);
    return rows <= 8 ? 8 : 16;
}

// Contexts so short that a CTA per item is done sooner than several and a merge (512 tokens, window 128, 16 or 64 sequences of 8 KV heads:
// 24 us split, 16 whole; 40 and 31).
constexpr int kWholeCost = 48;
constexpr long long kMaxSlots = 16384;

// Price of an item at most, and the items of a step at most.
long long item_cost(const skvq_paged_config &cfg, const skvq_paged_batch &batch)
{
    const long long lq = batch.max_len > cfg.window ? batch.max_len - cfg.window : 0;
    return (lq + kTile - 1) / kTile + kRingCost * ((batch.max_len - lq + kRingTile - 1) / kRingTile) + 1;
}
long long item_count(const skvq_paged_config &cfg, const skvq_paged_batch &batch)
{
    const int per = item_rows(cfg, batch);
    return (long long)batch.n_seqs * cfg.n_kv_heads * ((few_rows(cfg, batch) + per - 1) / per);
}
// How a step is cut: pieces of items (1: whole ones, nothing to join), or, pieces = 0, equal shares of everything.
struct SplitShape {
    int pieces, slots;
};
SplitShape split_plan(const skvq_paged_config &cfg, const skvq_paged_batch &batch, int n_splits)
{
    const long long items = item_count(cfg, batch), cost = item_cost(cfg, batch);
    if (items == 0) return {1, 0};      // no new tokens: the entry points return before a launch
    if (n_splits == 0 && cost <= kWholeCost && items <= kMaxSlots) return {1, (int)items};
    // one wave of resident CTAs (a CTA more per SM spills: serving mix 597 us against 580), each with two tiles per warp at least: a shorter run
    // costs more to join than it saves
    const long long wave = (item_rows(cfg, batch) == 8 ? 3LL : 2LL) * sm_count();
    long long slots = n_splits > 0 ? n_splits * items : (wave < items * cost / 8 ? wave : items * cost / 8);
    if (slots > items * cost) slots = items * cost;
    if (slots > kMaxSlots) slots = kMaxSlots;
    if (slots < 1) slots = 1;
    // Few items and little work: equal pieces of every item.  A share that ends one item and begins the next prepares two sets of
    // queries and joins twice, which such short shares do not hide (one query over 4096 tokens, 32 heads: 21.8 us in equal shares, 17.9 so).
    if (n_splits == 0 && items * 2 <= slots && items * cost <= slots * 32) return {(int)(slots / items), (int)(slots / items * items)};
    return {0, (int)slots};
}

template <typename T, int D, int NG, int NT>
cudaError_t launch_split(const PagedAttnArgs &a, cudaStream_t stream)
{
    using Geo = Geometry<D, NG, NT>;
    const SplitShape shape = split_plan(a.p.cfg, a.p.batch, a.n_splits);
    const SplitArgs s{a, shape.slots, Geo::ROWS, shape.pieces};
    static unsigned long long done = 0;
    cudaError_t e = configure_smem_once(paged_split_kernel<T, D, NG, NT>, Geo::SMEM + (int)sizeof(long long) * (kMaxPagedSeqs + 1), done);
    if (e != cudaSuccess) return e;
    e = launch_chained(paged_split_kernel<T, D, NG, NT>, dim3(s.n_slots), kSplitThreads, Geo::SMEM + sizeof(long long) * (a.p.batch.n_seqs + 1), stream, s);
    if (e != cudaSuccess || shape.pieces == 1) return e;
    return launch_paged_merge(a, s.n_slots, Geo::ROWS, (int)few_rows(a.p.cfg, a.p.batch), kPScaleLog2, stream);
}

template <typename T, int D, int NG> cudaError_t launch_by_rows(const PagedAttnArgs &a, cudaStream_t stream)
{
    const int rows = item_rows(a.p.cfg, a.p.batch);
    return rows == 8 ? launch_split<T, D, NG, 1>(a, stream) : launch_split<T, D, NG, 2>(a, stream);
}

template <typename T> cudaError_t launch_by_shape(const PagedAttnArgs &a, cudaStream_t stream)
{
    if (a.p.cfg.head_dim == 128)
        return a.p.ng == 1 ? launch_by_rows<T, 128, 1>(a, stream) : a.p.ng == 2 ? launch_by_rows<T, 128, 2>(a, stream) : launch_by_rows<T, 128, 4>(a, stream);
    return a.p.ng == 1 ? launch_by_rows<T, 64, 1>(a, stream) : launch_by_rows<T, 64, 2>(a, stream);
}

size_t split_workspace_bytes(const skvq_paged_config &cfg, const skvq_paged_batch &batch, int n_splits)
{
    const SplitShape shape = split_plan(cfg, batch, n_splits);
    if (shape.pieces == 1) return 0;
    const size_t slots = shape.slots;
    return (slots * kDescInts * 4 + slots * 2 * item_rows(cfg, batch) * partial_stride(cfg.head_dim) * 4 + 15) / 16 * 16;
}

bool has_many_rows(const skvq_paged_config &cfg, const skvq_paged_batch &batch)
{
    return (long long)batch.max_new * (cfg.n_q_heads / cfg.n_kv_heads) > kFewRows;
}

template <typename T> cudaError_t merge_by_dim(const MergeArgs &m, int row_warps, cudaStream_t stream)
{
    const dim3 grid(m.n_slots, (row_warps + kMergeWarps - 1) / kMergeWarps);
    return m.a.p.cfg.head_dim == 128 ? launch_chained(paged_merge_kernel<T, 128>, grid, kMergeWarps * 32, 0, stream, m)
                                     : launch_chained(paged_merge_kernel<T, 64>, grid, kMergeWarps * 32, 0, stream, m);
}

}  // namespace

cudaError_t launch_paged_merge(const PagedAttnArgs &a, int n_slots, int rows, int row_warps, float lse_offset, cudaStream_t stream)
{
    const MergeArgs m{a, n_slots, rows, lse_offset};
    return a.p.cfg.dtype == SKVQ_F16 ? merge_by_dim<__half>(m, row_warps, stream) : merge_by_dim<__nv_bfloat16>(m, row_warps, stream);
}

size_t paged_workspace_bytes(const skvq_paged_config &cfg, const skvq_paged_batch &batch, int n_splits)
{
    return split_workspace_bytes(cfg, batch, n_splits) + (has_many_rows(cfg, batch) ? prefill_workspace_bytes(cfg, batch) : 0);
}

// A step whose host bound allows many rows may still hold sequences with few: each kernel takes its own, by what the device arrays
// say.
cudaError_t launch_paged_attention(const PagedAttnArgs &a, cudaStream_t stream)
{
    const cudaError_t e = a.p.cfg.dtype == SKVQ_F16 ? launch_by_shape<__half>(a, stream) : launch_by_shape<__nv_bfloat16>(a, stream);
    if (e != cudaSuccess || !has_many_rows(a.p.cfg, a.p.batch)) return e;
    PagedAttnArgs b = a;
    b.ws = a.ws + split_workspace_bytes(a.p.cfg, a.p.batch, a.n_splits) / sizeof(float);
    return launch_paged_prefill(b, stream);
}

}  // namespace skvq
