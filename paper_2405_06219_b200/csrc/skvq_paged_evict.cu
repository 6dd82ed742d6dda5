// skvq_paged_evict: every KV head of a sequence keeps its oldest and newest tokens and the most looked-at ones between them; their
// rows close up, in order.
//
// Two kernels.  The first finds, per (sequence, KV head), the threshold of the middle's weights by a radix selection (three digits
// of 11, 11 and 10 bits of the order-preserving integer of a float) and writes the kept tokens' numbers in order: those above the
// threshold, and of those at it the lowest-numbered.  A CTA, or a cluster of up to eight that add their histograms up over
// distributed shared memory, holds the weights in registers: they are read once (of 32 weights a thread, in 64 registers, 92 bytes spill).  The second kernel moves rows: row i of the shortened
// sequence comes from token kept[i] >= i.  A CTA, or a cluster, has the keys or values of a pair; the rows of one pass are read before any of
// them is written, passes go upwards, and the sources of later passes lie behind what earlier passes write: so a sequence may be
// shortened inside its own pages.
// Measured (selection + rows): a 32k prompt of 8 KV heads to 2048 tokens 17 + 7 us; 64 sequences of 1024 to 16384 tokens, 32 heads, to 2048
// 168 + 377 us; 4 sequences of 131k tokens, 8 KV heads, to 65521 52 + 157 us, 69 % of the copy rate.  The rows' kernel is bound by scattered
// 64-byte reads and their latency; 256 threads with two rows in flight and six CTAs an SM took 537 and 221 us in all, against 554 and 213.
#include <cooperative_groups.h>

#include "skvq_mma_common.cuh"
#include "skvq_paged.cuh"
#include "skvq_paged_split.cuh"

namespace skvq {
namespace {

namespace cg = cooperative_groups;
using mmak::smem_u32;

constexpr int kSelectThreads = 512;
constexpr int kMaxCluster = 8;      // the portable size
constexpr int kMoveThreads = 256;
constexpr int kUnroll = 4;
constexpr int kBins = 2048;

// What the second kernel needs of the first: the caller may have lens_out = lens, ring_from_out = ring_from.
struct alignas(16) EvictSeq {
    int len, left, ring_from, ok;      // tokens before, after; first token of the ring before (of a skipped sequence as given)
};

__device__ __forceinline__ bool evict_sequence(const PagedEvictArgs &a, int b, EvictSeq &s)
{
    const skvq_paged_batch &p = a.p.batch;
    s.len = p.lens[b];
    s.ring_from = p.ring_from ? p.ring_from[b] : 0;
    const int from = p.slots ? p.slots[b] : b, to = a.e.slots_out ? a.e.slots_out[b] : from;
    const bool ok = s.len >= 0 && s.len <= p.max_len && from >= 0 && from < a.p.cfg.n_slots && to >= 0 && to < a.p.cfg.n_slots;
    if (ok) s.ring_from = max(min(s.ring_from, s.len), 0);
    s.left = min(s.len, a.e.keep);
    s.ok = ok;
    return ok;
}

// Larger weights have larger keys; -0 and +0 share one, and what is not a number has the smallest.
__device__ __forceinline__ uint32_t weight_key(float w)
{
    const uint32_t u = __float_as_uint(w + 0.f);
    const uint32_t key = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
    return w == w ? key : 0u;
}

// An increment of a word in shared memory.  `one` is 1, which the compiler must not know: increments by a constant become a loop over the
// distinct addresses of the warp (32 pairs of 131k weights: 121 us so).
__device__ __forceinline__ void count(uint32_t word, uint32_t one) { asm volatile("red.shared.add.u32 [%0], %1;" ::"r"(word), "r"(one) : "memory"); }

struct SelectArgs {
    PagedEvictArgs a;
    int ctas;      // of a cluster: they share the middle of a (sequence, KV head)
};

// ITEMS > 0: a CTA's share of the middle has at most kSelectThreads * ITEMS weights, which stay in registers; ITEMS = 0: any length, the weights
// are read again for every digit and for the result.
template <int ITEMS>
__global__ void __launch_bounds__(kSelectThreads, 2) evict_select_kernel(const __grid_constant__ SelectArgs args)
{
    constexpr int WARPS = kSelectThreads / 32, KEYS = ITEMS ? ITEMS : 1;
    __shared__ __align__(16) int hist[3 * kBins];      // of the three digits; read four bins at a time
    __shared__ int warp_sum[WARPS], found[2], totals[2];
    __shared__ int2 warp_count[WARPS];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const PagedEvictArgs &a = args.a;
    cg::cluster_group cluster = cg::this_cluster();
    const int H = a.p.cfg.n_kv_heads, C = args.ctas, pair = blockIdx.x / C, rank = blockIdx.x % C, b = pair / H, h = pair % H;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, all = rank * kSelectThreads + tid, step = C * kSelectThreads;
    EvictSeq s;
    const bool ok = evict_sequence(a, b, s);
    if (h == 0 && all == 0) {
        static_cast<EvictSeq *>(a.e.workspace)[b] = s;
        if (!ok) set_status(a.p.c.status, SKVQ_STATUS_BAD_BATCH);
    }
    int32_t *kept = a.e.kept + ((int64_t)b * H + h) * a.e.keep;
    if (!ok) s.left = 0;
    for (int64_t i = (int64_t)s.left + all; i < a.e.keep; i += step) kept[i] = -1;
    if (s.left == s.len || !ok) {
        for (int i = all; i < s.left; i += step) kept[i] = i;
        return;
    }
    const int first = a.e.first, end = s.len - a.e.recent, want = a.e.keep - first - a.e.recent;
    for (int i = all; i < first; i += step) kept[i] = i;
    for (int i = all; i < a.e.recent; i += step) kept[first + want + i] = end + i;
    if (want == 0) return;
    const float *w = a.e.weights + ((int64_t)(a.p.batch.slots ? a.p.batch.slots[b] : b) * H + h) * a.e.capacity;
    // this CTA's share: tokens [lo, hi), a warp's run of it is contiguous
    const int span = (end - first + C - 1) / C, lo = min(first + rank * span, end), hi = min(lo + span, end);
    const int items = (span + kSelectThreads - 1) / kSelectThreads, warp_span = items * 32, warp_lo = min(lo + warp * warp_span, hi);
    uint32_t keys[KEYS];
    if constexpr (ITEMS > 0) {
        float x[KEYS];      // all loads first: with the conversions between them they went one after the other, 8 us for 32
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            const int t = warp_lo + k * 32 + lane;
            x[k] = 0.f;
            if (k < items && t < hi) x[k] = w[t];
        }
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) keys[k] = weight_key(x[k]);
    }
    // calls f(token, key, is there one) for every place of the warp's run, the lanes side by side
    auto each = [&](auto &&f) {
        if constexpr (ITEMS > 0) {
#pragma unroll
            for (int k = 0; k < ITEMS; ++k) {
                const int t = warp_lo + k * 32 + lane;
                if (k < items) f(t, keys[k], t < hi);
            }
        } else {
            for (int t = warp_lo + lane; t - lane < min(warp_lo + warp_span, hi); t += 32) {
                const bool have = t < min(warp_lo + warp_span, hi);
                f(t, have ? weight_key(w[t]) : 0u, have);
            }
        }
    };
    // ---- the threshold: the want-th largest key
    for (int i = tid; i < 3 * kBins; i += kSelectThreads) hist[i] = 0;
    __syncthreads();
    uint32_t prefix = 0u, one;
    asm volatile("mov.u32 %0, 1;" : "=r"(one));
    int left = want;      // still to be found among the keys that begin with `prefix`
#pragma unroll 1
    for (int round = 0; round < 3; ++round) {
        const int shift = round == 0 ? 21 : (round == 1 ? 10 : 0), bits = round == 2 ? 10 : 11;
        int *bins = hist + round * kBins;
        each([&](int, uint32_t key, bool have) {
            if (have && (round == 0 || (key >> (shift + bits)) == prefix)) count(smem_u32(bins + ((key >> shift) & ((1u << bits) - 1u))), one);
        });
        if (C > 1) cluster.sync();
        else __syncthreads();
        // bins from the top: thread i owns the four below kBins - 4 i
        constexpr int OWN = kBins / kSelectThreads;
        int n[OWN], incl = 0;
#pragma unroll
        for (int k = 0; k < OWN; ++k) n[k] = 0;
        if (C > 1) {
#pragma unroll
            for (int r = 0; r < kMaxCluster; ++r) {      // all on their way together
                if (r >= C) continue;
                const int4 v = *reinterpret_cast<const int4 *>(cluster.map_shared_rank(bins, (rank + r) & (C - 1)) + kBins - OWN * (tid + 1));      // each begins with its own
                n[0] += v.w; n[1] += v.z; n[2] += v.y; n[3] += v.x;
            }
        } else {
            const int4 v = *reinterpret_cast<const int4 *>(bins + kBins - OWN * (tid + 1));
            n[0] = v.w; n[1] = v.z; n[2] = v.y; n[3] = v.x;
        }
        static_assert(OWN == 4, "a 16-byte read of four bins");
#pragma unroll
        for (int k = 0; k < OWN; ++k) incl += n[k];
        const int own = incl;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, incl, d);
            if (lane >= d) incl += v;
        }
        if (lane == 31) warp_sum[warp] = incl;
        __syncthreads();
        int before = incl - own;
#pragma unroll
        for (int k = 0; k < WARPS; ++k) before += k < warp ? warp_sum[k] : 0;
#pragma unroll
        for (int k = 0; k < OWN; ++k) {
            if (before < left && before + n[k] >= left) { found[0] = kBins - 1 - OWN * tid - k; found[1] = before; }
            before += n[k];
        }
        __syncthreads();
        prefix = prefix << bits | (uint32_t)found[0];
        left -= found[1];
    }
    // ---- the kept tokens in order: all above the threshold, the first `left` at it.  How many of each lie before this warp's?
    int above = 0, equal = 0;
    each([&](int, uint32_t key, bool have) {
        above += __popc(__ballot_sync(0xffffffffu, have && key > prefix));
        equal += __popc(__ballot_sync(0xffffffffu, have && key == prefix));
    });
    if (lane == 0) warp_count[warp] = make_int2(above, equal);
    __syncthreads();
    int g = 0, e = 0, all_g = 0, all_e = 0;
#pragma unroll
    for (int k = 0; k < WARPS; ++k) {
        const int2 v = warp_count[k];
        if (k < warp) { g += v.x; e += v.y; }
        all_g += v.x;
        all_e += v.y;
    }
    if (C > 1) {
        if (tid == 0) { totals[0] = all_g; totals[1] = all_e; }
        cluster.sync();
        for (int r = 0; r < rank; ++r) {
            const int *other = cluster.map_shared_rank(totals, r);
            g += other[0];
            e += other[1];
        }
    }
    const uint32_t below = (1u << lane) - 1u;
    each([&](int t, uint32_t key, bool have) {
        const bool gt = have && key > prefix, eq = have && key == prefix;
        const uint32_t gts = __ballot_sync(0xffffffffu, gt), eqs = __ballot_sync(0xffffffffu, eq);
        const int eb = e + __popc(eqs & below);
        if (gt || (eq && eb < left)) kept[first + g + __popc(gts & below) + min(eb, left)] = t;
        g += __popc(gts);
        e += __popc(eqs);
    });
    if (C > 1) cluster.sync();      // nobody leaves while another may still read its shared memory
}

struct MoveArgs {
    PagedEvictArgs a;
    int strip;      // bytes of a ring row that a CTA moves at a time
    int ctas;       // of a cluster: they share a unit
};

// Everybody in the cluster has loaded what it stores next.  Across a cluster: `seen` is made of the loaded values, so the loads are done;
// the arrival itself is relaxed, for a releasing one would wait for the stores of the pass before as well.
__device__ __forceinline__ void all_loaded(int ctas, uint32_t seen)
{
    if (ctas > 1) {
        asm volatile("{\n .reg .pred p;\n setp.eq.u32 p, %0, 0x5EED5EED;\n @p nanosleep.u32 0;\n}" ::"r"(seen) : "memory");
        asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    } else {
        __syncthreads();
    }
}

// Units: for every (sequence, KV head) its keys, its values and its weights; then for each the rings of keys and of values.  (With the
// weights read beside the keys, four bytes a row, the keys took twice the values' time.)
template <int NG> struct alignas(4 * NG) Parameters { uint32_t w[NG]; };      // of a row

template <int D, int NG>
__global__ void __launch_bounds__(kMoveThreads, 4) evict_move_kernel(const __grid_constant__ MoveArgs args)
{
    extern __shared__ __align__(16) uint8_t ring_rows[];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const PagedEvictArgs &a = args.a;
    const skvq_paged_config &cfg = a.p.cfg;
    const int H = cfg.n_kv_heads, pairs = H * a.p.batch.n_seqs, tid = threadIdx.x, C = args.ctas, rank = blockIdx.x % C, unit = blockIdx.x / C;
    const bool pages = unit < 3 * pairs;
    const int pair = pages ? unit / 3 : (unit - 3 * pairs) >> 1, side = pages ? unit % 3 : (unit - 3 * pairs) & 1, h = pair % H, b = pair / H;
    const EvictSeq s = static_cast<const EvictSeq *>(a.e.workspace)[b];
    const int slot = s.ok ? (a.p.batch.slots ? a.p.batch.slots[b] : b) : 0, slot_out = s.ok && a.e.slots_out ? a.e.slots_out[b] : slot;
    const int gone = s.len - s.left, R = cfg.ring_tokens;
    // ring rows that stay: of a sequence that lost tokens those of the recent ones, whose numbers all shift alike -- not at all, or by whole turns:
    // then no row has to move
    const bool in_place = cfg.window > 0 && slot == slot_out && gone % R == 0;
    const int t0 = cfg.window > 0 ? max(s.len - min(in_place ? R : min(R, kMaxRingMoved), gone ? a.e.recent : R), s.ring_from) : 0;
    if (pages && h == 0 && side == 0 && rank == 0 && tid == 0) {
        a.e.lens_out[b] = s.ok ? s.left : s.len;
        if (a.e.ring_from_out) a.e.ring_from_out[b] = s.ok && cfg.window > 0 ? max(t0, 0) - gone : s.ring_from;
    }
    if (!s.ok) return;
    if (pages && s.left == 0) return;
    const int32_t *kept = a.e.kept + ((int64_t)b * H + h) * a.e.keep;
    if (pages && side == 2) {
        const float *w = a.e.weights + ((int64_t)slot * H + h) * a.e.capacity;
        float *w_out = a.e.weights_out + ((int64_t)slot_out * H + h) * a.e.capacity;
        const int mine = rank * kMoveThreads * kUnroll + tid, pass = C * kMoveThreads * kUnroll;
        int next[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) next[u] = kept[min(mine + u * kMoveThreads, s.left - 1)];
        for (int base = 0; base < s.left; base += pass) {
            float x[kUnroll];
            uint32_t seen = 0u;
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) x[u] = w[next[u]];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                next[u] = kept[min(base + pass + mine + u * kMoveThreads, s.left - 1)];
                seen |= __float_as_uint(x[u]);
            }
            all_loaded(C, seen);
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const int i = base + mine + u * kMoveThreads;
                if (i < s.left) w_out[i] = x[u];
            }
        }
    } else if (pages) {
        constexpr int LANES = D / 32, PER_PASS = kMoveThreads / LANES;      // lanes of a row, 16 bytes each
        const int P = cfg.page_tokens, shift = __ffs(P) - 1;
        const int32_t *from = a.p.batch.page_table + (int64_t)b * a.p.batch.max_pages;
        const int32_t *to = a.e.page_table_out ? a.e.page_table_out + (int64_t)b * a.e.max_pages_out : from;
        uint4 *codes = static_cast<uint4 *>(side ? a.p.c.v_codes : a.p.c.k_codes);
        Parameters<NG> *meta = static_cast<Parameters<NG> *>(side ? a.p.c.v_meta : a.p.c.k_meta);
        const int lane = tid % LANES, row = rank * PER_PASS * kUnroll + tid / LANES, pass = C * PER_PASS * kUnroll;
        // Rows of the pool fit 32 bits: of one, keys and values take 72 bytes at least.  The pages that a row comes from and goes to are read a
        // pass ahead, the number of the token it is two passes ahead.
        constexpr uint32_t NONE = 0xFFFFFFFFu;
        int token[kUnroll], next[kUnroll], src_page[kUnroll], dst_page[kUnroll];
        uint32_t src[kUnroll], dst[kUnroll];
        // All of these load without a condition, from places that exist: behind branches the loads would wait for one another.
        auto numbers = [&](int base) {
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) next[u] = kept[min(base + u * PER_PASS + row, s.left - 1)];
        };
        auto pages_of = [&](int base) {      // of the tokens in `next`
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                token[u] = next[u];
                src_page[u] = from[next[u] >> shift];
                dst_page[u] = to[min(base + u * PER_PASS + row, s.left - 1) >> shift];
            }
        };
        auto places = [&](int base) {
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const int i = base + u * PER_PASS + row;
                const bool pages_exist = src_page[u] >= 0 && src_page[u] < cfg.n_pages && dst_page[u] >= 0 && dst_page[u] < cfg.n_pages;
                const bool moves = i < s.left && pages_exist && (src_page[u] != dst_page[u] || token[u] != i);
                src[u] = moves ? ((uint32_t)src_page[u] * H + h) * P + (token[u] & (P - 1)) : NONE;
                dst[u] = ((uint32_t)dst_page[u] * H + h) * P + (i & (P - 1));
                if (i < s.left && !pages_exist) set_status(a.p.c.status, SKVQ_STATUS_BAD_PAGE);
            }
        };
        numbers(0);
        pages_of(0);
        numbers(pass);
        for (int base = 0; base < s.left; base += pass) {
            uint4 c[kUnroll];
            Parameters<NG> m[kUnroll];
            places(base);
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                if (src[u] != NONE) {
                    c[u] = codes[(int64_t)src[u] * LANES + lane];
                    if (lane == 0) m[u] = meta[src[u]];
                }
            }
            pages_of(base + pass);
            numbers(base + 2 * pass);
            uint32_t seen = 0u;
            if (C > 1) {
#pragma unroll
                for (int u = 0; u < kUnroll; ++u) {
                    if (src[u] != NONE) seen |= c[u].x | c[u].y | c[u].z | c[u].w;
                    if (src[u] != NONE && lane == 0) {
#pragma unroll
                        for (int g = 0; g < NG; ++g) seen |= m[u].w[g];
                    }
                }
            }
            all_loaded(C, seen);
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                if (src[u] != NONE) {
                    codes[(int64_t)dst[u] * LANES + lane] = c[u];
                    if (lane == 0) meta[dst[u]] = m[u];
                }
            }
        }
    } else {
        // the ring: token t moves from row t % R to row (t - gone) % R, all rows of a strip through shared memory
        if (in_place) return;
        const int first = max(t0, 0), rows = s.len - first, pieces = args.strip / 16;
        uint8_t *win = static_cast<uint8_t *>(side ? a.p.c.v_win : a.p.c.k_win);
        const uint8_t *src = win + ((int64_t)slot * H + h) * R * (D * 2);
        uint8_t *dst = win + ((int64_t)slot_out * H + h) * R * (D * 2);
        uint4 *held = reinterpret_cast<uint4 *>(ring_rows);
        for (int c0 = rank * args.strip; c0 < D * 2; c0 += C * args.strip) {
            for (int e = tid; e < rows * pieces; e += kMoveThreads)
                held[e] = *reinterpret_cast<const uint4 *>(src + (int64_t)((first + e / pieces) % R) * (D * 2) + c0 + e % pieces * 16);
            __syncthreads();
            for (int e = tid; e < rows * pieces; e += kMoveThreads)
                *reinterpret_cast<uint4 *>(dst + (int64_t)((first - gone + e / pieces) % R) * (D * 2) + c0 + e % pieces * 16) = held[e];
            __syncthreads();
        }
    }
}

// A launch in clusters that may start while its predecessor on the stream drains.
template <typename Kern, typename Args>
cudaError_t launch_clusters(Kern kern, int clusters, int ctas, int threads, size_t smem, cudaStream_t stream, const Args &args)
{
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3((unsigned)clusters * ctas);
    lc.blockDim = dim3(threads);
    lc.dynamicSmemBytes = smem;
    lc.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = ctas;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    lc.attrs = attr;
    lc.numAttrs = 2;
    const cudaError_t e = cudaLaunchKernelEx(&lc, kern, args);
    if (e == cudaSuccess) count_launch();
    return e;
}

// A cluster's size: twice as many CTAs as long as the GPU has room for them (`room` per SM) and each keeps `least` of the `items`.
int cluster_size(long long units, long long items, long long least, int room)
{
    int c = 1;
    while (c < kMaxCluster && units * c * 2 <= (long long)room * sm_count() && items >= least * c * 2) c *= 2;
    return c;
}

cudaError_t launch_select(const PagedEvictArgs &a, cudaStream_t stream)
{
    const int pairs = a.p.cfg.n_kv_heads * a.p.batch.n_seqs;
    const long long most = a.p.batch.max_len - (long long)a.e.first - a.e.recent;      // of a middle
    constexpr int SMALL = 8, LARGE = 32;
    SelectArgs s{a, cluster_size(pairs, most, kSelectThreads * SMALL / 2, 4)};
    while (s.ctas < kMaxCluster && most > (long long)s.ctas * kSelectThreads * LARGE) s.ctas *= 2;      // what fits the registers is read once
    const long long share = (most + s.ctas - 1) / s.ctas;
    if (share <= kSelectThreads * SMALL) return launch_clusters(evict_select_kernel<SMALL>, pairs, s.ctas, kSelectThreads, 0, stream, s);
    if (share <= kSelectThreads * LARGE) return launch_clusters(evict_select_kernel<LARGE>, pairs, s.ctas, kSelectThreads, 0, stream, s);
    return launch_clusters(evict_select_kernel<0>, pairs, s.ctas, kSelectThreads, 0, stream, s);
}

template <int D, int NG> cudaError_t launch_move(const PagedEvictArgs &a, cudaStream_t stream)
{
    const skvq_paged_config &cfg = a.p.cfg;
    const int pairs = cfg.n_kv_heads * a.p.batch.n_seqs, rows = cfg.ring_tokens < kMaxRingMoved ? cfg.ring_tokens : kMaxRingMoved;
    constexpr int PASS = kMoveThreads / (D / 32) * kUnroll;
    // Shared memory for the ring's rows goes to every CTA, those of the pages too: rings of 1024 rows and more cost the pages occupancy.  The second and third
    // case above with rings of 264, 1024, 2048, 8192 rows (more of them to move in sequences that stay whole): 561, 740, 928, 1511 us; 227, 269, 273, 469.
    MoveArgs m{a, rows <= 1024 ? 64 : (rows <= 2048 ? 32 : 16), cluster_size(2LL * pairs, a.max_kept, PASS / 2, 6)};
    static unsigned long long done = 0;
    const cudaError_t e = configure_smem_once(evict_move_kernel<D, NG>, kMaxRingMoved * 16, done);
    if (e != cudaSuccess) return e;
    return launch_clusters(evict_move_kernel<D, NG>, (cfg.window > 0 ? 5 : 3) * pairs, m.ctas, kMoveThreads, cfg.window > 0 ? (size_t)rows * m.strip : 0, stream, m);
}

}  // namespace

size_t paged_evict_workspace_bytes(const skvq_paged_batch &batch) { return batch.n_seqs * sizeof(EvictSeq); }

cudaError_t launch_paged_evict(const PagedEvictArgs &a, cudaStream_t stream)
{
    const cudaError_t e = launch_select(a, stream);
    if (e != cudaSuccess) return e;
    if (a.p.cfg.head_dim == 128) return a.p.ng == 1 ? launch_move<128, 1>(a, stream) : a.p.ng == 2 ? launch_move<128, 2>(a, stream) : launch_move<128, 4>(a, stream);
    return a.p.ng == 1 ? launch_move<64, 1>(a, stream) : launch_move<64, 2>(a, stream);
}

}  // namespace skvq
