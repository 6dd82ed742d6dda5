// skvq_paged_evict: every KV head of a sequence keeps its oldest and newest tokens and the most looked-at ones between them; their
// rows close up, in order.
//
// Two kernels.  The first finds, per (sequence, KV head), the threshold of the middle's weights by a radix selection (three digits
// of 11, 11 and 10 bits of the order-preserving integer of a float) and writes the kept tokens' numbers in order: those above the
// threshold, and of those at it the lowest-numbered.  The second moves rows: row i of the shortened sequence comes from token
// kept[i] >= i.  Rows of one pass are read before any of them is written, passes go upwards, and the sources of later passes lie
// behind what earlier passes write: so a sequence may be shortened inside its own pages.
#include "skvq_paged.cuh"
#include "skvq_paged_split.cuh"

namespace skvq {
namespace {

constexpr int kSelectThreads = 1024;
constexpr int kMoveThreads = 256;
constexpr int kUnroll = 4;
constexpr int kBins = 2048;

// What the second kernel needs of the first: the caller may have lens_out = lens, ring_from_out = ring_from.
struct alignas(16) EvictSeq {
    int len, left, ring_from, ok;      // tokens before, after; first token of the ring before
};

__device__ __forceinline__ bool evict_sequence(const PagedEvictArgs &a, int b, EvictSeq &s)
{
    const skvq_paged_batch &p = a.p.batch;
    s.len = p.lens[b];
    s.ring_from = p.ring_from ? max(min(p.ring_from[b], s.len), 0) : 0;
    const int from = p.slots ? p.slots[b] : b, to = a.e.slots_out ? a.e.slots_out[b] : from;
    const bool ok = s.len >= 0 && s.len <= p.max_len && from >= 0 && from < a.p.cfg.n_slots && to >= 0 && to < a.p.cfg.n_slots;
    s.left = min(s.len, a.e.keep);
    s.ok = ok;
    return ok;
}

// Larger weights have larger keys; -0 and +0 share one, and what is not a number has the smallest.
__device__ __forceinline__ uint32_t weight_key(float w)
{
    if (w != w) return 0u;
    const uint32_t u = __float_as_uint(w + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__global__ void __launch_bounds__(kSelectThreads) evict_select_kernel(const __grid_constant__ PagedEvictArgs a)
{
    __shared__ int hist[kBins];
    __shared__ int warp_sum[32], found_bin, found_above;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const int H = a.p.cfg.n_kv_heads, b = blockIdx.x / H, h = blockIdx.x % H;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    EvictSeq s;
    const bool ok = evict_sequence(a, b, s);
    if (h == 0 && tid == 0) {
        static_cast<EvictSeq *>(a.e.workspace)[b] = s;
        if (!ok) set_status(a.p.c.status, SKVQ_STATUS_BAD_BATCH);
    }
    int32_t *kept = a.e.kept + ((int64_t)b * H + h) * a.e.keep;
    if (!ok) s.left = 0;
    for (int64_t i = (int64_t)s.left + tid; i < a.e.keep; i += kSelectThreads) kept[i] = -1;
    if (s.left == s.len || !ok) {
        for (int i = tid; i < s.left; i += kSelectThreads) kept[i] = i;
        return;
    }
    const int first = a.e.first, end = s.len - a.e.recent, want = a.e.keep - first - a.e.recent;
    for (int i = tid; i < first; i += kSelectThreads) kept[i] = i;
    for (int i = tid; i < a.e.recent; i += kSelectThreads) kept[first + want + i] = end + i;
    if (want == 0) return;
    const float *w = a.e.weights + ((int64_t)(a.p.batch.slots ? a.p.batch.slots[b] : b) * H + h) * a.e.capacity;
    // ---- the threshold: the want-th largest key
    uint32_t prefix = 0u;
    int left = want;      // still to be found among the keys that begin with `prefix`
#pragma unroll 1
    for (int round = 0; round < 3; ++round) {
        const int shift = round == 0 ? 21 : (round == 1 ? 10 : 0), bits = round == 2 ? 10 : 11;
        for (int i = tid; i < kBins; i += kSelectThreads) hist[i] = 0;
        __syncthreads();
        for (int t = first + tid; t < end; t += kSelectThreads) {
            const uint32_t key = weight_key(w[t]);
            if (round == 0 || (key >> (shift + bits)) == prefix) atomicAdd(&hist[(key >> shift) & ((1u << bits) - 1u)], 1);
        }
        __syncthreads();
        // bins from the top: thread i owns bins kBins - 1 - 2 i and the one below
        const int hi = hist[kBins - 1 - 2 * tid], lo = hist[kBins - 2 - 2 * tid];
        int incl = hi + lo;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, incl, d);
            if (lane >= d) incl += v;
        }
        if (lane == 31) warp_sum[warp] = incl;
        __syncthreads();
        int before = incl - hi - lo;
        for (int k = 0; k < warp; ++k) before += warp_sum[k];
        if (before < left && before + hi >= left) { found_bin = kBins - 1 - 2 * tid; found_above = before; }
        else if (before + hi < left && before + hi + lo >= left) { found_bin = kBins - 2 - 2 * tid; found_above = before + hi; }
        __syncthreads();
        prefix = prefix << bits | (uint32_t)found_bin;
        left -= found_above;
        __syncthreads();
    }
    // ---- the kept tokens in order: all above the threshold, the first `left` at it
    int above = 0, equal = 0;      // so far
    for (int base = first; base < end; base += kSelectThreads) {
        const int t = base + tid;
        const uint32_t key = t < end ? weight_key(w[t]) : 0u;
        const bool gt = t < end && key > prefix, eq = t < end && key == prefix;
        const uint32_t gts = __ballot_sync(0xffffffffu, gt), eqs = __ballot_sync(0xffffffffu, eq);
        if (lane == 0) warp_sum[warp] = __popc(gts) << 16 | __popc(eqs);
        __syncthreads();
        int g = above, e = equal;
        for (int k = 0; k < 32; ++k) {
            const int v = warp_sum[k];
            if (k < warp) { g += v >> 16; e += v & 0xFFFF; }
            above += v >> 16;
            equal += v & 0xFFFF;
        }
        const uint32_t below = (1u << lane) - 1u;
        g += __popc(gts & below);
        e += __popc(eqs & below);
        if (gt || (eq && e < left)) kept[first + g + min(e, left)] = t;
        __syncthreads();
    }
}

struct MoveArgs {
    PagedEvictArgs a;
    int strip;      // bytes of a ring row that a CTA moves at a time
};

// blockIdx.x = 2 * (sequence * KV heads + KV head) + side (0 keys, 1 values), first for the pages, then again for the rings.
template <int D, int NG>
__global__ void __launch_bounds__(kMoveThreads) evict_move_kernel(const __grid_constant__ MoveArgs args)
{
    extern __shared__ __align__(16) uint8_t ring_rows[];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;");
    const PagedEvictArgs &a = args.a;
    const skvq_paged_config &cfg = a.p.cfg;
    const int H = cfg.n_kv_heads, units = 2 * H * a.p.batch.n_seqs, tid = threadIdx.x;
    const bool pages = (int)blockIdx.x < units;
    const int unit = pages ? blockIdx.x : blockIdx.x - units;
    const int side = unit & 1, h = (unit >> 1) % H, b = (unit >> 1) / H;
    const EvictSeq s = static_cast<const EvictSeq *>(a.e.workspace)[b];
    const int slot = s.ok ? (a.p.batch.slots ? a.p.batch.slots[b] : b) : 0, slot_out = s.ok && a.e.slots_out ? a.e.slots_out[b] : slot;
    const int gone = s.len - s.left, R = cfg.ring_tokens;
    // ring rows that stay: of a sequence that lost tokens those of the recent ones, whose numbers all shift alike
    const int t0 = cfg.window > 0 ? max(s.len - min(min(R, kMaxRingMoved), gone ? a.e.recent : R), s.ring_from) : 0;
    if (pages && h == 0 && side == 0 && tid == 0) {
        a.e.lens_out[b] = s.ok ? s.left : s.len;
        if (a.e.ring_from_out) a.e.ring_from_out[b] = s.ok && cfg.window > 0 ? max(t0, 0) - gone : s.ring_from;
    }
    if (!s.ok) return;
    if (pages) {
        constexpr int LANES = D / 32, PER_PASS = kMoveThreads / LANES;      // lanes of a row, 16 bytes each
        const int P = cfg.page_tokens, shift = __ffs(P) - 1;
        const int32_t *kept = a.e.kept + ((int64_t)b * H + h) * a.e.keep;
        const int32_t *from = a.p.batch.page_table + (int64_t)b * a.p.batch.max_pages;
        const int32_t *to = a.e.page_table_out ? a.e.page_table_out + (int64_t)b * a.e.max_pages_out : from;
        uint4 *codes = static_cast<uint4 *>(side ? a.p.c.v_codes : a.p.c.k_codes);
        uint32_t *meta = static_cast<uint32_t *>(side ? a.p.c.v_meta : a.p.c.k_meta);
        const float *w = a.e.weights + ((int64_t)slot * H + h) * a.e.capacity;
        float *w_out = a.e.weights_out + ((int64_t)slot_out * H + h) * a.e.capacity;
        const int lane = tid % LANES, row = tid / LANES;
        for (int base = 0; base < s.left; base += PER_PASS * kUnroll) {
            uint4 c[kUnroll];
            uint32_t m[kUnroll][NG];
            float x[kUnroll];
            int64_t dst[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const int i = base + u * PER_PASS + row;
                dst[u] = -1;
                if (i >= s.left) continue;
                const int t = kept[i], src_page = from[t >> shift], dst_page = to[i >> shift];
                if (src_page < 0 || src_page >= cfg.n_pages || dst_page < 0 || dst_page >= cfg.n_pages) set_status(a.p.c.status, SKVQ_STATUS_BAD_PAGE);
                else if (src_page != dst_page || t != i) {
                    const int64_t src = ((int64_t)src_page * H + h) * P + (t & (P - 1));
                    dst[u] = ((int64_t)dst_page * H + h) * P + (i & (P - 1));
                    c[u] = codes[src * LANES + lane];
                    if (lane == 0) {
#pragma unroll
                        for (int g = 0; g < NG; ++g) m[u][g] = meta[src * NG + g];
                    }
                }
                if (lane == 0 && side == 0) x[u] = w[t];
            }
            __syncthreads();
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const int i = base + u * PER_PASS + row;
                if (i >= s.left) continue;
                if (lane == 0 && side == 0) w_out[i] = x[u];
                if (dst[u] < 0) continue;
                codes[dst[u] * LANES + lane] = c[u];
                if (lane == 0) {
#pragma unroll
                    for (int g = 0; g < NG; ++g) meta[dst[u] * NG + g] = m[u][g];
                }
            }
        }
    } else {
        // the ring: token t moves from row t % R to row (t - gone) % R, all rows of a strip through shared memory
        if (slot == slot_out && gone % R == 0) return;
        const int first = max(t0, 0), rows = s.len - first, pieces = args.strip / 16;
        uint8_t *win = static_cast<uint8_t *>(side ? a.p.c.v_win : a.p.c.k_win);
        const uint8_t *src = win + ((int64_t)slot * H + h) * R * (D * 2);
        uint8_t *dst = win + ((int64_t)slot_out * H + h) * R * (D * 2);
        uint4 *held = reinterpret_cast<uint4 *>(ring_rows);
        for (int c0 = 0; c0 < D * 2; c0 += args.strip) {
            for (int e = tid; e < rows * pieces; e += kMoveThreads)
                held[e] = *reinterpret_cast<const uint4 *>(src + (int64_t)((first + e / pieces) % R) * (D * 2) + c0 + e % pieces * 16);
            __syncthreads();
            for (int e = tid; e < rows * pieces; e += kMoveThreads)
                *reinterpret_cast<uint4 *>(dst + (int64_t)((first - gone + e / pieces) % R) * (D * 2) + c0 + e % pieces * 16) = held[e];
            __syncthreads();
        }
    }
}

template <int D, int NG> cudaError_t launch_move(const PagedEvictArgs &a, cudaStream_t stream)
{
    const skvq_paged_config &cfg = a.p.cfg;
    const int units = 2 * cfg.n_kv_heads * a.p.batch.n_seqs, rows = cfg.ring_tokens < kMaxRingMoved ? cfg.ring_tokens : kMaxRingMoved;
    MoveArgs m{a, rows <= 1024 ? 64 : (rows <= 2048 ? 32 : 16)};
    static unsigned long long done = 0;
    const cudaError_t e = configure_smem_once(evict_move_kernel<D, NG>, kMaxRingMoved * 16, done);
    if (e != cudaSuccess) return e;
    return launch_chained(evict_move_kernel<D, NG>, dim3(cfg.window > 0 ? 2 * units : units), kMoveThreads, cfg.window > 0 ? (size_t)rows * m.strip : 0, stream, m);
}

}  // namespace

size_t paged_evict_workspace_bytes(const skvq_paged_batch &batch) { return batch.n_seqs * sizeof(EvictSeq); }

cudaError_t launch_paged_evict(const PagedEvictArgs &a, cudaStream_t stream)
{
    const cudaError_t e = launch_chained(evict_select_kernel, dim3(a.p.cfg.n_kv_heads * a.p.batch.n_seqs), kSelectThreads, 0, stream, a);
    if (e != cudaSuccess) return e;
    if (a.p.cfg.head_dim == 128) return a.p.ng == 1 ? launch_move<128, 1>(a, stream) : a.p.ng == 2 ? launch_move<128, 2>(a, stream) : launch_move<128, 4>(a, stream);
    return a.p.ng == 1 ? launch_move<64, 1>(a, stream) : launch_move<64, 2>(a, stream);
}

}  // namespace skvq
