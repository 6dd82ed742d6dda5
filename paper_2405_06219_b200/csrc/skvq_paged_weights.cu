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

#include "skvq_paged.cuh"
#include "skvq_paged_split.cuh"

namespace skvq {
namespace {

constexpr int kQueryThreads = 128;
constexpr int kQueryTokens = kQueryThreads / 16;
constexpr int kTileRows = 128;      // rows of a query tile where sequences may have many

// A query tile: `rows` rows of D fp16, 64-channel halves one after the other, a half's rows 128 bytes each with 16-byte piece c of row r
// at c ^ (r & 7) (the 128-byte swizzle of the tensor core's operands); then floats [rows] factor of a score in units of log2, [rows]
// minus the lse in units of log2 (minus infinity: the row adds nothing), [NG][rows] sums of the row over a group's channels.
struct WeightPlan {
    PagedWeightArgs a;
    int tile_rows;        // 16 or kTileRows
    int seq_tiles;        // > 0: sequence b's tiles begin at b * seq_tiles; 0: at starts[b] * Hq/Hkv / tile_rows + b
    int heads;            // query heads that a CTA of the first kernel walks over
};
__host__ __device__ inline int tile_bytes(int rows, int D, int ng) { return rows * (D * 2 + (2 + ng) * 4); }

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
    const int64_t base = p.seq_tiles ? (int64_t)b * p.seq_tiles : (int64_t)w.s.row0 * w.rep / p.tile_rows + b;
    return p.a.ws + ((base + tile) * p.a.p.cfg.n_kv_heads + h) * tile_bytes(p.tile_rows, p.a.p.cfg.head_dim, p.a.p.ng);
}

// Position 0..7 inside a run of eight operand channels -> stored channel: nibbles i and i + 4 of a code word become neighbours.
__device__ __forceinline__ int channel_at(int pos) { return (pos >> 1) + 4 * (pos & 1); }

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
    if (!w.ok) return;
    // a tile that is read whole has zeros behind its last row
    const int filled = plan.tile_rows == kTileRows ? (w.rows + kTileRows - 1) / kTileRows * kTileRows : w.rows;
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
        float up = 1.f;      // the row's largest to [2^13, 2^14): exact, whatever the type's range
        if (mx > 0.f && counts) up = __int_as_float((127 + min(13 - (__float_as_int(mx) >> 23) + 127, 60)) << 23);
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
        uint8_t *tile = const_cast<uint8_t *>(query_tile(plan, w, b, hk, r / plan.tile_rows));
        const int tr = r % plan.tile_rows;
        uint8_t *dst = tile + (c0 >> 6) * plan.tile_rows * 128 + tr * 128 + (((((c0 >> 3) & 7) ^ (tr & 7)) << 4)) + (c0 & 7) * 2;
        if constexpr (C == 8)
            *reinterpret_cast<uint4 *>(dst) = make_uint4(packed<__half>(x[0], x[1]), packed<__half>(x[2], x[3]), packed<__half>(x[4], x[5]), packed<__half>(x[6], x[7]));
        else *reinterpret_cast<uint2 *>(dst) = make_uint2(packed<__half>(x[0], x[1]), packed<__half>(x[2], x[3]));
        float *constants = reinterpret_cast<float *>(tile + plan.tile_rows * D * 2) + tr;
        if (sub == 0) {
            constants[0] = a.sm_scale * 1.4426950408889634f / up;
            constants[plan.tile_rows] = counts ? lse * -1.4426950408889634f : -CUDART_INF_F;
        }
        if (sub % (16 / NG) == 0) constants[(2 + sub / (16 / NG)) * plan.tile_rows] = sum;
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
    if (!w.ok) {
        if (threadIdx.x == 0) set_status(a.p.c.status, SKVQ_STATUS_BAD_BATCH);
        return;
    }
    if ((int)blockIdx.x * kTokens >= w.s.len) return;
    const int P = cfg.page_tokens;
    bool have = t < w.s.len && w.rows > 0;
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
            const int r = r0 + e / D, c = e % D, tr = r % plan.tile_rows;
            if (r >= w.rows) break;
            const uint8_t *tile = query_tile(plan, w, b, h, r / plan.tile_rows);
            query[e / D][(c & ~7) + channel_at(c & 7)] = __half2float(*reinterpret_cast<const __half *>(
                tile + (c >> 6) * plan.tile_rows * 128 + tr * 128 + ((((c >> 3) & 7) ^ (tr & 7)) << 4) + (c & 7) * 2));
            if (c < 2 + NG) constants[e / D][c] = reinterpret_cast<const float *>(tile + plan.tile_rows * D * 2)[c * plan.tile_rows + tr];
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

// The layout of the query tiles.
void plan_tiles(const skvq_paged_config &cfg, const skvq_paged_batch &batch, int last, WeightPlan &p, int64_t &tiles)
{
    const int64_t rep = cfg.n_q_heads / cfg.n_kv_heads, most = last && last < batch.max_new ? last : batch.max_new;
    p.tile_rows = most * rep <= 16 ? 16 : kTileRows;
    const int64_t uniform = (most * rep + p.tile_rows - 1) / p.tile_rows, together = batch.n_tokens * rep / p.tile_rows + batch.n_seqs;
    const bool by_seq = uniform * batch.n_seqs <= together || (last && last < batch.max_new);
    p.seq_tiles = by_seq ? (int)uniform : 0;
    tiles = by_seq ? uniform * batch.n_seqs : together;
}

template <typename T, int D, int NG> cudaError_t launch_weights(const PagedWeightArgs &a, cudaStream_t stream)
{
    const skvq_paged_config &cfg = a.p.cfg;
    const skvq_paged_batch &batch = a.p.batch;
    WeightPlan p{};
    p.a = a;
    int64_t tiles;
    plan_tiles(cfg, batch, a.last, p, tiles);
    cudaError_t e;
    const int64_t rep = cfg.n_q_heads / cfg.n_kv_heads, most = a.last && a.last < batch.max_new ? a.last : batch.max_new;
    if (batch.n_tokens > 0 && most > 0) {
        const int64_t rows = p.tile_rows == kTileRows ? (most * rep + kTileRows - 1) / kTileRows * kTileRows : most * rep;
        const int64_t chunks = ((rows + rep - 1) / rep + kQueryTokens - 1) / kQueryTokens;
        p.heads = cfg.n_q_heads;
        while (p.heads > 4 && chunks * batch.n_seqs * ((cfg.n_q_heads + p.heads - 1) / p.heads) < 32LL * sm_count()) p.heads = (p.heads + 1) / 2;
        e = launch_chained(weight_queries_kernel<T, D, NG>, dim3((unsigned)chunks, (cfg.n_q_heads + p.heads - 1) / p.heads, batch.n_seqs), kQueryThreads, 0, stream, p);
        if (e != cudaSuccess) return e;
    }
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
    WeightPlan p{};
    int64_t tiles;
    plan_tiles(cfg, batch, last, p, tiles);
    return (size_t)tiles * cfg.n_kv_heads * tile_bytes(p.tile_rows, cfg.head_dim, cfg.head_dim / cfg.group_size);
}

cudaError_t launch_paged_weights(const PagedWeightArgs &a, cudaStream_t stream)
{
    if (a.p.batch.max_len == 0) return cudaSuccess;
    return a.p.cfg.dtype == SKVQ_F16 ? launch_by_shape<__half>(a, stream) : launch_by_shape<__nv_bfloat16>(a, stream);
}

}  // namespace skvq
