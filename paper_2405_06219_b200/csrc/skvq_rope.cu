// Rotary positions: frequencies (host), the cos/sin table, and the rotation of packed queries and keys.
//
// The rotation reads every element once and writes it once; the table adds 4 bytes per channel and token, shared by all
// heads of the token.  A thread therefore keeps the table entries of its channels in registers and walks over heads.
// Measured: 32k tokens of 32 + 8 heads of 128 channels, fp16: 123 us, 83 % of the copy rate; a decode step of 64 tokens 2.6 us, its launch.
#include <cmath>

#include "skvq_paged.cuh"

namespace skvq {
namespace {

constexpr int kMaxFreq = 128;
constexpr int kRopeThreads = 256;

struct TableArgs {
    double f[kMaxFreq];
    double amplitude;
    long long first;
    int n_freq, n_positions;
    float2 *table;
};

// p f is formed in two doubles (product and its rounding error), so the angle is good to 2^-53 whatever the position.
__global__ void __launch_bounds__(256) rope_table_kernel(const __grid_constant__ TableArgs a)
{
    const long long n = (long long)a.n_positions * a.n_freq;
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (long long)gridDim.x * blockDim.x) {
        const int j = (int)(i % a.n_freq);
        const double p = (double)(a.first + i / a.n_freq), f = a.f[j];
        const double hi = p * f, lo = fma(p, f, -hi);
        double s, c;
        sincos(hi, &s, &c);
        a.table[i] = make_float2((float)(a.amplitude * (c - lo * s)), (float)(a.amplitude * (s + lo * c)));
    }
}

struct RopeOperand {
    const void *x;
    void *y;
    int64_t xt, xh, yt, yh;
    int n_heads;
};
struct RopeArgs {
    RopeOperand op[2];
    const float *table;
    const int32_t *positions;
    int32_t *status;
    int n_tokens, n_positions, rot_dim, head_dim;
    float sign;               // -1: rotate back
    int heads, per_thread;    // heads of both operands; heads a thread walks over
    int groups, tasks;        // ceil(heads / per_thread); tasks per (token, head): pair vectors, then copied vectors
    int pair_tasks;
};

template <typename T, int V> struct alignas(sizeof(T) * V) Vec { T v[V]; };

// A task is V pairs of the rotated part (half layout: V channels and their V partners; interleaved: 2V neighbouring channels)
// or 2V channels behind it.
template <typename T, int V, bool INTERLEAVED>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const __grid_constant__ RopeArgs a)
{
    const long long i = (long long)blockIdx.x * kRopeThreads + threadIdx.x;
    const int task = (int)(i % a.tasks);
    const long long rest = i / a.tasks;
    const int group = (int)(rest % a.groups);
    const long long tok = rest / a.groups;
    if (tok >= a.n_tokens) return;
    const int p = a.positions[tok];
    if (p < 0 || p >= a.n_positions) {
        if (task == 0 && group == 0) set_status(a.status, SKVQ_STATUS_BAD_POSITION);
        return;
    }
    using VecT = Vec<T, V>;
    const bool rot = task < a.pair_tasks;
    const int half = a.rot_dim / 2;
    int c1, c2;             // first channels of the task's two vectors
    float cs[V], sn[V];
    if (rot) {
        const int j = task * V;
        c1 = INTERLEAVED ? 2 * j : j;
        c2 = INTERLEAVED ? 2 * j + V : j + half;
        const float *row = a.table + ((int64_t)p * half + j) * 2;
        Vec<float, V >= 2 ? 4 : 2> e;
        constexpr int PER = V >= 2 ? 2 : 1;       // pairs per load
#pragma unroll
        for (int k = 0; k < V; k += PER) {
            e = *reinterpret_cast<const decltype(e) *>(row + 2 * k);
#pragma unroll
            for (int m = 0; m < PER; ++m) { cs[k + m] = e.v[2 * m]; sn[k + m] = a.sign * e.v[2 * m + 1]; }
        }
    } else {
        c1 = a.rot_dim + (task - a.pair_tasks) * 2 * V;
        c2 = c1 + V;
    }
    const bool second = c2 < a.head_dim;      // the copied part may end inside a task
#pragma unroll 2
    for (int hh = 0; hh < a.per_thread; ++hh) {
        int h = group + hh * a.groups;        // neighbouring groups work on neighbouring heads
        if (h >= a.heads) break;
        const RopeOperand &o = h < a.op[0].n_heads ? a.op[0] : a.op[1];
        if (h >= a.op[0].n_heads) h -= a.op[0].n_heads;
        const T *x = static_cast<const T *>(o.x) + tok * o.xt + h * o.xh;
        T *y = static_cast<T *>(o.y) + tok * o.yt + h * o.yh;
        VecT u = *reinterpret_cast<const VecT *>(x + c1), w;
        if (second) w = *reinterpret_cast<const VecT *>(x + c2);
        if (rot) {
            if constexpr (INTERLEAVED) {
                // channels 2j .. 2j+V-1 in u, 2j+V .. 2j+2V-1 in w
                T e[2 * V];
#pragma unroll
                for (int k = 0; k < V; ++k) { e[k] = u.v[k]; e[V + k] = w.v[k]; }
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    const float x1 = Elem<T>::to_float(e[2 * k]), x2 = Elem<T>::to_float(e[2 * k + 1]);
                    e[2 * k] = Elem<T>::from_float(rotate_first(x1, x2, cs[k], sn[k]));
                    e[2 * k + 1] = Elem<T>::from_float(rotate_second(x1, x2, cs[k], sn[k]));
                }
#pragma unroll
                for (int k = 0; k < V; ++k) { u.v[k] = e[k]; w.v[k] = e[V + k]; }
            } else {
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    const float x1 = Elem<T>::to_float(u.v[k]), x2 = Elem<T>::to_float(w.v[k]);
                    u.v[k] = Elem<T>::from_float(rotate_first(x1, x2, cs[k], sn[k]));
                    w.v[k] = Elem<T>::from_float(rotate_second(x1, x2, cs[k], sn[k]));
                }
            }
        } else if (x == y) {
            continue;
        }
        *reinterpret_cast<VecT *>(y + c1) = u;
        if (second) *reinterpret_cast<VecT *>(y + c2) = w;
    }
}

template <typename T, int V>
cudaError_t launch_rope(RopeArgs a, bool interleaved, cudaStream_t stream)
{
    a.pair_tasks = a.rot_dim / 2 / V;
    a.tasks = a.pair_tasks + (a.head_dim - a.rot_dim + 2 * V - 1) / (2 * V);
    // Enough threads to fill the GPU first, then as many heads per thread as remain: the table is read once per thread.
    const long long all = (long long)a.n_tokens * a.heads * a.tasks, want = (long long)sm_count() * 2048;
    long long per = all / want;
    a.per_thread = (int)(per < 1 ? 1 : (per > 8 ? 8 : per));
    a.groups = (a.heads + a.per_thread - 1) / a.per_thread;
    const long long threads = (long long)a.n_tokens * a.groups * a.tasks, blocks = (threads + kRopeThreads - 1) / kRopeThreads;
    if (blocks > 0x7fffffffLL) return cudaErrorInvalidValue;
    if (interleaved) rope_kernel<T, V, true><<<(unsigned)blocks, kRopeThreads, 0, stream>>>(a);
    else rope_kernel<T, V, false><<<(unsigned)blocks, kRopeThreads, 0, stream>>>(a);
    count_launch();
    return cudaGetLastError();
}

// Rows t * ts + h * hs (dim elements each) that share an element would be written by several threads, in an order that nobody knows.
bool rows_overlap(int n_tokens, int n_heads, int64_t ts, int64_t hs, int dim)
{
    using Wide = __int128;
    const Wide t = ts < 0 ? -(Wide)ts : ts, h = hs < 0 ? -(Wide)hs : hs;
    if ((n_tokens > 1 && t < dim) || (n_heads > 1 && h < dim)) return true;
    if (n_tokens == 1 || n_heads == 1 || t >= (n_heads - 1) * h + dim || h >= (n_tokens - 1) * t + dim) return false;
    for (int dh = 1; dh < n_heads; ++dh) {      // neither lies within the other: the tokens nearest to dh heads away
        const Wide near = dh * h / t;
        for (Wide dt = near; dt <= near + 1; ++dt)
            if (dt < n_tokens && (dh * h > dt * t ? dh * h - dt * t : dt * t - dh * h) < dim) return true;
    }
    return false;
}

bool plain_pointer(const void *p, int elt) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(elt - 1)) == 0; }

}  // namespace
}  // namespace skvq

using namespace skvq;

extern "C" {

int skvq_rope_frequencies(int32_t rot_dim, const skvq_rope_scaling *s, double *f, double *amplitude)
{
    if (!s || !f || !amplitude || rot_dim < 2 || (rot_dim & 1)) return SKVQ_ERR_INVALID_ARG;
    if (rot_dim > 2 * kMaxFreq) return SKVQ_ERR_UNSUPPORTED;
    if (s->kind < SKVQ_ROPE_PLAIN || s->kind > SKVQ_ROPE_YARN) return SKVQ_ERR_UNSUPPORTED;
    if (!(s->base > 1.0) || !std::isfinite(s->base)) return SKVQ_ERR_INVALID_ARG;
    if (s->kind != SKVQ_ROPE_PLAIN && (!(s->factor >= 1.0) || !std::isfinite(s->factor))) return SKVQ_ERR_INVALID_ARG;
    if (s->kind == SKVQ_ROPE_NTK && rot_dim < 4) return SKVQ_ERR_UNSUPPORTED;
    if (s->kind == SKVQ_ROPE_YARN &&
        (s->original_positions < 1 || !(s->slow >= 0.0) || !(s->fast > s->slow) || !std::isfinite(s->fast)))
        return SKVQ_ERR_INVALID_ARG;
    double base = s->base;
    if (s->kind == SKVQ_ROPE_NTK) base *= std::pow(s->factor, (double)rot_dim / (rot_dim - 2));
    *amplitude = s->kind == SKVQ_ROPE_YARN ? 0.1 * std::log(s->factor) + 1.0 : 1.0;
    for (int j = 0; j < rot_dim / 2; ++j) {
        f[j] = std::pow(base, -2.0 * j / rot_dim);
        if (s->kind == SKVQ_ROPE_LINEAR) f[j] /= s->factor;
        if (s->kind == SKVQ_ROPE_YARN) {
            const double turns = s->original_positions * f[j] / (2.0 * 3.14159265358979323846);
            double keep = (turns - s->slow) / (s->fast - s->slow);      // 1: the frequency stays, 0: it is divided by the factor
            keep = keep < 0.0 ? 0.0 : (keep > 1.0 ? 1.0 : keep);
            f[j] = keep * f[j] + (1.0 - keep) * f[j] / s->factor;
        }
    }
    return SKVQ_OK;
}

int skvq_rope_table(const double *frequencies_host, int32_t n_freq, double amplitude, int64_t first_position,
                    int32_t n_positions, void *table, void *cuda_stream)
{
    if (!frequencies_host || n_freq < 1 || n_positions < 0 || first_position < 0 || !std::isfinite(amplitude)) return SKVQ_ERR_INVALID_ARG;
    if (n_freq > kMaxFreq || first_position > 0x7fffffffLL - n_positions) return SKVQ_ERR_UNSUPPORTED;
    if (n_positions == 0) return SKVQ_OK;
    if (!table) return SKVQ_ERR_INVALID_ARG;
    if (!plain_pointer(table, 8)) return SKVQ_ERR_MISALIGNED;
    TableArgs a;
    for (int j = 0; j < n_freq; ++j) {
        if (!std::isfinite(frequencies_host[j])) return SKVQ_ERR_INVALID_ARG;
        a.f[j] = frequencies_host[j];
    }
    for (int j = n_freq; j < kMaxFreq; ++j) a.f[j] = 0.0;
    a.amplitude = amplitude;
    a.first = first_position;
    a.n_freq = n_freq;
    a.n_positions = n_positions;
    a.table = static_cast<float2 *>(table);
    const long long n = (long long)n_positions * n_freq, blocks = (n + 255) / 256, most = (long long)sm_count() * 64;
    rope_table_kernel<<<(unsigned)(blocks < most ? blocks : most), 256, 0, static_cast<cudaStream_t>(cuda_stream)>>>(a);
    count_launch();
    return cudaGetLastError() == cudaSuccess ? SKVQ_OK : SKVQ_ERR_CUDA;
}

int skvq_rope_apply(const skvq_rope *rope, int32_t dtype, int32_t head_dim, const skvq_rope_tensor *ta,
                    const skvq_rope_tensor *tb, const int32_t *positions, int32_t n_tokens, int32_t inverse, int32_t *status,
                    void *cuda_stream)
{
    if (!rope || !ta || n_tokens < 0 || head_dim < 1 || (inverse != 0 && inverse != 1)) return SKVQ_ERR_INVALID_ARG;
    if (dtype != SKVQ_F16 && dtype != SKVQ_BF16 && dtype != SKVQ_F32) return SKVQ_ERR_UNSUPPORTED;
    if (rope->rot_dim < 2 || (rope->rot_dim & 1) || rope->rot_dim > head_dim || rope->n_positions < 0 ||
        (rope->interleaved != 0 && rope->interleaved != 1))
        return SKVQ_ERR_INVALID_ARG;
    if (head_dim > 512) return SKVQ_ERR_UNSUPPORTED;
    const int elt = dtype == SKVQ_F32 ? 4 : 2;
    RopeArgs a;
    const skvq_rope_tensor *t[2] = {ta, tb};
    bool wide = head_dim * elt % 16 == 0;      // 16-byte vectors everywhere
    a.heads = 0;
    for (int i = 0; i < 2; ++i) {
        a.op[i] = RopeOperand{};
        if (!t[i]) continue;
        if (t[i]->n_heads < 0) return SKVQ_ERR_INVALID_ARG;
        if (t[i]->n_heads > 65535) return SKVQ_ERR_UNSUPPORTED;
        if (t[i]->n_heads > 0 && n_tokens > 0 && (!t[i]->x || !t[i]->y)) return SKVQ_ERR_INVALID_ARG;
        if (!plain_pointer(t[i]->x, elt) || !plain_pointer(t[i]->y, elt)) return SKVQ_ERR_MISALIGNED;
        if (n_tokens > 0 && t[i]->n_heads > 0) {
            if (rows_overlap(n_tokens, t[i]->n_heads, t[i]->y_token_stride, t[i]->y_head_stride, head_dim)) return SKVQ_ERR_INVALID_ARG;
            if (t[i]->x == t[i]->y && ((n_tokens > 1 && t[i]->x_token_stride != t[i]->y_token_stride) ||
                                       (t[i]->n_heads > 1 && t[i]->x_head_stride != t[i]->y_head_stride)))
                return SKVQ_ERR_INVALID_ARG;
        }
        a.op[i] = RopeOperand{t[i]->x, t[i]->y, t[i]->x_token_stride, t[i]->x_head_stride, t[i]->y_token_stride, t[i]->y_head_stride, t[i]->n_heads};
        a.heads += t[i]->n_heads;
        wide = wide && plain_pointer(t[i]->x, 16) && plain_pointer(t[i]->y, 16) &&
               ((t[i]->x_token_stride | t[i]->x_head_stride | t[i]->y_token_stride | t[i]->y_head_stride) * elt) % 16 == 0;
    }
    if (n_tokens == 0 || a.heads == 0) return SKVQ_OK;
    if (!rope->table || !positions) return SKVQ_ERR_INVALID_ARG;
    if (!plain_pointer(rope->table, 16) || !plain_pointer(positions, 4) || !plain_pointer(status, 4)) return SKVQ_ERR_MISALIGNED;
    a.table = static_cast<const float *>(rope->table);
    a.positions = positions;
    a.status = status;
    a.n_tokens = n_tokens;
    a.n_positions = rope->n_positions;
    a.rot_dim = rope->rot_dim;
    a.head_dim = head_dim;
    a.sign = inverse ? -1.0f : 1.0f;
    // Vectors of 16 bytes where rows, heads and the halves of the rotated part start on 16-byte boundaries; single elements else.
    const int v = 16 / elt;
    wide = wide && (rope->interleaved ? rope->rot_dim % (2 * v) : rope->rot_dim / 2 % v) == 0;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    cudaError_t e;
    if (dtype == SKVQ_F16) e = wide ? launch_rope<__half, 8>(a, rope->interleaved, stream) : launch_rope<__half, 1>(a, rope->interleaved, stream);
    else if (dtype == SKVQ_BF16) e = wide ? launch_rope<__nv_bfloat16, 8>(a, rope->interleaved, stream) : launch_rope<__nv_bfloat16, 1>(a, rope->interleaved, stream);
    else e = wide ? launch_rope<float, 4>(a, rope->interleaved, stream) : launch_rope<float, 1>(a, rope->interleaved, stream);
    return e == cudaSuccess ? SKVQ_OK : SKVQ_ERR_CUDA;
}

}  // extern "C"
