/*
 * skvq.h -- C ABI of the B200-native SKVQ hot path (sliding-window KV-cache
 * quantization, arXiv 2405.06219): append tokens to a cache whose older part is
 * 2/4-bit group-quantized, and run decode attention directly on that cache.
 *
 * General rules
 *   - Every pointer is a DEVICE pointer owned by the caller unless its comment
 *     says "host".  The library allocates nothing, frees nothing and keeps no
 *     pointer after a call returns.
 *   - Every device buffer must be 16-byte aligned.
 *   - Calls only enqueue work on `cuda_stream` (a cudaStream_t passed as void*,
 *     NULL = the default stream); they never synchronise.  Lengths are read on
 *     the device.
 *   - Return value: SKVQ_OK or a negative SKVQ_ERR_* code.  On an error nothing
 *     is launched.  Conditions only the device can see (a sequence that would
 *     exceed its capacity) leave that sequence untouched and OR a bit into
 *     the cache's status word.
 *   - Kernels of one call, and of consecutive calls on a stream, are chained with programmatic
 *     dependent launches: a kernel may be scheduled while its predecessor on the stream drains
 *     and waits on the device before it touches that predecessor's results.  Nothing changes for
 *     the caller: stream order is kept.
 *   - Compiled for sm_100a only; there is no CPU path.
 *
 * Notation: B sequences, Hq query heads, Hkv KV heads (Hq % Hkv == 0, query head
 * hq reads KV head hq / (Hq/Hkv)), D = head_dim, W = window, G = group size,
 * ng = D/G groups per row, L_b = lengths[b], Lq_b = max(L_b - W, 0) tokens of
 * sequence b that have left the window; of those, positions below n_sink (attention
 * sinks) stay fp16 and the rest are quantized.
 */
#ifndef SKVQ_H_
#define SKVQ_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SKVQ_OK 0
#define SKVQ_ERR_INVALID_ARG (-1) /* NULL where a buffer is required, negative size, ... */
#define SKVQ_ERR_UNSUPPORTED (-2) /* head_dim != 128, k_bits not in {2,3,4}, v_bits not in {2,3,4,15}, G not in {32,64,128}, Hq % Hkv != 0, Hq/Hkv > 8 */
#define SKVQ_ERR_MISALIGNED (-3)  /* a device buffer is not 16-byte aligned */
#define SKVQ_ERR_CAPACITY (-4)    /* host-visible overflow: n_new or max_len_hint beyond max_tokens */
#define SKVQ_ERR_WORKSPACE (-5)   /* workspace missing or smaller than skvq_workspace_size() */
#define SKVQ_ERR_CUDA (-6)        /* the CUDA runtime reported an error at launch */
#define SKVQ_ERR_SCRATCH_LIMIT (-7) /* skvq_decode_attention_noalloc: the split partials of this shape need more
                                     than SKVQ_NOALLOC_SCRATCH_BYTES */

#define SKVQ_STATUS_OVERFLOW 1    /* bit set in *status when a sequence would have exceeded max_tokens */
#define SKVQ_STATUS_COPY_TIMEOUT 2 /* bit set when a shared-memory copy inside decode attention never completed (bounded
                                     wait ran out); the affected tokens contribute nothing to the result;
                                     skvq_paged_attention: the affected rows are NaN; skvq_paged_weights: the
                                     affected weights are NaN */
#define SKVQ_STATUS_BOUNDS 4       /* only from a library built with -DSKVQ_CHECKED (a debugging build): a kernel was about to
                                     use a row, slot or partial index outside its buffer; the access was skipped */

#define SKVQ_STATUS_BAD_BATCH 8    /* paged calls: a sequence's lens/starts/slots entry is out of range; that sequence was skipped */
#define SKVQ_STATUS_BAD_PAGE 16    /* paged calls: a page-table entry is not a page of the pool; its tokens were skipped */
#define SKVQ_STATUS_BAD_POSITION 32 /* skvq_rope_apply, skvq_rope_apply_axes: a position lies outside the table; that token's rows were not written */

/* Rows of the quantized segment are allocated in multiples of this many tokens so
 * that a kernel may stage whole tiles; see skvq_quant_capacity(). */
#define SKVQ_TOKEN_ALIGN 64

/* Group boundaries (skvq_cache::group_bounds_*) are multiples of this many channels. */
#define SKVQ_GROUP_GRANULE 32

/* v_bits value of the "1.5-bit" setting for values (abstract; Sec. 4.2: keys at 2 bits, values at 1.5 bits): three
 * levels per code (2^1.5 = 2.83 rounds to 3), five codes per byte in base 3.  The paper gives neither the levels nor the
 * storage of that setting; this is the library's reading of it. */
#define SKVQ_BITS_TERNARY 15

/* Shape and quantization settings (host struct). */
typedef struct skvq_config {
    int32_t batch;       /* B >= 1 */
    int32_t n_q_heads;   /* Hq */
    int32_t n_kv_heads;  /* Hkv */
    int32_t head_dim;    /* D, must be 128 */
    int32_t k_bits;      /* 2, 3 or 4 (3: the 3-bit setting of the paper's comparison with KVQuant, Sec. 4.3) */
    int32_t v_bits;      /* 2, 3, 4 or SKVQ_BITS_TERNARY (three-level codes, 1.625 bits per element stored) */
    int32_t group_size;  /* G: 32, 64 or 128; a row has ng = D/G groups that share scale/zero: equal runs of G consecutive
                            (reordered) channels, or, with skvq_cache::group_bounds_*, ng runs of unequal width whose
                            AVERAGE width is G (Sec. 4.2: the number of groups is kept, not their size) */
    int32_t window;      /* W >= 0 latest tokens kept in fp16 (Sec. 3.2); 0 quantizes everything */
    int32_t max_tokens;  /* per-sequence capacity (quantized segment + window) */
    int32_t n_sink;      /* 0..64: the first n_sink positions of a sequence are never quantized (Sec. 3.2, filter
                            rules; the paper's experiments keep 5); 0 = none */
    int32_t meta_fp8;    /* 0: scale and zero point stored in fp16; 1: in FP8 E4M3 (Sec. 4.1 "Quantization"; 2.5
                            instead of 3 bits per element at 2 bits and group 32).  The codes are computed
                            against the stored, rounded parameters either way. */
} skvq_config;

/*
 * The cache (host struct of device pointers).  cap = skvq_quant_capacity(cfg).
 * Layouts are row-major:
 *   k_codes/v_codes  uint8   [B][Hkv][cap][D*bits/8]  a row is a little-endian bit stream: code j = bits [j*bits, (j+1)*bits)
 *                                                     of the row, j counted in reordered order (2- and 4-bit codes never
 *                                                     cross a byte; a 3-bit code may: 8 codes per 3 bytes, 48-byte rows).
 *                                                     v_bits = SKVQ_BITS_TERNARY: (D+4)/5 = 26 bytes per row, code j is
 *                                                     base-3 digit j % 5 (weight 3^(j % 5)) of byte j / 5; the two unused
 *                                                     digits of the last byte are 0
 *   k_meta/v_meta    half2   [B][Hkv][cap][ng]        {scale h, zero z}; dequantized x^ = h*code + z.  With meta_fp8:
 *                    uint8   [B][Hkv][cap][ng][2]     {E4M3 byte of h, E4M3 byte of z} (1 sign, 4 exponent bits with
 *                                                     bias 7, 3 mantissa bits, no infinities, largest finite 448;
 *                                                     rounded to nearest even from fp32, saturating)
 *   k_win/v_win      half    [B][Hkv][W][D]           ring; token t sits in slot t % W, reordered order
 *   lengths          int32   [B]                      tokens appended so far (start at 0)
 *   reorder_k/_v     int32   [Hkv][D]                 gather index: stored[j] = source[idx[j]]; each
 *                                                     row must be a permutation of 0..D-1 (Eq. 1)
 *   alpha_k/_v       float   [Hkv][ng]                clip factor per group in (0,1] (Eq. 2)
 *   status           int32   [1]                      optional (may be NULL); SKVQ_STATUS_* bits are OR-ed in
 *   k_sink/v_sink    half    [B][Hkv][n_sink][D]      position t < n_sink once it has left the window, reordered
 *                                                     order; may be NULL when n_sink == 0
 *   group_bounds_k/_v int32  [Hkv][ng+1]              optional (NULL = equal groups): group g of KV head h covers reordered
 *                                                     channels [bounds[h][g], bounds[h][g+1]); bounds[h][0] = 0,
 *                                                     bounds[h][ng] = D, strictly increasing, every entry a multiple of
 *                                                     SKVQ_GROUP_GRANULE (Sec. 3.1: channels of similar range share a
 *                                                     group; split_groups(X, group_indices) of Algorithm 1).  The arrays
 *                                                     live on the device, so the library cannot check them: validate the
 *                                                     host copy with skvq_check_group_bounds() before uploading it.
 * Rows at or beyond Lq_b, and rows below n_sink, of the quantized buffers hold unspecified bytes.  The buffers fully describe the state:
 * copying them is a checkpoint.
 */
typedef struct skvq_cache {
    void *k_codes, *v_codes;
    void *k_meta, *v_meta;
    void *k_win, *v_win;
    int32_t *lengths;
    const int32_t *reorder_k, *reorder_v;
    const float *alpha_k, *alpha_v;
    int32_t *status;
    void *k_sink, *v_sink;
    const int32_t *group_bounds_k, *group_bounds_v;
} skvq_cache;

/* Options of one decode-attention call (host struct). */
typedef struct skvq_attn_args {
    float sm_scale;         /* softmax scale, e.g. 1/sqrt(D) */
    int32_t max_len_hint;   /* host upper bound on lengths[] (sizes the grid); <= max_tokens */
    int32_t n_splits;       /* 0 = library chooses (one CTA per resident slot of the GPU, all with the same share of
                               the batch's quantized tokens); n > 0 asks for about n pieces per (sequence, KV head) */
    void *workspace;        /* device scratch for the split partials, >= skvq_workspace_size() bytes */
    size_t workspace_bytes;
    void *ev_begin, *ev_end;/* optional cudaEvent_t (else NULL) recorded on the stream immediately
                               before / after the partition kernel, for profiling; events keep the merge kernel from
                               overlapping the partition kernel's tail, so leave them NULL in production */
} skvq_attn_args;

/* Library version (major*100 + minor). */
int skvq_version(void);

/* Static text for a return code. */
const char *skvq_strerror(int code);

/* Number of CUDA kernels this library has launched in this process (monotonic). */
uint64_t skvq_launch_count(void);

/* Validate cfg (host only).  Returns SKVQ_OK or the error a call with it would return. */
int skvq_check_config(const skvq_config *cfg);

/* Validate group boundaries on the host: bounds is int32 [n_kv_heads][ng+1] with ng = head_dim / group_size.  Returns
 * SKVQ_OK, or SKVQ_ERR_INVALID_ARG when a row does not start at 0, end at head_dim, increase strictly, or holds an entry
 * that is not a multiple of SKVQ_GROUP_GRANULE. */
int skvq_check_group_bounds(const skvq_config *cfg, const int32_t *bounds_host);

/* Rows per (sequence, KV head) in the quantized segment:
 * round_up(max(max_tokens - W, 0), SKVQ_TOKEN_ALIGN), at least SKVQ_TOKEN_ALIGN.  Negative on a bad cfg. */
int32_t skvq_quant_capacity(const skvq_config *cfg);

/* Bytes of k_codes, v_codes, k_meta, v_meta, k_win, v_win (in that order) for cfg.  Host only. */
int skvq_cache_sizes(const skvq_config *cfg, size_t bytes_out[6]);

/* Bytes of k_sink (= v_sink) for cfg; 0 when n_sink == 0 or on a bad cfg.  Host only. */
size_t skvq_sink_bytes(const skvq_config *cfg);

/*
 * Append tokens (Sec. 3.2, Algorithm 1 body, clipping_quant; Eq. 2).
 * Sequence b receives n_b = n_new_per_seq ? n_new_per_seq[b] : n_new tokens (0 <= n_b <= n_new).
 * With L0 = lengths[b], L1 = L0 + n_b: every token in [max(L0-W,0), max(L1-W,0)) is reordered
 * (stored[j] = x[idx[j]]), split into groups of G channels and quantized per group:
 *   lo = alpha*min, hi = alpha*max, h = fp16((hi-lo)/qmax), z = fp16(lo),
 *   code = clamp(rint((x - z)/h), 0, qmax)   (fp32, IEEE division, ties to even; h == 0 -> code 0;
 *                                             qmax = 2^bits-1, or 2 for the three-level codes)
 * (min, max and alpha are those of the channel's group: equal runs of G channels, or the runs given by group_bounds_*)
 * the last min(L1, W) tokens are kept in fp16 in the ring, and lengths[b] becomes L1.
 * Exception (Sec. 3.2, the filter mask of Algorithm 1): a token at a position below n_sink is copied, reordered,
 * to k_sink/v_sink when it leaves the window instead of being quantized.
 * One bulk call equals the same tokens appended one at a time.
 *   k, v           half [B][n_new][Hkv][D], original channel order (rows beyond n_b are ignored)
 *   n_new_per_seq  device int32 [B] or NULL
 * If L1 > max_tokens the sequence is left unchanged and SKVQ_STATUS_OVERFLOW is set in *status.
 * NaN/Inf inputs give unspecified codes.
 */
int skvq_quantize_append(const skvq_config *cfg, const skvq_cache *cache, const void *k, const void *v,
                         const int32_t *n_new_per_seq, int32_t n_new, void *cuda_stream);

/* Scratch bytes skvq_decode_attention needs for lengths up to max_len_hint and the given n_splits
 * (0 = the library's choice for that hint; the choice depends on the GPU's SM count, so ask on the
 * machine that will run the call).  0 on a bad cfg. */
size_t skvq_workspace_size(const skvq_config *cfg, int32_t max_len_hint, int32_t n_splits);

/*
 * Decode attention of one query per sequence over [quantized prefix || fp16 window]
 * (Eq. 1 and the first lines of Algorithm 1; softmax and its scale written out):
 *   q' = q[reorder_k],  s_t = sm_scale * sum_j q'_j K~[t][j],  p = softmax_t(s),
 *   o'_j = sum_t p_t V~[t][j],  out[reorder_v[j]] = o'_j,
 * where K~/V~ are h*code+z for t < Lq_b (the sink row for t < n_sink) and the ring value for Lq_b <= t < L_b.  Dequantization
 * happens in registers; no dequantized cache is written.  A sequence of length 0 yields zeros.
 * Tokens beyond max_len_hint (a sequence longer than the hint) are not looked at.
 *   q    half [B][Hq][D]      out  half [B][Hq][D]
 * The workspace contents are overwritten; calls sharing a workspace must be stream-ordered.
 */
int skvq_decode_attention(const skvq_config *cfg, const skvq_cache *cache, const void *q, void *out,
                          const skvq_attn_args *args, void *cuda_stream);

/*
 * One decode step driven from HOST buffers: copies k_new, v_new (half [B][1][Hkv][D]) and q
 * (half [B][Hq][D]) from host memory into `staging`, appends the token, runs decode attention and
 * copies out (half [B][Hq][D]) back to host memory, all enqueued on the stream (the caller
 * synchronises before reading out_host).  Pinned host memory keeps the copies asynchronous; when k_new, v_new
 * and q lie back to back in host memory in that order they travel in one copy instead of three.
 *   staging  device scratch of at least skvq_step_staging_size(cfg) bytes
 */
size_t skvq_step_staging_size(const skvq_config *cfg);
int skvq_decode_step_host(const skvq_config *cfg, const skvq_cache *cache, const void *k_new_host,
                          const void *v_new_host, const void *q_host, void *out_host, void *staging,
                          const skvq_attn_args *args, void *cuda_stream);

/*
 * Decode attention for callers that have no device memory left to lend and must not allocate.
 * (The paper has no counterpart: this is a packaging variant of skvq_decode_attention, same result.)
 *
 * Who needs it: a serving engine usually sizes its KV cache to swallow whatever HBM remains after the
 * weights, so by the time the decode loop runs there is no spare buffer to pass as `workspace`, and a
 * cudaMalloc inside that loop would either fail or stall every stream on the device while it runs.  The
 * same holds for code that runs as a plug-in inside somebody else's memory pool and may not call the
 * allocator at all.  For them the split partials go into an array that is part of the library image:
 * SKVQ_NOALLOC_SCRATCH_BYTES of device memory on every GPU that loads the library, held until exit.
 * The call itself allocates and frees nothing (no cudaMalloc/cudaFree, no allocating library routine).
 *
 * Arguments are those of skvq_decode_attention with the fields of skvq_attn_args passed directly; q, out and
 * the cache are still the caller's.  Limits and rules:
 *   - Shapes whose partials need more than SKVQ_NOALLOC_SCRATCH_BYTES (that is,
 *     skvq_workspace_size(cfg, max_len_hint, n_splits) > SKVQ_NOALLOC_SCRATCH_BYTES) are refused with
 *     SKVQ_ERR_SCRATCH_LIMIT before anything is launched; ask for fewer splits or use the workspace variant.
 *   - The first call on each device looks up the array's device address (with that device current).  The CUDA
 *     runtime loads a library's device image lazily, so this first lookup is also the moment the image, and the
 *     array in it, is placed in that device's memory: on a device that is already full it fails with
 *     SKVQ_ERR_CUDA.  Make the first call on every device at start-up -- before the engine sizes its KV cache to
 *     the remaining memory, and outside any stream capture; later calls only launch kernels.
 *   - The looked-up address is kept until the process exits.  cudaDeviceReset() (or anything else that destroys
 *     the device's primary context) invalidates it; this entry point must not be used on that device afterwards.
 *   - All calls on a device share the one array, and it keeps whatever the last call left there.  Nothing
 *     needs clearing (a call writes every partial before it reads it), but two calls that overlap on the GPU
 *     -- different streams, no ordering between them -- race on it.  Keep them stream-ordered.
 */
#define SKVQ_NOALLOC_SCRATCH_BYTES (8u << 20)
int skvq_decode_attention_noalloc(const skvq_config *cfg, const skvq_cache *cache, const void *q, void *out,
                                  float sm_scale, int32_t max_len_hint, int32_t n_splits, void *cuda_stream);

/* ------------------------------------------------------------------------------------------------------------------
 * Rotary positions, and a paged 4-bit cache for serving engines: keys are rotated, reordered and quantized straight
 * into pages that sequences share and give back; attention takes any number of queries per sequence.
 *
 * Notation: T rows of new tokens packed back to back, sequence b owns rows [starts[b], starts[b+1]), n_b of them;
 * L_b = lens[b] counts the sequence's tokens INCLUDING those n_b, so the rows are its last n_b tokens and row i of
 * them is token (and position) L_b - n_b + i.  P = page_tokens, R = ring_tokens, W = window, D = head_dim, G =
 * group_size, ng = D/G.
 * The calls keep no state: lengths, page table and starts are the caller's device arrays, read on the device.
 * ------------------------------------------------------------------------------------------------------------------ */

/* Element types of k, v, q and outputs. */
#define SKVQ_F16 0
#define SKVQ_BF16 1
#define SKVQ_F32 2  /* skvq_rope_apply and skvq_rope_apply_axes only */

/* How the frequencies of a rotation are stretched for contexts longer than the model was trained on. */
#define SKVQ_ROPE_PLAIN 0  /* f_j = base^(-2j/rot_dim) */
#define SKVQ_ROPE_LINEAR 1 /* f_j / factor (position interpolation) */
#define SKVQ_ROPE_NTK 2    /* base * factor^(rot_dim/(rot_dim-2)) in place of base; rot_dim > 2 */
#define SKVQ_ROPE_YARN 3   /* f_j / factor where the pair turns fewer than `slow` times over original_positions, f_j where it
                              turns more than `fast` times, a linear mix in the number of turns between; amplitude 0.1 ln(factor) + 1 */
typedef struct skvq_rope_scaling {
    int32_t kind;               /* SKVQ_ROPE_* */
    int32_t original_positions; /* YARN: positions of the training context, >= 1 */
    double base;                /* > 1, e.g. 10000 */
    double factor;              /* >= 1; ignored by PLAIN */
    double fast, slow;          /* YARN: turns, fast > slow >= 0 (e.g. 32 and 1) */
} skvq_rope_scaling;

/* Frequencies f_j (radians per position), j = 0..rot_dim/2-1, and the amplitude that multiplies cos and sin.  Host only:
 * both outputs are host pointers.  rot_dim even, 2..256. */
int skvq_rope_frequencies(int32_t rot_dim, const skvq_rope_scaling *scaling, double *frequencies_host, double *amplitude_host);

/* The table a rotation reads: row p = {amplitude cos(p f_j), amplitude sin(p f_j)} for j = 0..n_freq-1, fp32, computed from
 * angles reduced in 64 bits (the angle of position 10^6 needs them); p = first_position .. first_position + n_positions - 1
 * land in rows 0 .. n_positions - 1 of `table`, so a table can be extended in place.
 *   frequencies_host  host double [n_freq], 1 <= n_freq <= 128 (any scheme; skvq_rope_frequencies has four)
 *   table             device float [n_positions][n_freq][2] */
int skvq_rope_table(const double *frequencies_host, int32_t n_freq, double amplitude, int64_t first_position,
                    int32_t n_positions, void *table, void *cuda_stream);

/* A rotation (host struct): the first rot_dim channels of a head, position p by row p of the table. */
typedef struct skvq_rope {
    const void *table;   /* device float [n_positions][rot_dim/2][2] {cos, sin}, 16-byte aligned */
    int32_t rot_dim;     /* even, 2..head_dim */
    int32_t interleaved; /* 0: pair j = channels (j, j + rot_dim/2); 1: pair j = channels (2j, 2j+1) */
    int32_t n_positions; /* rows of the table */
} skvq_rope;

/* One operand of skvq_rope_apply (host struct).  Strides are in elements, between tokens and between heads; the channels of
 * a head are contiguous.  x may be broadcast (a stride of 0); rows of y that share elements are refused.  y may be x itself (same
 * pointer and strides); other overlaps are not allowed. */
typedef struct skvq_rope_tensor {
    const void *x;
    void *y;
    int64_t x_token_stride, x_head_stride, y_token_stride, y_head_stride;
    int32_t n_heads;
} skvq_rope_tensor;

/*
 * Rotary positions of packed tokens, queries and keys in one launch:
 *   y1 = x1 c - x2 s,  y2 = x2 c + x1 s   for every pair, {c, s} = table[positions[t]][j];
 * fp32, each product rounded, then the sum, then once to the type; channels at or beyond rot_dim are copied.
 * inverse = 1 rotates back (s -> -s): the gradient of the rotation with respect to x, for an amplitude of 1 also its inverse.
 *   a, b        operands, e.g. queries and keys; b may be NULL
 *   positions   device int32 [n_tokens]; a token whose position is outside the table is not written and sets
 *               SKVQ_STATUS_BAD_POSITION
 *   head_dim    1..512, rot_dim <= head_dim;  dtype SKVQ_F16, SKVQ_BF16 or SKVQ_F32
 *   status      device int32 or NULL
 * x and y need the alignment of their type only (16-byte alignment and strides that are multiples of 16 bytes are faster).
 */
int skvq_rope_apply(const skvq_rope *rope, int32_t dtype, int32_t head_dim, const skvq_rope_tensor *a,
                    const skvq_rope_tensor *b, const int32_t *positions, int32_t n_tokens, int32_t inverse, int32_t *status,
                    void *cuda_stream);

/* Which axis of a position turns which pair (host struct): for tokens with several coordinates, e.g. time, height and width. */
typedef struct skvq_rope_axes {
    int32_t n_axes;    /* 1..4 */
    uint8_t axis[128]; /* axis of pair j, below n_axes, for j < rot_dim/2; any assignment (runs of pairs, taking turns, ...) */
} skvq_rope_axes;

/*
 * skvq_rope_apply for tokens with several positions each: pair j of token t turns by {c, s} = table[p][j], p the token's position
 * on axis[j].  All axes read the one table; its frequencies are the caller's (skvq_rope_table takes any list, so axes may begin at
 * the highest frequency each, or share one sequence of them).  With one axis this is skvq_rope_apply, bit for bit.
 * inverse = 1 is the gradient with respect to x.
 *   positions   device int32; token t's position on axis i is positions[i * axis_stride + t * token_stride] (strides in elements,
 *               any, 0 included).  A token with a position outside the table on any axis is not written and sets
 *               SKVQ_STATUS_BAD_POSITION
 *   rot_dim     at most 256; everything else as for skvq_rope_apply
 * For keys and queries whose positions are not their token numbers in the cache (images; sequences that skvq_paged_evict has
 * shortened): rotate here, then call skvq_paged_append and skvq_paged_attention without a rotation.
 */
int skvq_rope_apply_axes(const skvq_rope *rope, const skvq_rope_axes *axes, int32_t dtype, int32_t head_dim,
                         const skvq_rope_tensor *a, const skvq_rope_tensor *b, const int32_t *positions, int64_t axis_stride,
                         int64_t token_stride, int32_t n_tokens, int32_t inverse, int32_t *status, void *cuda_stream);

/* Shape of a paged cache (host struct). */
typedef struct skvq_paged_config {
    int32_t n_q_heads;   /* Hq, a multiple of Hkv, Hq/Hkv <= 16 */
    int32_t n_kv_heads;  /* Hkv */
    int32_t head_dim;    /* D: 64 or 128 */
    int32_t group_size;  /* G: 32, 64 or 128, <= D */
    int32_t window;      /* W >= 0 newest tokens of a sequence are attended unquantized */
    int32_t ring_tokens; /* R >= W rows per slot of the ring; R - W tokens can be taken back (lens lowered) without
                            touching what the window then needs */
    int32_t page_tokens; /* P: 16, 32, 64, 128 or 256 tokens per page */
    int32_t n_pages;     /* pages of the pool */
    int32_t n_slots;     /* slots of the ring (sequences that can be live at once) */
    int32_t dtype;       /* SKVQ_F16 or SKVQ_BF16: k, v, q, out and the ring */
} skvq_paged_config;

/*
 * The pool (host struct of device pointers), row-major:
 *   k_codes/v_codes  uint8  [n_pages][Hkv][P][D/2]    code j of a row in bits [4j, 4j+4) of its little-endian bit stream,
 *                                                     j counted in reordered order (the 4-bit rows of skvq_cache)
 *   k_meta/v_meta    half2  [n_pages][Hkv][P][ng]     {scale h, zero z}; value h*code + z
 *   k_win/v_win      dtype  [n_slots][Hkv][R][D]      ring; token t in row t % R, reordered order; may be NULL when W == 0
 *   reorder_k/_v     int32  [Hkv][D]                  stored[j] = source[idx[j]], rows are permutations; NULL = identity
 *   alpha_k/_v       float  [Hkv][ng]                 clip factors; NULL = 1
 *   status           int32  [1] or NULL               SKVQ_STATUS_* bits are OR-ed in
 * EVERY token is quantized into its page when it is appended, and the newest are kept in the ring as well: a page is
 * complete at any time (it can be shared, moved or kept for another request with the same prefix).  The ring is not: a
 * sequence that begins on kept pages, or comes back in another slot, says in skvq_paged_batch::ring_from where its slot's
 * rows begin.
 */
typedef struct skvq_paged_cache {
    void *k_codes, *v_codes;
    void *k_meta, *v_meta;
    void *k_win, *v_win;
    const int32_t *reorder_k, *reorder_v;
    const float *alpha_k, *alpha_v;
    int32_t *status;
} skvq_paged_cache;

/* The sequences of one step (host struct of device pointers and host bounds). */
typedef struct skvq_paged_batch {
    const int32_t *page_table; /* [n_seqs][max_pages]: token t of sequence b lives in page page_table[b][t / P] */
    const int32_t *lens;       /* [n_seqs] */
    const int32_t *starts;     /* [n_seqs + 1], non-decreasing; rows at or beyond starts[n_seqs] are left alone */
    const int32_t *slots;      /* [n_seqs] ring slot of every sequence, or NULL: sequence b uses slot b */
    int32_t n_seqs;            /* 1..2048 */
    int32_t max_pages;         /* row length of page_table */
    int32_t n_tokens;          /* T: rows that k, v, q and outputs have */
    int32_t max_new;           /* host upper bound on n_b; max_new * Hq/Hkv <= 2^30 */
    int32_t max_len;           /* host upper bound on lens[], <= max_pages * P and <= 2^30 */
    const int32_t *ring_from;  /* [n_seqs] or NULL: the slot's ring holds the sequence's tokens from ring_from[b] on -- the first
                                  token appended since the sequence has had this slot; older tokens of the window are read from
                                  their pages, quantized.  (After more than R - W tokens were taken back it is the longest length
                                  reached minus R.)  Values below 0 count as 0, values above L_b as L_b.  NULL: 0, every token of
                                  the window was appended to this slot, by this sequence */
} skvq_paged_batch;

/* Validate a paged configuration (host only). */
int skvq_check_paged_config(const skvq_paged_config *cfg);

/* Bytes of k_codes, v_codes, k_meta, v_meta, k_win, v_win (in that order) for cfg.  Host only. */
int skvq_paged_cache_sizes(const skvq_paged_config *cfg, size_t bytes_out[6]);

/*
 * Append the new tokens of every sequence: rotate the keys (rope != NULL; token t by row t of the table; the rotated key is
 * rounded to dtype), reorder, quantize each group, write the rows to their pages, and the last min(n_b, R) of them to the ring
 * as well.  The quantizer is that of skvq_quantize_append at 4 bits with fp16 parameters, but for the step's quotient:
 *   lo = alpha*min, hi = alpha*max, h = fp16((hi-lo) * fp32(1/15)), z = fp16(lo), code = clamp(rint((x - z)/h), 0, 15)
 * (the product with 1/15 is within one fp32 step of the quotient by 15; h == 0 -> code 0).
 *   k, v             dtype [T][Hkv][D]; k_stride/v_stride: elements between tokens (a multiple of 8, >= Hkv*D)
 * A sequence is skipped and SKVQ_STATUS_BAD_BATCH set when its starts are not 0 <= starts[b] <= starts[b+1] <= T, n_b exceeds
 * max_new or L_b, L_b exceeds max_len or the table's rows, or its slot is not in [0, n_slots); a token whose page-table entry is
 * not in [0, n_pages) is skipped and sets SKVQ_STATUS_BAD_PAGE.  Two tokens of one call must not share a page row, two sequences
 * with new tokens no slot.  Magnitudes above 65440 (and NaN) give unspecified rows: the parameters are
 * fp16, and the highest code's value can lie a rounding of 15 steps above the group's maximum, where fp16 ends.
 * Repeating a call with the same arguments gives the same cache.
 */
int skvq_paged_append(const skvq_paged_config *cfg, const skvq_paged_cache *cache, const skvq_paged_batch *batch,
                      const skvq_rope *rope, const void *k, const void *v, int64_t k_stride, int64_t v_stride, void *cuda_stream);

/*
 * The last n_b tokens of every sequence as values, channels back in source order: h*code + z in fp32, rounded to dtype; with
 * window = 1 those of the newest W tokens of a sequence that its ring holds (ring_from) come from the ring instead (what attention sees).  Keys come out rotated, as
 * they are held.  Rows of skipped sequences and tokens (see skvq_paged_append) are left alone.
 *   k, v             dtype [T][Hkv][D], token strides as for skvq_paged_append; either may be NULL
 */
int skvq_paged_read(const skvq_paged_config *cfg, const skvq_paged_cache *cache, const skvq_paged_batch *batch, int32_t window,
                    void *k, void *v, int64_t k_stride, int64_t v_stride, void *cuda_stream);

/* Options of one paged attention call (host struct). */
typedef struct skvq_paged_attn_args {
    float sm_scale;       /* softmax scale, e.g. 1/sqrt(D) */
    int32_t causal;       /* 1: row i of a sequence sees tokens 0 .. L_b - n_b + i; 0: all L_b tokens */
    int32_t n_splits;     /* 0: the library chooses; n > 0: about n pieces of the context per (sequence, KV head), for sequences with
                             at most 16 rows (new tokens * Hq/Hkv) per KV head */
    void *workspace;      /* device scratch of at least skvq_paged_workspace_size() bytes; may be NULL when that is 0 */
    size_t workspace_bytes;
} skvq_paged_attn_args;

/* Scratch bytes that skvq_paged_attention needs (depends on the host bounds in `batch`, not on the device arrays, and on the
 * GPU's SM count): partial results of (sequence, KV head) pairs that several CTAs share, and, where max_new * Hq/Hkv exceeds 16, the
 * rotated queries, T * Hq * (2 D + 4) bytes.  0 also for a step without new tokens (n_tokens or max_new 0) and on bad arguments.  Host only. */
size_t skvq_paged_workspace_size(const skvq_paged_config *cfg, const skvq_paged_batch *batch, int32_t n_splits);

/*
 * Attention of the new tokens' queries over the cache (append first: the cache then holds them):
 *   q' = rope(q) rounded to dtype (rope != NULL),  s_t = sm_scale sum_j q'_j K~[t][j],  p = softmax over the tokens the row sees,
 *   out_j = sum_t p_t V~[t][j]
 * The window is the sequence's: all rows of a call read the same W newest tokens of L_b unquantized, and what lies before those
 * quantized, even where a row's own W newest tokens reach further back.  So rows of a chunk, or of several drafted tokens, differ
 * by the quantization of those tokens from what single-token steps give.
 * K~, V~ as skvq_paged_read(window = 1) defines them, before its rounding to dtype; as operands of the tensor core they are rounded to
 * fp16 once (with at most 16 rows, n_b * Hq/Hkv, per KV head only V~ is), and so are the probabilities.  Scores, softmax statistics
 * and sums are fp32.
 * A row that sees no token (n_b > L_b, or L_b = 0) gives zeros and a log-sum-exp of -infinity.
 *   q, out           dtype [T][Hq][D], token strides in elements (multiples of 8, >= Hq*D)
 *   lse              float [T][Hq], natural logarithm of the softmax denominator of every row, or NULL
 * Waits inside are bounded: one that runs out (it never should) sets SKVQ_STATUS_COPY_TIMEOUT, and the rows that it concerns are NaN.
 * Skipped sequences (as for skvq_paged_append, except that n_b may exceed L_b): their rows are left alone.  Tokens behind a bad
 * page-table entry, those of the window too, are left out of the softmax and SKVQ_STATUS_BAD_PAGE is set.  Rows of the cache at or beyond L_b are never
 * used, whatever they hold.  A query that is not finite gives its own row NaN and no other.  Keys and values have to be finite,
 * at most 65440 (as for skvq_paged_append): one that is not can reach every row of its sequence, those that do not see it too.
 * The workspace is overwritten; calls sharing one must be stream-ordered.  out and lse must not overlap the inputs.
 */
int skvq_paged_attention(const skvq_paged_config *cfg, const skvq_paged_cache *cache, const skvq_paged_batch *batch,
                         const skvq_rope *rope, const void *q, int64_t q_stride, void *out, int64_t out_stride, void *lse,
                         const skvq_paged_attn_args *args, void *cuda_stream);

/* ------------------------------------------------------------------------------------------------------------------
 * Shrinking a paged cache by what attention looked at: every step adds the probabilities that its rows gave each token to the
 * token's weight (skvq_paged_weights, after skvq_paged_attention with an lse); when a sequence is too long, every KV head keeps
 * its oldest, its newest and its heaviest tokens (skvq_paged_evict).  Weights are the caller's: float [n_slots][Hkv][capacity],
 * token t of the sequence in slot s and KV head h at [s][h][t]; slots are those of the batch (without `slots` sequence b uses slot b).
 * After an eviction a token's number in the cache is no longer its position: rotate by positions with skvq_rope_apply_axes (or
 * skvq_rope_apply) and append and attend without a rotation.
 * ------------------------------------------------------------------------------------------------------------------ */

/* Options of one skvq_paged_weights call (host struct). */
typedef struct skvq_paged_weights_args {
    float sm_scale;       /* as for the attention that gave lse */
    int32_t causal;       /* the same */
    int32_t last;         /* 0: every new token's rows count; n > 0: those of a sequence's last n new tokens alone */
    int32_t capacity;     /* tokens per row of the weights, >= max_len */
    const float *weights; /* [n_slots][Hkv][capacity], or NULL: zeros */
    float *weights_out;   /* the same shape; may be `weights` itself, other overlaps are not allowed */
    void *workspace;      /* device scratch of at least skvq_paged_weights_workspace_size() bytes; may be NULL when that is 0 */
    size_t workspace_bytes;
} skvq_paged_weights_args;

/* Scratch bytes that skvq_paged_weights needs (from the host bounds in `batch`): the counted queries, rotated, in the tensor
 * core's layout.  0 without new tokens and on bad arguments.  Host only. */
size_t skvq_paged_weights_workspace_size(const skvq_paged_config *cfg, const skvq_paged_batch *batch, int32_t last);

/*
 * Attention weights of a step, added up per token and KV head:
 *   weights_out[s][h][t] = (t < L_b - n_b ? weights[s][h][t] : 0) + sum over the counted rows r of KV head h that see token t of
 *                          exp(sm_scale q'_r . K~_t - lse_r)
 * for t < L_b; entries at or beyond L_b are left alone, and a new token's old entry is not read (a slot needs no clearing).  q' and K~ are
 * those of skvq_paged_attention; here the keys are not rounded to fp16 (but for bf16 rows of the window below 2^-14, to 2^-25): scores
 * are fp32 sums.  With at most 16 rows per KV head they are sum_g h (q'.c) + sum_g z (sum q'), whose parts may be larger than the score; of a
 * code's product with an entry of q' what lies below 2^-17 of the row's largest entry is lost there (entries from 2^-7 of it on: nothing).
 * Rows: the Hq/Hkv query heads of KV head h for each counted token; row i of a sequence sees tokens as attention's `causal` says.  A row whose lse is not finite, or
 * whose query is not, adds nothing.  Sums are fp32, in an order that the batch's host bounds and lengths decide and that does not change
 * from run to run.
 *   q                dtype [T][Hq][D], token stride in elements (a multiple of 8, >= Hq*D), 16-byte aligned; not rotated when rope is
 *                    given, as for attention
 *   lse              float [T][Hq], as skvq_paged_attention wrote it
 * A sequence without new tokens is copied (nothing is done when weights_out is weights).  Skipped sequences (as for
 * skvq_paged_attention; here a slot outside [0, n_slots) always skips): their entries are left alone, SKVQ_STATUS_BAD_BATCH is set.  A token behind a bad page-table
 * entry gains nothing and sets SKVQ_STATUS_BAD_PAGE.  Values are not read (v_codes, v_meta and v_win must
 * point to buffers all the same, as for every call).
 * Two sequences of a call must not share a slot.  Waits inside are bounded: one that runs out (it never should) sets
 * SKVQ_STATUS_COPY_TIMEOUT, and the weights that it concerns are NaN.
 */
int skvq_paged_weights(const skvq_paged_config *cfg, const skvq_paged_cache *cache, const skvq_paged_batch *batch,
                       const skvq_rope *rope, const void *q, int64_t q_stride, const void *lse,
                       const skvq_paged_weights_args *args, void *cuda_stream);

/* Options of one skvq_paged_evict call (host struct of device pointers and host numbers). */
typedef struct skvq_paged_evict_args {
    int32_t keep;          /* tokens that a sequence has afterwards at most, >= 1 */
    int32_t first;         /* its oldest tokens that always stay, >= 0 */
    int32_t recent;        /* its newest tokens that always stay, >= window; first + recent <= keep */
    int32_t capacity;      /* tokens per row of the weights, >= max_len */
    const float *weights;  /* [n_slots][Hkv][capacity] */
    float *weights_out;    /* the same shape: the kept tokens' weights, in the destination slot; may be `weights` itself */
    const int32_t *page_table_out; /* [n_seqs][max_pages_out]: pages that receive the kept rows, or NULL: the batch's page table */
    int32_t max_pages_out;
    const int32_t *slots_out;      /* [n_seqs] ring and weight slots afterwards, or NULL: the batch's */
    int32_t *lens_out;             /* [n_seqs] lengths afterwards; may be the batch's lens */
    int32_t *ring_from_out;        /* [n_seqs] ring_from afterwards, or NULL; may be the batch's ring_from */
    int32_t *kept;                 /* [n_seqs][Hkv][keep]: the old number of every token, increasing; -1 behind the last */
    void *workspace;               /* device scratch of at least skvq_paged_evict_workspace_size() bytes */
    size_t workspace_bytes;
} skvq_paged_evict_args;

/* Scratch bytes that skvq_paged_evict needs.  0 on bad arguments.  Host only. */
size_t skvq_paged_evict_workspace_size(const skvq_paged_config *cfg, const skvq_paged_batch *batch);

/*
 * Shorten sequences to `keep` tokens.  Of a sequence with L_b > keep every KV head keeps tokens 0 .. first-1, the last `recent` ones, and
 * of those between them the keep - first - recent with the largest weights: at equal weights the lower token number, -0 equal to
 * +0, a weight that is not a number below all others.  The kept rows of keys, values and weights become tokens 0 .. keep-1, in the order they
 * had (heads differ in which tokens these are), and the ring's rows of the `recent` tokens follow (8192 rows are moved at most).  Sequences with L_b <= keep
 * stay as they are, and are copied where the destination is another.  What lies behind the new length, rows and weights, is left as it is.
 *   batch            page_table, lens, slots, ring_from, max_len; starts (may be NULL), n_tokens and max_new are not looked at
 * A destination page is the source's page of the same place in the table, or one that no sequence of the call reads; a destination slot is
 * the sequence's own or one that no sequence of the call has.  So pages that sequences share must not be shortened in place: give
 * page_table_out.  Pages behind the new length are the caller's to free.
 * Pass ring_from_out to later batches if ring_from was given or tokens may be taken back (it tells which tokens the ring still
 * holds); otherwise, since recent >= window, the ring holds what the window needs.
 * A sequence is skipped and SKVQ_STATUS_BAD_BATCH set when its length is not in [0, max_len] or a slot of it is not in [0, n_slots): it keeps its
 * length and ring_from, its kept numbers are -1.  A row whose source or destination page is not in [0, n_pages) is not moved and
 * sets SKVQ_STATUS_BAD_PAGE.  SKVQ_ERR_UNSUPPORTED for a window beyond 8192.
 */
int skvq_paged_evict(const skvq_paged_config *cfg, const skvq_paged_cache *cache, const skvq_paged_batch *batch,
                     const skvq_paged_evict_args *args, void *cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* SKVQ_H_ */
