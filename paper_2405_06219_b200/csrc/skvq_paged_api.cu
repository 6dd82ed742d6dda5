// C-ABI entry points of the paged cache: argument validation and sizing.
#include "skvq_paged.cuh"

namespace skvq {
namespace {

int check_paged_cfg(const skvq_paged_config *c)
{
    if (!c) return SKVQ_ERR_INVALID_ARG;
    if (c->n_q_heads < 1 || c->n_kv_heads < 1 || c->window < 0 || c->ring_tokens < c->window || c->n_pages < 1 || c->n_slots < 1)
        return SKVQ_ERR_INVALID_ARG;
    if (c->head_dim != 64 && c->head_dim != 128) return SKVQ_ERR_UNSUPPORTED;
    if ((c->group_size != 32 && c->group_size != 64 && c->group_size != 128) || c->group_size > c->head_dim) return SKVQ_ERR_UNSUPPORTED;
    if (c->page_tokens != 16 && c->page_tokens != 32 && c->page_tokens != 64 && c->page_tokens != 128 && c->page_tokens != 256) return SKVQ_ERR_UNSUPPORTED;
    if (c->dtype != SKVQ_F16 && c->dtype != SKVQ_BF16) return SKVQ_ERR_UNSUPPORTED;
    if (c->n_q_heads % c->n_kv_heads != 0 || c->n_q_heads / c->n_kv_heads > 16 || c->n_kv_heads > 65535) return SKVQ_ERR_UNSUPPORTED;
    return SKVQ_OK;
}

bool off(const void *p, uintptr_t align) { return (reinterpret_cast<uintptr_t>(p) & (align - 1)) != 0; }

int check_pool(const skvq_paged_config *cfg, const skvq_paged_cache *c)
{
    if (!c || !c->k_codes || !c->v_codes || !c->k_meta || !c->v_meta) return SKVQ_ERR_INVALID_ARG;
    if (cfg->window > 0 && (!c->k_win || !c->v_win)) return SKVQ_ERR_INVALID_ARG;
    const void *ptrs[] = {c->k_codes, c->v_codes, c->k_meta, c->v_meta, c->k_win, c->v_win};
    for (const void *p : ptrs)
        if (off(p, 16)) return SKVQ_ERR_MISALIGNED;
    if (off(c->reorder_k, 4) || off(c->reorder_v, 4) || off(c->alpha_k, 4) || off(c->alpha_v, 4) || off(c->status, 4)) return SKVQ_ERR_MISALIGNED;
    return SKVQ_OK;
}

int check_batch(const skvq_paged_config *cfg, const skvq_paged_batch *b)
{
    if (!b || !b->page_table || !b->lens || !b->starts) return SKVQ_ERR_INVALID_ARG;
    if (b->n_seqs < 1 || b->max_pages < 1 || b->n_tokens < 0 || b->max_new < 0 || b->max_len < 0) return SKVQ_ERR_INVALID_ARG;
    if (b->n_seqs > kMaxPagedSeqs || b->max_len > kMaxPagedLen) return SKVQ_ERR_UNSUPPORTED;
    if ((int64_t)b->max_new * (cfg->n_q_heads / cfg->n_kv_heads) > (1 << 30)) return SKVQ_ERR_UNSUPPORTED;      // packed rows of a KV head
    if (b->max_len > (int64_t)b->max_pages * cfg->page_tokens) return SKVQ_ERR_CAPACITY;
    if (off(b->page_table, 4) || off(b->lens, 4) || off(b->starts, 4) || off(b->slots, 4) || off(b->ring_from, 4)) return SKVQ_ERR_MISALIGNED;
    if (!b->slots && cfg->window > 0 && b->n_seqs > cfg->n_slots) return SKVQ_ERR_CAPACITY;
    return SKVQ_OK;
}

int check_rope(const skvq_paged_config *cfg, const skvq_rope *r)
{
    if (!r) return SKVQ_OK;
    if (!r->table || r->n_positions < 0 || (r->interleaved != 0 && r->interleaved != 1)) return SKVQ_ERR_INVALID_ARG;
    if (r->rot_dim < 2 || (r->rot_dim & 1) || r->rot_dim > cfg->head_dim) return SKVQ_ERR_INVALID_ARG;
    if (off(r->table, 16)) return SKVQ_ERR_MISALIGNED;
    return SKVQ_OK;
}

int check_rows(const void *p, int64_t stride, int64_t least)
{
    if (stride < least) return SKVQ_ERR_INVALID_ARG;
    if (off(p, 16) || stride % 8 != 0) return SKVQ_ERR_MISALIGNED;
    return SKVQ_OK;
}

PagedArgs make_args(const skvq_paged_config *cfg, const skvq_paged_cache *cache, const skvq_paged_batch *batch, const skvq_rope *rope)
{
    PagedArgs a;
    a.cfg = *cfg;
    a.c = *cache;
    a.batch = *batch;
    a.rope = rope ? *rope : skvq_rope{};
    a.ng = cfg->head_dim / cfg->group_size;
    return a;
}

}  // namespace
}  // namespace skvq

using namespace skvq;

extern "C" {

int skvq_check_paged_config(const skvq_paged_config *cfg) { return check_paged_cfg(cfg); }

int skvq_paged_cache_sizes(const skvq_paged_config *cfg, size_t bytes_out[6])
{
    const int rc = check_paged_cfg(cfg);
    if (rc != SKVQ_OK) return rc;
    if (!bytes_out) return SKVQ_ERR_INVALID_ARG;
    const size_t rows = (size_t)cfg->n_pages * cfg->n_kv_heads * cfg->page_tokens;
    bytes_out[0] = bytes_out[1] = rows * (cfg->head_dim / 2);
    bytes_out[2] = bytes_out[3] = rows * (cfg->head_dim / cfg->group_size) * 4;
    bytes_out[4] = bytes_out[5] = cfg->window > 0 ? (size_t)cfg->n_slots * cfg->n_kv_heads * cfg->ring_tokens * cfg->head_dim * 2 : 0;
    return SKVQ_OK;
}

int skvq_paged_append(const skvq_paged_config *cfg, const skvq_paged_cache *cache, const skvq_paged_batch *batch,
                      const skvq_rope *rope, const void *k, const void *v, int64_t k_stride, int64_t v_stride, void *cuda_stream)
{
    int rc = check_paged_cfg(cfg);
    if (rc == SKVQ_OK) rc = check_pool(cfg, cache);
    if (rc == SKVQ_OK) rc = check_batch(cfg, batch);
    if (rc == SKVQ_OK) rc = check_rope(cfg, rope);
    if (rc != SKVQ_OK) return rc;
    if (batch->n_tokens == 0 || batch->max_new == 0) return SKVQ_OK;
    if (!k || !v) return SKVQ_ERR_INVALID_ARG;
    const int64_t least = (int64_t)cfg->n_kv_heads * cfg->head_dim;
    rc = check_rows(k, k_stride, least);
    if (rc == SKVQ_OK) rc = check_rows(v, v_stride, least);
    if (rc != SKVQ_OK) return rc;
    const cudaError_t e = launch_paged_append(make_args(cfg, cache, batch, rope), k, v, k_stride, v_stride, static_cast<cudaStream_t>(cuda_stream));
    return e == cudaSuccess ? SKVQ_OK : SKVQ_ERR_CUDA;
}

int skvq_paged_read(const skvq_paged_config *cfg, const skvq_paged_cache *cache, const skvq_paged_batch *batch, int32_t window,
                    void *k, void *v, int64_t k_stride, int64_t v_stride, void *cuda_stream)
{
    int rc = check_paged_cfg(cfg);
    if (rc == SKVQ_OK) rc = check_pool(cfg, cache);
    if (rc == SKVQ_OK) rc = check_batch(cfg, batch);
    if (rc != SKVQ_OK) return rc;
    if (window != 0 && window != 1) return SKVQ_ERR_INVALID_ARG;
    if (batch->n_tokens == 0 || batch->max_new == 0 || (!k && !v)) return SKVQ_OK;
    const int64_t least = (int64_t)cfg->n_kv_heads * cfg->head_dim;
    if (k) rc = check_rows(k, k_stride, least);
    if (rc == SKVQ_OK && v) rc = check_rows(v, v_stride, least);
    if (rc != SKVQ_OK) return rc;
    const cudaError_t e = launch_paged_read(make_args(cfg, cache, batch, nullptr), window, k, v, k_stride, v_stride, static_cast<cudaStream_t>(cuda_stream));
    return e == cudaSuccess ? SKVQ_OK : SKVQ_ERR_CUDA;
}

size_t skvq_paged_workspace_size(const skvq_paged_config *cfg, const skvq_paged_batch *batch, int32_t n_splits)
{
    if (check_paged_cfg(cfg) != SKVQ_OK || !batch || batch->n_seqs < 1 || batch->n_seqs > kMaxPagedSeqs || batch->max_new < 1 ||
        batch->n_tokens < 1 || batch->max_len < 0 || batch->max_len > kMaxPagedLen || n_splits < 0)
        return 0;
    return paged_workspace_bytes(*cfg, *batch, n_splits);
}

int skvq_paged_attention(const skvq_paged_config *cfg, const skvq_paged_cache *cache, const skvq_paged_batch *batch,
                         const skvq_rope *rope, const void *q, int64_t q_stride, void *out, int64_t out_stride, void *lse,
                         const skvq_paged_attn_args *args, void *cuda_stream)
{
    int rc = check_paged_cfg(cfg);
    if (rc == SKVQ_OK) rc = check_pool(cfg, cache);
    if (rc == SKVQ_OK) rc = check_batch(cfg, batch);
    if (rc == SKVQ_OK) rc = check_rope(cfg, rope);
    if (rc != SKVQ_OK) return rc;
    if (!args || args->n_splits < 0 || (args->causal != 0 && args->causal != 1)) return SKVQ_ERR_INVALID_ARG;
    if (batch->n_tokens == 0 || batch->max_new == 0) return SKVQ_OK;
    if (!q || !out) return SKVQ_ERR_INVALID_ARG;
    const int64_t least = (int64_t)cfg->n_q_heads * cfg->head_dim;
    rc = check_rows(q, q_stride, least);
    if (rc == SKVQ_OK) rc = check_rows(out, out_stride, least);
    if (rc != SKVQ_OK) return rc;
    if (off(lse, 4) || off(args->workspace, 16)) return SKVQ_ERR_MISALIGNED;
    const size_t need = paged_workspace_bytes(*cfg, *batch, args->n_splits);
    if (need && (!args->workspace || args->workspace_bytes < need)) return SKVQ_ERR_WORKSPACE;
    PagedAttnArgs a;
    a.p = make_args(cfg, cache, batch, rope);
    a.q = q;
    a.out = out;
    a.lse = static_cast<float *>(lse);
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    a.sm_scale = args->sm_scale;
    a.causal = args->causal;
    a.n_splits = args->n_splits;
    a.ws = static_cast<float *>(args->workspace);
    const cudaError_t e = launch_paged_attention(a, static_cast<cudaStream_t>(cuda_stream));
    return e == cudaSuccess ? SKVQ_OK : SKVQ_ERR_CUDA;
}

}  // extern "C"
