// C-ABI entry points of the reading step (pq_read.h): argument validation.
#include <limits.h>
#include <math.h>

#include "elem.h"
#include "pq_internal.h"

using namespace pq;

namespace {

int check_elem(pq_ctx *ctx, const char *who, int elem) {
    if (elem != PQ_ELEM_F32 && elem != PQ_ELEM_F16 && elem != PQ_ELEM_BF16) return fail(ctx, PQ_EINVAL, "%s: bad element type %d", who, elem);
    return PQ_OK;
}

bool aligned_to(const void *p, size_t bytes) { return (uintptr_t)p % bytes == 0; }

int check_cache(pq_ctx *ctx, const char *who, const pq_kv_cache *c, int most_dim) {
    if (!c) return fail(ctx, PQ_EINVAL, "%s: null cache", who);
    if (const int rc = check_elem(ctx, who, c->elem)) return rc;
    if (c->nblocks < 0 || c->block_size <= 0 || c->heads <= 0 || c->dim <= 0) return fail(ctx, PQ_EINVAL, "%s: sizes of the cache must be positive", who);
    if (c->nblocks > INT_MAX) return fail(ctx, PQ_EUNSUPPORTED, "%s: %lld blocks in the cache", who, (long long)c->nblocks);
    if (c->dim % 2 != 0 || c->dim > most_dim) return fail(ctx, PQ_EUNSUPPORTED, "%s: dim=%d: even, up to %d", who, c->dim, most_dim);
    if (!c->keys || !c->values) return fail(ctx, PQ_EINVAL, "%s: null cache", who);
    const size_t e = elem_bytes(c->elem);
    if (!aligned_to(c->keys, e) || !aligned_to(c->values, e)) return fail(ctx, PQ_EINVAL, "%s: the cache is not aligned to its elements", who);
    for (int i = 0; i < 3; ++i)
        if (c->key_strides[i] < 0 || c->value_strides[i] < 0) return fail(ctx, PQ_EINVAL, "%s: strides must not be negative", who);
    return PQ_OK;
}

int check_heads(pq_ctx *ctx, const char *who, const char *what, const pq_heads *h, size_t e) {
    if (!h || !h->p) return fail(ctx, PQ_EINVAL, "%s: null %s", who, what);
    if (h->token_stride < 0 || h->head_stride < 0) return fail(ctx, PQ_EINVAL, "%s: strides must not be negative", who);
    if (!aligned_to(h->p, e)) return fail(ctx, PQ_EINVAL, "%s: %s is not aligned to its elements", who, what);
    return PQ_OK;
}

// memory that a call takes
struct span {
    const void *p;
    size_t bytes;
};
bool overlap(const span &a, const span &b) {
    return a.bytes > 0 && b.bytes > 0 && (uintptr_t)a.p < (uintptr_t)b.p + b.bytes && (uintptr_t)b.p < (uintptr_t)a.p + a.bytes;
}

}  // namespace

extern "C" {

int pq_kv_plan(pq_ctx *ctx, const int32_t *new_lens, const int32_t *cached_lens, int nreq, int32_t *block_tables, int width,
               const int32_t *free_blocks, int nfree, int block_size, int64_t ntokens, int32_t *cu_new, int32_t *kv_lens,
               int32_t *positions, int64_t *slots, int32_t *taken) {
    if (!ctx) return PQ_EINVAL;
    if (nreq < 0 || width < 0 || nfree < 0 || block_size <= 0 || ntokens < 0) return fail(ctx, PQ_EINVAL, "kv_plan: bad size");
    if ((int64_t)width * block_size > INT_MAX) return fail(ctx, PQ_EUNSUPPORTED, "kv_plan: width * block_size must be below 2^31");
    if (ntokens > INT_MAX) return fail(ctx, PQ_EUNSUPPORTED, "kv_plan: ntokens must be below 2^31");
    if (!cu_new || !taken || (nreq > 0 && (!new_lens || !cached_lens || !kv_lens)) || (nreq > 0 && width > 0 && !block_tables) ||
        (nfree > 0 && !free_blocks) || (ntokens > 0 && (!positions || !slots)))
        return fail(ctx, PQ_EINVAL, "kv_plan: null pointer");
    // (all blocks of the kernel read the lengths while others already write results; what is only read comes last)
    const size_t n = (size_t)nreq, t = (size_t)ntokens;
    const span spans[] = {{cu_new, 4 * (n + 1)}, {kv_lens, 4 * n},  {positions, 4 * t},   {slots, 8 * t},          {taken, 4},
                          {block_tables, 4 * n * (size_t)width},   {new_lens, 4 * n}, {cached_lens, 4 * n}, {free_blocks, 4 * (size_t)nfree}};
    for (int i = 0; i < 6; ++i)
        for (int j = i + 1; j < 9; ++j)
            if (overlap(spans[i], spans[j])) return fail(ctx, PQ_EINVAL, "kv_plan: results overlap each other or what is read");
    return launch_kv_plan(ctx, new_lens, cached_lens, nreq, block_tables, width, free_blocks, nfree, block_size, ntokens, cu_new, kv_lens,
                          positions, slots, taken);
}

int pq_kv_append(pq_ctx *ctx, const pq_kv_cache *cache, const pq_heads *q, int q_heads, const pq_heads *k, const pq_heads *v,
                 int64_t ntokens, const int32_t *positions, const int64_t *slots, const float *cos_table, const float *sin_table,
                 int64_t max_positions, int rot, int pairs, int norm, const float *q_weight, const float *k_weight, float eps,
                 void *q_out) {
    if (!ctx) return PQ_EINVAL;
    if (const int rc = check_cache(ctx, "kv_append", cache, 1024)) return rc;
    if (q_heads < 0 || ntokens < 0 || rot < 0 || max_positions < 0) return fail(ctx, PQ_EINVAL, "kv_append: bad size");
    if (rot % 2 != 0 || rot > cache->dim) return fail(ctx, PQ_ESHAPE, "kv_append: rot=%d of dim=%d", rot, cache->dim);
    if (!(eps >= 0.f)) return fail(ctx, PQ_EINVAL, "kv_append: eps must not be negative");
    if (ntokens == 0) return PQ_OK;
    const size_t e = elem_bytes(cache->elem);
    if (const int rc = check_heads(ctx, "kv_append", "keys", k, e)) return rc;
    if (const int rc = check_heads(ctx, "kv_append", "values", v, e)) return rc;
    if (q_heads > 0) {
        if (const int rc = check_heads(ctx, "kv_append", "queries", q, e)) return rc;
        if (!q_out || !aligned_to(q_out, e)) return fail(ctx, PQ_EINVAL, "kv_append: bad q_out");
    }
    if (!positions || !slots || (rot > 0 && (!cos_table || !sin_table))) return fail(ctx, PQ_EINVAL, "kv_append: null pointer");
    return launch_kv_append(ctx, cache, q, q_heads, k, v, ntokens, positions, slots, cos_table, sin_table, max_positions, rot, pairs, norm,
                            q_weight, k_weight, eps, q_out);
}

int pq_kv_attention(pq_ctx *ctx, const pq_kv_cache *cache, const pq_heads *q, int q_heads, int64_t ntokens,
                    const int32_t *cu_new, const int32_t *kv_lens, int nreq, const int32_t *block_tables, int width, int max_new,
                    float scale, int window, void *out, float *lse) {
    if (!ctx) return PQ_EINVAL;
    if (const int rc = check_cache(ctx, "kv_attention", cache, 512)) return rc;
    if (q_heads <= 0 || ntokens < 0 || nreq < 0 || width < 0 || max_new < 0 || window < 0) return fail(ctx, PQ_EINVAL, "kv_attention: bad size");
    if (q_heads % cache->heads != 0)
        return fail(ctx, PQ_ESHAPE, "kv_attention: %d query heads are no multiple of the cache's %d", q_heads, cache->heads);
    // (the kernels look some tiles of keys ahead)
    if ((int64_t)width * cache->block_size > INT_MAX - 4096) return fail(ctx, PQ_EUNSUPPORTED, "kv_attention: width * block_size must be below 2^31 - 4096");
    if ((int64_t)nreq * cache->heads > INT_MAX) return fail(ctx, PQ_EUNSUPPORTED, "kv_attention: %d requests in one call", nreq);
    if (ntokens > INT_MAX) return fail(ctx, PQ_EUNSUPPORTED, "kv_attention: ntokens must be below 2^31");
    if (!isfinite(scale)) return fail(ctx, PQ_EINVAL, "kv_attention: scale must be finite");
    if (ntokens == 0 || nreq == 0 || max_new == 0) return PQ_OK;
    const size_t e = elem_bytes(cache->elem);
    if (const int rc = check_heads(ctx, "kv_attention", "queries", q, e)) return rc;
    if (!cu_new || !kv_lens || !out || (width > 0 && !block_tables)) return fail(ctx, PQ_EINVAL, "kv_attention: null pointer");
    if (!aligned_to(out, e)) return fail(ctx, PQ_EINVAL, "kv_attention: out is not aligned to its elements");
    if (width == 0 || cache->nblocks == 0) return fail(ctx, PQ_ESHAPE, "kv_attention: no blocks to read from");
    return launch_kv_attention(ctx, cache, q, q_heads, ntokens, cu_new, kv_lens, nreq, block_tables, width, max_new, scale, window, out, lse);
}

int pq_sample_tokens(pq_ctx *ctx, const void *logits, pq_elem elem, int64_t row_stride, int rows, int vocab, const float *noise,
                     int64_t noise_stride, const float *temperature, const int32_t *top_k, const float *top_p,
                     const float *min_p, int64_t *tokens, float *logprobs) {
    if (!ctx) return PQ_EINVAL;
    if (const int rc = check_elem(ctx, "sample_tokens", elem)) return rc;
    if (rows < 0 || vocab <= 0 || row_stride < 0 || noise_stride < 0) return fail(ctx, PQ_EINVAL, "sample_tokens: bad size");
    if (vocab >= 1 << 20) return fail(ctx, PQ_EUNSUPPORTED, "sample_tokens: vocab=%d not below 2^20", vocab);
    if (rows == 0) return PQ_OK;
    if (!logits || !tokens) return fail(ctx, PQ_EINVAL, "sample_tokens: null pointer");
    if (!aligned_to(logits, elem_bytes(elem))) return fail(ctx, PQ_EINVAL, "sample_tokens: logits are not aligned to their elements");
    if (!aligned_to(noise, 4)) return fail(ctx, PQ_EINVAL, "sample_tokens: noise is not aligned to its elements");
    return launch_sample_tokens(ctx, logits, elem, row_stride, rows, vocab, noise, noise_stride, temperature, top_k, top_p, min_p, tokens,
                                logprobs);
}

}  // extern "C"
