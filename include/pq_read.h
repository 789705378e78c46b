/*
 * pq_read.h -- the reading step next to the search of pq_adc.h: what a language model does with the passages that a
 * search has found.  Four calls on the same context, stream and error rules as pq_adc.h, in the order of one step:
 *
 *   pq_kv_plan        block tables, positions and slots of a paged cache of keys and values, from the requests' lengths
 *   pq_kv_append      norm and position rotation of queries and keys, keys and values written into the cache
 *   pq_kv_attention   attention of the new tokens over the cache
 *   pq_sample_tokens  the next tokens, drawn from the logits with given random numbers
 *
 * All data pointers are device pointers.  None of the calls waits for the stream, unless their scratch memory has to
 * grow: pq_kv_plan (for more than 4096 requests), pq_kv_attention and pq_sample_tokens use a buffer of the context that is
 * theirs alone, grown on demand (a HIP graph that captured a call holds its address, which stays valid until a call that
 * needs more).
 * Requests that the plan refuses have the length -1: their tokens are not written and see nothing, and a plan that is given that
 * length refuses them again, so one step's kv_lens can be the next one's cached_lens.  What a refused request holds in the cache and
 * in its row of the table is left as it is; to try it again, give its length from before.
 */
#ifndef PQ_READ_H
#define PQ_READ_H

#include "pq_adc.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { PQ_ELEM_F32 = 0, PQ_ELEM_F16 = 1, PQ_ELEM_BF16 = 2 } pq_elem;

/* A paged cache of keys and values: nblocks blocks of block_size places, each with `heads` rows of dim elements.
 * Element x of head h at place s of block b is at keys[b * key_strides[0] + s * key_strides[1] + h * key_strides[2] + x]
 * (strides in elements, none negative), and likewise for the values.  Slot s of the cache is place s % block_size of
 * block s / block_size. */
typedef struct {
    void *keys, *values;
    int64_t key_strides[3], value_strides[3];
    int64_t nblocks;
    int block_size, heads, dim;
    pq_elem elem;
} pq_kv_cache;

/* Rows of dim elements, one for each token and head: row (t, h) starts at p + t * token_stride + h * head_stride
 * (strides in elements, none negative). */
typedef struct {
    const void *p;
    int64_t token_stride, head_stride;
} pq_heads;

/* Plan of one step.  Request r has cached_lens[r] tokens in the cache and brings new_lens[r] more (a negative number of new ones
 * counts as 0).  It needs the blocks that its new tokens begin, ceil((cached + new) / block_size) - ceil(cached / block_size) of
 * them; requests take theirs from free_blocks in order.  A request is refused if its cached length is negative or its blocks do not
 * fit its row of the table (then it needs none), if the free blocks are used up by its own and the earlier ones' needs (of these
 * all count, refused ones' too, so behind a request that found too few blocks all are refused, also those that need none: put
 * first what must go on), or if its tokens end behind row ntokens of the outputs.
 *   new_lens, cached_lens [nreq] i32; block_tables [nreq][width] i32, in and out: the entries of the cached blocks are
 *   read, those of the fresh blocks written, the others left; free_blocks [nfree] i32
 *   -> cu_new [nreq+1] i32 = sums of the new lengths of the requests before (2^31-1 where they pass it);
 *      kv_lens [nreq] i32 = cached + new, -1 for a refused request;
 *      positions [ntokens] i32 and slots [ntokens] i64 of the new tokens, request after request, -1 for those of refused
 *      requests and for rows behind the last token; taken [1] i32 = number of blocks taken from free_blocks.
 * Results and block_tables must overlap neither each other nor the other inputs (kv_lens is not cached_lens updated in place).
 * Requires width * block_size < 2^31, ntokens < 2^31. */
int pq_kv_plan(pq_ctx *ctx, const int32_t *new_lens, const int32_t *cached_lens, int nreq, int32_t *block_tables, int width,
               const int32_t *free_blocks, int nfree, int block_size, int64_t ntokens, int32_t *cu_new, int32_t *kv_lens,
               int32_t *positions, int64_t *slots, int32_t *taken);

/* Queries, keys and values of ntokens tokens, in cache->elem.  With norm != 0 every query and key head x becomes
 * x / sqrt(mean(x^2) + eps) * weight (q_weight, k_weight [dim] f32; NULL: ones).  Then the first rot dimensions are rotated
 * by the token's position p: the pair (a, b) becomes (a cos - b sin, a sin + b cos) with entry i of row p of the tables
 * cos, sin [max_positions][rot/2] f32, where (a, b) are dimensions (i, i + rot/2), or (2i, 2i+1) with pairs != 0.
 * rot = 0: no rotation (tables may be NULL).  Computed in fp32, rounded once.
 *   q -> q_out [ntokens][q_heads][dim], k and v -> the cache at slots[t].
 * q_heads = 0: keys and values only (q, q_out may be NULL).  A token whose position is not in 0 .. max_positions-1 (any
 * negative one if rot = 0) has zeros in q_out and is not written to the cache; nor is one whose slot is not in the cache.
 * Two tokens with one slot: either may remain.  Requires dim and rot even, rot <= dim <= 1024. */
int pq_kv_append(pq_ctx *ctx, const pq_kv_cache *cache, const pq_heads *q, int q_heads, const pq_heads *k, const pq_heads *v,
                 int64_t ntokens, const int32_t *positions, const int64_t *slots, const float *cos_table, const float *sin_table,
                 int64_t max_positions, int rot, int pairs, int norm, const float *q_weight, const float *k_weight, float eps,
                 void *q_out);

/* Attention of the new tokens of nreq requests over a paged cache that already holds them.  Request r owns rows
 * cu_new[r] .. cu_new[r+1]-1 of the queries; its keys are at positions 0 .. kv_lens[r]-1, position j in block
 * block_tables[r][j / block_size]; its new tokens are the last of them, and each sees the keys up to itself, with
 * window > 0 only the last `window` of these.  Query head h reads head h / (q_heads / cache->heads) of the cache.
 *   out[t][h] = sum_j softmax_j(scale * q . k_j) v_j,  lse[t][h] = log sum_j exp(scale * q . k_j)  over the keys seen.
 *   q rows in cache->elem; out [ntokens][q_heads][dim] in cache->elem; lse [ntokens][q_heads] f32, may be NULL.
 * A row that sees nothing (a refused request, kv_lens below the number of new tokens) is 0, its lse -inf.  Rows behind
 * cu_new[nreq] are left.  max_new: the largest number of new tokens of a request (rows of a request behind it are not
 * written).  Keys behind the last position of the table are not seen.  Keys and values that no row sees may hold anything,
 * NaN included, and inf and NaN among values reach only the rows that see them.  Products of f16 and bf16 are summed in fp32
 * on the matrix cores, softmax statistics are fp32, the weights are rounded to the cache's type for the product with the
 * values.  With block numbers outside the cache among those of a request's keys its rows are unspecified (nothing outside the
 * cache is read).
 * Requires q_heads a multiple of cache->heads, width * block_size < 2^31 - 4096.  dim 64, 96, 128 or 256 in f16 or bf16, with
 * rows of the queries, the cache and out on 16 bytes, takes the matrix cores, any other even dim <= 512 and f32 a general
 * kernel. */
int pq_kv_attention(pq_ctx *ctx, const pq_kv_cache *cache, const pq_heads *q, int q_heads, int64_t ntokens,
                    const int32_t *cu_new, const int32_t *kv_lens, int nreq, const int32_t *block_tables, int width, int max_new,
                    float scale, int window, void *out, float *lse);

/* One token for each row of logits.  With x_i = (l_i - max l) / temperature and w_i = exp(x_i), tokens in order of falling
 * logit (equal ones: the smaller index first), a token stays if
 *   - it is among the first top_k                                        (top_k <= 0: all),
 *   - the weights before it sum to less than top_p * those of the first top_k  (top_p >= 1: all),
 *   - w_i >= min_p                                                         (min_p <= 0: all);
 * the first token always stays.  The token drawn is the one of those that stay with the largest
 * x_i - log(-log(noise_i)), ties to the smaller index: for noise uniform in (0, 1) a draw from their softmax.  Temperature
 * <= 0, or noise NULL: the token of the largest logit.
 *   logits [rows] rows of vocab elements at row_stride, noise likewise f32; temperature, top_p, min_p [rows] f32, top_k
 *   [rows] i32, each may be NULL (1, all, all, all)
 *   -> tokens [rows] i64; logprobs [rows] f32 = log of the token's share of the weights that stay (0 for temperature <= 0),
 *      may be NULL.
 * Logits of -inf and NaN are never drawn; a row that holds nothing else gives token -1, logprob -inf.  If some are +inf,
 * those share the weight.  Weights of less than 2^-60 of the largest may count as 0.  Requires vocab < 2^20. */
int pq_sample_tokens(pq_ctx *ctx, const void *logits, pq_elem elem, int64_t row_stride, int rows, int vocab, const float *noise,
                     int64_t noise_stride, const float *temperature, const int32_t *top_k, const float *top_p,
                     const float *min_p, int64_t *tokens, float *logprobs);

#ifdef __cplusplus
}
#endif
#endif /* PQ_READ_H */
