// Attention of new tokens over a paged cache (pq_kv_attention).
#include "kv_attention.h"

namespace pq {

// ---- any type and layout ------------------------------------------------------------------------------
//
// One block per row.  Each wave takes 64 keys at a time: a lane forms the product with one key, the wave updates the running
// maximum and sum, then the lanes hold the dimensions and add up the weighted values.  The four waves' results are joined
// at the end.  Keys are read by one lane each and no row shares what another one reads: simple, not fast.  It is
// for f32 and for layouts and dimensions that the other kernels do not take; the products' operands stay fp32 there.  64 single
// tokens over up to 8192 keys, 32 heads of 128 dimensions on 8, bf16: 2.4 ms (kv_attention_few.h: 0.16); two chunks of 2048 over
// 14 336 keys: 183 ms (kv_attention_chunk.h: 0.69 to 0.73).
constexpr int GENERAL_WAVES = 4;
constexpr int GENERAL_DIM = 512;

template <class T> __global__ __launch_bounds__(64 * GENERAL_WAVES) void kv_attention_general_kernel(attention_args a) {
    __shared__ float q[GENERAL_DIM], acc[GENERAL_WAVES][GENERAL_DIM], stat[GENERAL_WAVES][2];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, dim = a.cache.dim;
    const int64_t t = blockIdx.x / a.q_heads;
    const int h = (int)(blockIdx.x - t * a.q_heads), kvh = h / (a.q_heads / a.cache.heads);
    const int r = attention_request(a.cu, a.nreq, t);
    if (r < 0 || t - a.cu[r] >= a.max_new) return;
    const int position = attention_length(a, r) - (a.cu[r + 1] - (int)t), at = min(position, attention_keys(a, r) - 1);
    const int from = a.window > 0 ? (int)max((int64_t)0, (int64_t)position - a.window + 1) : 0;
    const T *qrow = (const T *)a.q.p + t * a.q.token_stride + h * a.q.head_stride;
    for (int i = tid; i < dim; i += 64 * GENERAL_WAVES) q[i] = (float)qrow[i];
    for (int i = lane; i < dim; i += 64) acc[wave][i] = 0.f;
    __syncthreads();
    float top = -INFINITY, sum = 0.f, part[GENERAL_DIM / 64] = {};
    for (int base = from + wave * 64; base <= at; base += 64 * GENERAL_WAVES) {
        const int j = base + lane;
        float s = -INFINITY;
        int64_t block = 0;
        int place = 0;
        if (j <= at) {
            attention_place(a, r, j, block, place);
            const T *k = (const T *)a.cache.keys + block * a.cache.key_strides[0] + place * a.cache.key_strides[1] + kvh * a.cache.key_strides[2];
            s = 0.f;
            for (int i = 0; i < dim; ++i) s += q[i] * (float)k[i];
            s *= a.scale_log2;
        }
        float high = s;
        for (int d = 32; d > 0; d /= 2) high = fmaxf(high, __shfl_xor(high, d));
        high = fmaxf(high, top);
        // (all weights so far zero, as by products of -inf: nothing to scale, and -inf - -inf is not formed)
        const float ref = high == -INFINITY ? 0.f : high;
        const float shrink = exp2f(top - ref), w = exp2f(s - ref);
        top = high;
        sum = sum * shrink + w;
        const int64_t row = block * a.cache.value_strides[0] + place * a.cache.value_strides[1];
        for (int e = 0; e < GENERAL_DIM / 64; ++e) part[e] *= shrink;
        const int count = min(64, at - base + 1);
        for (int l = 0; l < count; ++l) {
            const float wl = __shfl(w, l);
            const T *v = (const T *)a.cache.values + __shfl((long long)row, l) + kvh * a.cache.value_strides[2];
#pragma unroll
            for (int e = 0; e < GENERAL_DIM / 64; ++e)
                if (e * 64 + lane < dim) part[e] += wl * (float)v[e * 64 + lane];
        }
    }
    for (int d = 32; d > 0; d /= 2) sum += __shfl_xor(sum, d);
#pragma unroll
    for (int e = 0; e < GENERAL_DIM / 64; ++e)
        if (e * 64 + lane < dim) acc[wave][e * 64 + lane] = part[e];
    if (lane == 0) {
        stat[wave][0] = top;
        stat[wave][1] = sum;
    }
    __syncthreads();
    float all = -INFINITY, total = 0.f, share[GENERAL_WAVES];
    for (int w = 0; w < GENERAL_WAVES; ++w) all = fmaxf(all, stat[w][0]);
    const float ref = all == -INFINITY ? 0.f : all;
    for (int w = 0; w < GENERAL_WAVES; ++w) {
        share[w] = exp2f(stat[w][0] - ref);
        total += share[w] * stat[w][1];
    }
    T *out = (T *)a.out + (t * a.q_heads + h) * dim;
    for (int i = tid; i < dim; i += 64 * GENERAL_WAVES) {
        float o = 0.f;
        for (int w = 0; w < GENERAL_WAVES; ++w) o += share[w] * acc[w][i];
        out[i] = (T)(total != 0.f ? o / total : 0.f);
    }
    if (tid == 0 && a.lse) a.lse[t * a.q_heads + h] = total != 0.f ? (ref + log2f(total)) * LN2 : -INFINITY;
}

// rows of 16-bit elements that 16-byte accesses fit, in the dimensions that are built
static bool attention_on_matrix_cores(const attention_args &a) {
    const pq_kv_cache &c = a.cache;
    if (c.elem == PQ_ELEM_F32 || (c.dim != 64 && c.dim != 96 && c.dim != 128 && c.dim != 256)) return false;
    uint64_t bits = (uint64_t)(uintptr_t)c.keys | (uint64_t)(uintptr_t)c.values | (uint64_t)(uintptr_t)a.q.p | (uint64_t)(uintptr_t)a.out;
    for (int i = 0; i < 3; ++i) bits |= (uint64_t)(c.key_strides[i] | c.value_strides[i]) * 2;
    // (strides of blocks and places are multiplied in 32 bits)
    for (int i = 0; i < 2; ++i)
        if (c.key_strides[i] > INT_MAX || c.value_strides[i] > INT_MAX) return false;
    bits |= (uint64_t)(a.q.token_stride | a.q.head_stride) * 2;
    return bits % 16 == 0;
}

int launch_kv_attention(pq_ctx *ctx, const pq_kv_cache *cache, const pq_heads *q, int q_heads, int64_t ntokens,
                        const int32_t *cu_new, const int32_t *kv_lens, int nreq, const int32_t *block_tables, int width,
                        int max_new, float scale, int window, void *out, float *lse) {
    attention_args a = {};
    a.cache = *cache;
    a.q = *q;
    a.cu = cu_new;
    a.kv_lens = kv_lens;
    a.tables = block_tables;
    a.out = out;
    a.lse = lse;
    a.ntokens = ntokens;
    a.q_heads = q_heads;
    a.nreq = nreq;
    a.width = width;
    a.window = window;
    a.max_new = max_new;
    a.group = q_heads / cache->heads;
    a.by_block = fast_div((uint32_t)cache->block_size);
    a.by_group = fast_div((uint32_t)a.group);
    a.scale_log2 = scale * 1.4426950408889634f;
    if (attention_on_matrix_cores(a)) {
        for (int i = 0; i < 2; ++i) {
            a.k_strides[i] = (uint32_t)cache->key_strides[i];
            a.v_strides[i] = (uint32_t)cache->value_strides[i];
        }
        // Requests of few rows and others in one call: over long contexts each kind has blocks of its own, as keys and values are
        // read faster by those of few rows; over short ones what counts is one launch of one kind (64 requests of 1 to 50 tokens,
        // 4 heads on each of 8, up to 8000 keys: 237 us, all as chunks 252 us; 23 requests of 1 to 100 tokens, 16 heads, up to 700
        // keys: 24 and 19 us).  Where all requests have max_new tokens there is one kind only.
        const int64_t most_rows = (int64_t)max_new * a.group, held = (int64_t)width * cache->block_size;
        // (64 single tokens over up to 8192 keys, 4 heads on each of 8: 164 us, as chunks 233.  One token over 131 038 keys is the call
        // that chunks serve faster, 109 us for 115: how many of a call's requests are as long is known on the GPU only, and a wrong
        // guess costs more than that.)
        if (most_rows <= FEW_ROWS) return launch_kv_attention_few(ctx, a, (int)most_rows);
        const bool is_long = held >= 4096 && (window == 0 || window >= 4096);
        return launch_kv_attention_chunk(ctx, a, is_long && a.group <= FEW_ROWS && ntokens < (int64_t)nreq * max_new);
    }
    const int64_t grid = ntokens * q_heads;
    if (grid > INT_MAX) return fail(ctx, PQ_EUNSUPPORTED, "kv_attention: %lld rows in one call", (long long)grid);
    if (cache->elem == PQ_ELEM_F32) kv_attention_general_kernel<float><<<(int)grid, 64 * GENERAL_WAVES, 0, ctx->stream>>>(a);
    else if (cache->elem == PQ_ELEM_F16) kv_attention_general_kernel<_Float16><<<(int)grid, 64 * GENERAL_WAVES, 0, ctx->stream>>>(a);
    else kv_attention_general_kernel<__bf16><<<(int)grid, 64 * GENERAL_WAVES, 0, ctx->stream>>>(a);
    PQ_HIP(ctx, hipGetLastError());
    return PQ_OK;
}

}  // namespace pq
