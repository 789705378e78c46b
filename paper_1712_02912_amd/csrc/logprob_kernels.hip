// Log-probabilities of given tokens, their ranks, the entropy and the likeliest tokens (pq_token_logprobs).
#include "elem.h"
#include "pq_internal.h"

namespace pq {

constexpr int LOGPROB_THREADS = 256;

struct logprob_args {
    const void *logits;
    const int64_t *tokens;
    float *logprobs, *entropy, *top_logprobs;
    int32_t *ranks;
    int64_t *top_tokens;
    int64_t row_stride;
    int rows, vocab, top;
};

// A logit as its order counts it: NaN as -inf, one zero.
template <class T> __device__ __forceinline__ float logit_of(T v) { return fmaxf((float)v, -INFINITY) + 0.f; }
// One whole number for each token of a row, in the order of its logits, of equal ones the smaller index first; 0 is none.
__device__ __forceinline__ uint64_t order_key(float v, int i) {
    const uint32_t b = __builtin_bit_cast(uint32_t, v);
    return (uint64_t)(b >> 31 ? ~b : b | 0x80000000u) << 20 | (uint32_t)((1 << 20) - 1 - i);
}
__device__ __forceinline__ int key_token(uint64_t key) { return (1 << 20) - 1 - (int)(key & ((1 << 20) - 1)); }
__device__ __forceinline__ float key_logit(uint64_t key) {
    const uint32_t b = (uint32_t)(key >> 20);
    return __builtin_bit_cast(float, b >> 31 ? b & 0x7fffffffu : ~b);
}

template <class V, class F> __device__ __forceinline__ V block_join(V v, F f) {
    __shared__ V parts[LOGPROB_THREADS / 64];
    for (int d = 32; d > 0; d /= 2) v = f(v, (V)__shfl_xor(v, d));
    if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = v;
    __syncthreads();
    v = parts[0];
    for (int w = 1; w < LOGPROB_THREADS / 64; ++w) v = f(v, parts[w]);
    __syncthreads();
    return v;
}

// One block for each row, which reads it for the maximum, for the sums, and for every token that is listed.
template <class T> __global__ __launch_bounds__(LOGPROB_THREADS) void token_logprobs_kernel(logprob_args a) {
    const int64_t r = blockIdx.x;
    const int tid = threadIdx.x;
    const T *const row = (const T *)a.logits + r * a.row_stride;
    auto most = [](auto x, auto y) { return x > y ? x : y; };
    auto plus = [](auto x, auto y) { return x + y; };
    const int64_t token = a.tokens ? a.tokens[r] : -1;
    const bool given = token >= 0 && token < a.vocab;
    const uint64_t chosen = given ? order_key(logit_of(row[token]), (int)token) : ~0ull;
    float high = -INFINITY;
    int before = 0;
    for (int i = tid; i < a.vocab; i += LOGPROB_THREADS) {
        const float v = logit_of(row[i]);
        high = fmaxf(high, v);
        before += order_key(v, i) > chosen;
    }
    high = block_join(high, most);
    before = block_join(before, plus);
    // distance from the maximum; where that is infinite, 0 for those that are it
    auto below = [&](float v) { return v == high ? 0.f : v - high; };
    float sum = 0.f, moment = 0.f;
    for (int i = tid; i < a.vocab; i += LOGPROB_THREADS) {
        const float d = below(logit_of(row[i])), w = expf(d);
        sum += w;
        if (w > 0.f) moment += w * d;
    }
    sum = block_join(sum, plus);
    moment = block_join(moment, plus);
    const float log_sum = logf(sum);
    const bool none = high == -INFINITY;
    if (tid == 0) {
        if (a.logprobs) a.logprobs[r] = given && !none ? below(key_logit(chosen)) - log_sum : -INFINITY;
        if (a.ranks) a.ranks[r] = given ? before : -1;
        if (a.entropy) a.entropy[r] = none ? 0.f : log_sum - moment / sum;
    }
    uint64_t last = ~0ull;
    for (int n = 0; n < a.top; ++n) {
        uint64_t best = 0;
        for (int i = tid; i < a.vocab; i += LOGPROB_THREADS) {
            const float v = logit_of(row[i]);
            const uint64_t key = order_key(v, i);
            if (v > -INFINITY && key < last && key > best) best = key;
        }
        last = block_join(best, most);
        if (tid == 0) {
            if (a.top_tokens) a.top_tokens[r * a.top + n] = last ? key_token(last) : -1;
            if (a.top_logprobs) a.top_logprobs[r * a.top + n] = last ? below(key_logit(last)) - log_sum : -INFINITY;
        }
    }
}

int launch_token_logprobs(pq_ctx *ctx, const void *logits, int elem, int64_t row_stride, int rows, int vocab, const int64_t *tokens, int top,
                          float *logprobs, int32_t *ranks, float *entropy, int64_t *top_tokens, float *top_logprobs) {
    const logprob_args a = {logits, tokens, logprobs, entropy, top_logprobs, ranks, top_tokens, row_stride, rows, vocab, top_tokens || top_logprobs ? top : 0};
    if (elem == PQ_ELEM_F32) token_logprobs_kernel<float><<<rows, LOGPROB_THREADS, 0, ctx->stream>>>(a);
    else if (elem == PQ_ELEM_F16) token_logprobs_kernel<_Float16><<<rows, LOGPROB_THREADS, 0, ctx->stream>>>(a);
    else token_logprobs_kernel<__bf16><<<rows, LOGPROB_THREADS, 0, ctx->stream>>>(a);
    PQ_HIP(ctx, hipGetLastError());
    return PQ_OK;
}

}  // namespace pq
