// Log-probabilities of given tokens, their ranks, the entropy and the likeliest tokens (pq_token_logprobs).
#include "elem.h"
#include "pq_internal.h"
#include "wave_sums.h"

namespace pq {

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
__device__ __forceinline__ uint32_t key_of(float v) {
    const uint32_t b = __builtin_bit_cast(uint32_t, v);
    return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ uint64_t order_key(float v, int i) { return (uint64_t)key_of(v) << 20 | (uint32_t)((1 << 20) - 1 - i); }
__device__ __forceinline__ int key_token(uint64_t key) { return (1 << 20) - 1 - (int)(key & ((1 << 20) - 1)); }
__device__ __forceinline__ float key_logit(uint64_t key) {
    const uint32_t b = (uint32_t)(key >> 20);
    return __builtin_bit_cast(float, b >> 31 ? b & 0x7fffffffu : ~b);
}

// the next number above (of +inf: NaN, which nothing reaches)
__device__ __forceinline__ float next_above(float v) {
    const uint32_t b = __builtin_bit_cast(uint32_t, v);
    return __builtin_bit_cast(float, v == 0.f ? 1u : b >> 31 ? b - 1 : b + 1);
}

// over a block, for the rare paths
template <int THREADS, class OP, class V> __device__ __forceinline__ V block_total(V v) {
    __shared__ V parts[THREADS / 64];
    v = wave_total<OP>(v);
    if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = v;
    __syncthreads();
    v = parts[0];
    for (int w = 1; w < THREADS / 64; ++w) v = OP::template of<V>(v, parts[w]);
    __syncthreads();
    return v;
}

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
// A reference: a logit times log2(e), rounded.  (The compiler may not take the product into what it is subtracted from: the difference of two
// references would be one of numbers that the sums are not formed with, and rows of 30 000 off by a thousandth.)
__device__ __forceinline__ float reference_of(float v) {
#pragma clang fp contract(off)
    return v * LOG2E;
}
// The sums are formed of logits from -WILD on (what is less, -inf and NaN count as -WILD), and hold for rows whose largest is between
// -WILD / 2 and WILD / 2: there what was raised has weight 0, 0 times it is 0, and a reference that is a logit times log2(e), rounded, is
// off by less than one.  Other rows are summed once more, by differences.  (A power of two: -WILD times log2(e) is not rounded.)
constexpr float WILD = 0x1p20f;

// the lowest bit of a logit, as fp32, that its type has (f16 numbers have 10 bits of fraction, bf16 7)
template <class T> constexpr int LEAST_BIT = __is_same(T, float) ? 0 : __is_same(T, _Float16) ? 13 : 16;
constexpr int STRETCHES = 16;  // parts of its logits that a thread keeps the maximum of
constexpr int GROUPS = 256;    // groups of threads whose maxima give the limit
constexpr int CANDIDATES = 1024, LISTED = 512;   // logits that are sorted, stretches that are read again

// One block for each row, which is read once.  A thread sums weights 2^y and y 2^y, y = logit * log2(e) - reference, by batches, and the
// reference is the largest logit of the batches so far.  The entropy is log2(sum) - (sum of y 2^y) / sum, of terms of one sign.
//
// The likeliest tokens cost the pass one store of a maximum for each batch.  `top` groups of threads have a maximum of at
// least the limit, the (top)th largest of the groups' maxima, so no smaller logit is listed, and nearly all that are as large are: for 20
// of 256 groups 20.8 are expected.  The few stretches that reach the limit are read again, their logits of at least the limit are
// sorted by counting.  Of too many (equal ones, or the largest all with one thread) those above the limit
// are, by one more pass, and the rest is searched by a pass for each different logit (1024 rows of 131 072, bf16, all but 20 logits -9984:
// 56 us with 10 listed, 410 with 50).
//
// Bound by memory where rows are many: 4096 rows of 131 072, bf16, 20 listed: 1.07 GB in 195 to 199 us = 5.4 TB/s; 1024 of these in f32
// without a list: 537 MB in 93 us = 5.8 TB/s.  A logit takes a conversion, a bound, half a maximum, two multiply-adds, an addition and a
// power of two (at a quarter of the rate), about 60 % of the cycles in bf16.  Few rows are bound by latency: 8 rows of 32 000, bf16: sums alone
// 4.6 us, a token's logit 0.8, the meeting, the stretches that are read again and the sort 3.0 us for one token listed, 4.3 for 20.
template <class T, int THREADS, int BATCH> __global__ __launch_bounds__(THREADS) void token_logprobs_kernel(logprob_args a) {
    constexpr int E = 16 / sizeof(T), WAVES = THREADS / 64;
    typedef elem_vec<T, E> vec;
    __shared__ float stretch_max[STRETCHES][THREADS];
    __shared__ uint64_t candidates[CANDIDATES];
    __shared__ uint32_t group_keys[GROUPS];
    __shared__ uint16_t stretches[LISTED];
    __shared__ float wave_high[WAVES], wave_sum[WAVES], wave_moment[WAVES], limit_at;
    __shared__ int wave_before[WAVES];
    __shared__ int nstretches, ncandidates;
    const int64_t r = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const T *const row = (const T *)a.logits + r * a.row_stride;

    // `head` logits before the first whole vector, and some behind the last, one for each of the first threads
    const int head = min(a.vocab, (int)((0 - (uintptr_t)row / sizeof(T)) % E)), nvec = (a.vocab - head) / E, tail = a.vocab - head - nvec * E;
    const vec *const vectors = (const vec *)(row + head);
    const int odd = tid < head ? tid : tid >= E && tid - E < tail ? head + nvec * E + tid - E : -1;

    // (the first batch is on its way before the token's logit is asked for)
    const int batches = (nvec + BATCH * THREADS - 1) / (BATCH * THREADS), per_stretch = (batches + STRETCHES - 1) / STRETCHES;
    vec next[BATCH];
    auto load = [&](int b) {
        const int j0 = b * BATCH * THREADS + tid;
        if ((b + 1) * BATCH * THREADS <= nvec) {
#pragma unroll
            for (int u = 0; u < BATCH; ++u) next[u] = vectors[j0 + u * THREADS];
        } else {
#pragma unroll
            for (int u = 0; u < BATCH; ++u) {
                if (j0 + u * THREADS < nvec) next[u] = vectors[j0 + u * THREADS];
                else
#pragma unroll
                    for (int e = 0; e < E; ++e) next[u].v[e] = (T)-INFINITY;
            }
        }
    };
    load(0);
    const int64_t token = a.tokens ? a.tokens[r] : -1;
    const bool given = token >= 0 && token < a.vocab;
    const float chosen = given ? logit_of(row[token]) : INFINITY, chosen_tame = fmaxf(chosen, -WILD), chosen_above = next_above(chosen);
    int before = 0;
    auto count = [&](float v, int i) { before += v > chosen || (v == chosen && i < token); };

    float high = -WILD, ref = -WILD * LOG2E, sum = 0.f, moment = 0.f;
    if (odd >= 0) {
        const float v = logit_of(row[odd]);
        if (given) count(v, odd);
        if (v > high) {
            high = v;
            ref = reference_of(v);
            const float y = fmaf(v, LOG2E, -ref), w = __builtin_amdgcn_exp2f(y);
            sum = w;
            moment = w * y;
        }
    }
    float stretch = -WILD;
    int stretch_at = 0, left = per_stretch;
    for (int b = 0; b < batches; ++b) {
        vec v[BATCH];
#pragma unroll
        for (int u = 0; u < BATCH; ++u) v[u] = next[u];
        if (b + 1 < batches) load(b + 1);
        const int j0 = b * BATCH * THREADS + tid;
        float x[BATCH * E], largest = -WILD;
#pragma unroll
        for (int i = 0; i < BATCH * E; ++i) {
            x[i] = fmaxf((float)v[i / E].v[i % E], -WILD);
            largest = fmaxf(largest, x[i]);
        }
        if (given && __any(largest >= chosen_tame)) {
#pragma unroll
            for (int u = 0; u < BATCH; ++u) {
                const int i0 = head + (j0 + u * THREADS) * E;
                if (chosen > -WILD && (i0 + E <= token || i0 > token)) {   // all before the token, or all behind it
                    const float least = i0 > token ? chosen_above : chosen;
#pragma unroll
                    for (int e = 0; e < E; ++e) before += x[u * E + e] >= least;
                } else if (j0 + u * THREADS < nvec) {
#pragma unroll
                    for (int e = 0; e < E; ++e) count(logit_of(v[u].v[e]), i0 + e);
                }
            }
        }
        if (a.top > 0) {
            stretch = fmaxf(stretch, largest);
            if (--left == 0) {
                stretch_max[stretch_at++][tid] = stretch;
                stretch = -WILD;
                left = per_stretch;
            }
        }
        high = fmaxf(high, largest);
        // (summed for itself first: a long chain of additions would be off by ten times as much)
        const float moved = reference_of(high), by = ref - moved, shrink = __builtin_amdgcn_exp2f(by);
        ref = moved;
        float batch_sum = 0.f, batch_moment = 0.f;
#pragma unroll
        for (int i = 0; i < BATCH * E; ++i) {
            const float y = fmaf(x[i], LOG2E, -ref), w = __builtin_amdgcn_exp2f(y);
            batch_sum += w;
            batch_moment = fmaf(w, y, batch_moment);
        }
        moment = fmaf(fmaf(sum, by, moment), shrink, batch_moment);
        sum = fmaf(sum, shrink, batch_sum);
    }
    if (a.top > 0)
        for (; stretch_at < STRETCHES; ++stretch_at) {
            stretch_max[stretch_at][tid] = stretch;
            stretch = -WILD;
        }
    const float own_high = high;

    // one meeting for the maximum and the groups' keys, one for the sums and the limit
    high = wave_total<op_larger>(high);
    if (lane == 0) wave_high[wave] = high;
    if (a.top > 0) {
        float group = own_high;
        for (int d = THREADS / GROUPS / 2; d > 0; d /= 2) group = fmaxf(group, __shfl_xor(group, d));
        if (tid % (THREADS / GROUPS) == 0) group_keys[tid / (THREADS / GROUPS)] = key_of(group);
    }
    if (tid == 0) nstretches = ncandidates = 0;
    __syncthreads();
    for (int w = 0; w < WAVES; ++w) high = fmaxf(high, wave_high[w]);
    const float joint = reference_of(high), by = ref - joint, shrink = __builtin_amdgcn_exp2f(by);
    moment = wave_total<op_add>(fmaf(sum, by, moment) * shrink);
    sum = wave_total<op_add>(sum * shrink);
    if (given) before = wave_total<op_add>(before);
    if (lane == 0) {
        wave_sum[wave] = sum;
        wave_moment[wave] = moment;
        wave_before[wave] = before;
    }
    // the limit, by the bits of the groups' maxima in their order (those that T has): as high as `top` groups reach it
    if (a.top > 0 && tid < 64) {
        uint32_t keys[GROUPS / 64], found = 0;
#pragma unroll
        for (int i = 0; i < GROUPS / 64; ++i) keys[i] = group_keys[64 * i + tid];
        for (int bit = 31; bit >= LEAST_BIT<T>; --bit) {
            const uint32_t next_key = found | 1u << bit;
            int reach = 0;
#pragma unroll
            for (int i = 0; i < GROUPS / 64; ++i) reach += __popcll(__ballot(keys[i] >= next_key));
            if (reach >= a.top) found = next_key;
        }
        // (the bits that T has not are ones in the key of a negative number: with zeros the limit would lie below the logit that it is)
        if (!(found >> 31)) found |= (1u << LEAST_BIT<T>) - 1;
        if (tid == 0) limit_at = key_logit((uint64_t)found << 20);
    }
    __syncthreads();
    sum = moment = 0.f;
    before = 0;
    for (int w = 0; w < WAVES; ++w) {
        sum += wave_sum[w];
        moment += wave_moment[w];
        before += wave_before[w];
    }
    // log of the sum of exp(logit - high)
    float log_sum = LN2 * (log2f(sum) - fmaf(high, LOG2E, -joint)), entropy = fmaxf(LN2 * (log2f(sum) - moment / sum), 0.f);
    // distance from the largest; where that is infinite, 0 for those that are it
    auto below = [&](float v) { return v == high ? 0.f : v - high; };
    if (!(fabsf(high) < WILD / 2)) {
        high = -INFINITY;
        for (int i = tid; i < a.vocab; i += THREADS) high = fmaxf(high, logit_of(row[i]));
        high = block_total<THREADS, op_larger>(high);
        // (in 64 bits: chains of up to 4096 additions of like terms drift by 4e-5 of the sum in 32)
        double all = 0.0, all_moments = 0.0;
        for (int i = tid; i < a.vocab; i += THREADS) {
            const float d = below(logit_of(row[i])), w = expf(d);
            all += (double)w;
            if (w > 0.f) all_moments += (double)w * (double)d;
        }
        all = block_total<THREADS, op_add>(all);
        all_moments = block_total<THREADS, op_add>(all_moments);
        log_sum = logf((float)all);
        entropy = high == -INFINITY ? 0.f : fmaxf(log_sum - (float)(all_moments / all), 0.f);
    }
    const bool none = high == -INFINITY;
    if (tid == 0) {
        if (a.logprobs) a.logprobs[r] = given && !none ? below(chosen) - log_sum : -INFINITY;
        if (a.ranks) a.ranks[r] = given ? before : -1;
        if (a.entropy) a.entropy[r] = entropy;
    }
    if (a.top == 0) return;
    auto put = [&](int n, uint64_t key) {   // 0: no token
        if (a.top_tokens) a.top_tokens[r * a.top + n] = key ? key_token(key) : -1;
        if (a.top_logprobs) a.top_logprobs[r * a.top + n] = key ? below(key_logit(key)) - log_sum : -INFINITY;
    };

    const float limit = fmaxf(limit_at, -0x1.fffffep19f);   // (above -WILD: of what lies from there on down, see the end)
    auto offer = [&](float v, int i) {
        const int n = atomicAdd(&ncandidates, 1);
        if (n < CANDIDATES) candidates[n] = order_key(v, i);
    };
    auto look = [&](float v, int i) {
        if (v >= limit) offer(v, i);
    };
    if (odd >= 0) look(logit_of(row[odd]), odd);
    if (own_high >= limit)
#pragma unroll
        for (int s = 0; s < STRETCHES; ++s)
            if (stretch_max[s][tid] >= limit) {
                const int n = atomicAdd(&nstretches, 1);
                if (n < LISTED) stretches[n] = (uint16_t)(s * THREADS + tid);
            }
    __syncthreads();
    const int per = per_stretch * BATCH, items = min(nstretches, LISTED) * per;
    for (int k = tid; k < items; k += THREADS) {
        const int s = stretches[k / per], j = (s / THREADS * per + k % per) * THREADS + s % THREADS;
        if (j >= nvec) continue;
        const vec v = vectors[j];
#pragma unroll
        for (int e = 0; e < E; ++e) look(logit_of(v.v[e]), head + j * E + e);
    }
    __syncthreads();
    bool listed = ncandidates <= CANDIDATES && nstretches <= LISTED;
    if (!listed) {   // too many are as large as the limit: those that are larger
        __syncthreads();
        if (tid == 0) ncandidates = 0;
        __syncthreads();
        for (int i = tid; i < a.vocab; i += THREADS) {
            const float v = logit_of(row[i]);
            if (v > limit) offer(v, i);
        }
        __syncthreads();
        listed = ncandidates <= CANDIDATES;
    }
    uint32_t last = ~0u;   // the least logit of those that are done
    int done = 0;
    if (listed) {
        const int n = ncandidates;
        for (int k = tid; k < n; k += THREADS) {
            const uint64_t mine = candidates[k];
            int place = 0;
            for (int i = 0; i < n; ++i) place += candidates[i] > mine;
            if (place < a.top) put(place, mine);
        }
        if (n >= a.top) return;
        for (int i = 0; i < n; ++i) last = min(last, (uint32_t)(candidates[i] >> 20));
        done = n;
    }
    // the rest one logit after the other, its tokens in their order
    while (done < a.top) {
        uint64_t best = 0;
        int times = 0;
        for (int i = tid; i < a.vocab; i += THREADS) {
            const float v = logit_of(row[i]);
            const uint32_t key = key_of(v), so_far = (uint32_t)(best >> 20);
            if (v == -INFINITY || key >= last || key < so_far) continue;
            times = key == so_far ? times + 1 : 1;
            if (key > so_far) best = order_key(v, i);
        }
        const uint64_t all = block_total<THREADS, op_larger>(best);
        if (!all) break;
        last = (uint32_t)(all >> 20);
        times = block_total<THREADS, op_add>((uint32_t)(best >> 20) == last ? times : 0);
        if (times == 1) {
            if (tid == 0) put(done, all);
            ++done;
            continue;
        }
        for (int i0 = key_token(all), until = min(a.top, done + times); done < until && i0 < a.vocab; i0 += THREADS) {
            const int i = i0 + tid;
            const bool is = i < a.vocab && key_of(logit_of(row[i])) == last;
            const uint64_t same = __ballot(is);
            __syncthreads();   // (what was read here before is)
            if (lane == 0) wave_before[wave] = __popcll(same);
            __syncthreads();
            int place = done + __popcll(same & ((1ull << lane) - 1));
            for (int w = 0; w < WAVES; ++w) {
                if (w < wave) place += wave_before[w];
                done += wave_before[w];
            }
            if (is && place < a.top) put(place, order_key(key_logit(all), i));
        }
    }
    for (int k = done + tid; k < a.top; k += THREADS) put(k, 0);
}

template <class T> static int logprobs_typed(pq_ctx *ctx, const logprob_args &a) {
    // 16 logits of a thread at a time: with 32, longer rows gain 3 % at most and short ones lose as much in occupancy.
    constexpr int E = 16 / sizeof(T), BATCH = 16 / E;
    // Few rows: more threads for each, so long as all of them have logits (8 rows of 32 000, bf16: 10.0 us, 12.4 with 256 threads; 256 rows
    // of 131 072: 20 and 29 us); with more rows than compute units not (300 rows of 50 021: 23.6 us, 18.8 with 256).  Long rows: fewer ends, which
    // are not hidden (131 072, bf16: 4096 rows 195 us with 512 threads, 205 with 256, 517 rows 38 and 42; but 1024 rows 67 and 58, and of 32 000
    // 4096 rows 72 and 63).
    const int threads = a.rows <= ctx->num_cu && a.vocab >= 1024 * E ? 1024 : a.vocab >= 65536 ? 512 : 256;
    if (!grid_fits(a.rows, threads)) return fail(ctx, PQ_EUNSUPPORTED, "token_logprobs: %d rows in one call", a.rows);
    if (threads == 1024) token_logprobs_kernel<T, 1024, BATCH><<<a.rows, 1024, 0, ctx->stream>>>(a);
    else if (threads == 512) token_logprobs_kernel<T, 512, BATCH><<<a.rows, 512, 0, ctx->stream>>>(a);
    else token_logprobs_kernel<T, 256, BATCH><<<a.rows, 256, 0, ctx->stream>>>(a);
    PQ_HIP(ctx, hipGetLastError());
    return PQ_OK;
}

int launch_token_logprobs(pq_ctx *ctx, const void *logits, int elem, int64_t row_stride, int rows, int vocab, const int64_t *tokens, int top,
                          float *logprobs, int32_t *ranks, float *entropy, int64_t *top_tokens, float *top_logprobs) {
    const logprob_args a = {logits, tokens, logprobs, entropy, top_logprobs, ranks, top_tokens, row_stride, rows, vocab, top_tokens || top_logprobs ? top : 0};
    if (elem == PQ_ELEM_F32) return logprobs_typed<float>(ctx, a);
    return elem == PQ_ELEM_F16 ? logprobs_typed<_Float16>(ctx, a) : logprobs_typed<__bf16>(ctx, a);
}

}  // namespace pq
