// The draw of the next tokens (pq_sample_tokens).
//
// A row's tokens are ordered by key = (falling logit, index), so what the filters leave is always a beginning of that order
// and a cut is one key.  The draw itself is a race: the token with the largest x_i - log(-log u_i) among those that stay is
// a sample of their softmax, and takes one pass without any running sum over the vocabulary, so it does not depend on how
// sums round.  Weights are summed as whole numbers of 2^-42: the sums, and with them the cuts, do not depend on the order
// of additions.
#include "elem.h"
#include "pq_internal.h"
#include "topk_device.h"

namespace pq {

constexpr int SAMPLE_THREADS = 1024;
constexpr int SAMPLE_BINS = 2048;
constexpr float SAMPLE_BINS_PER_UNIT = 23.5f;   // bins of x: 2048 of them reach down to x = -87, where exp(x) leaves fp32
constexpr float SAMPLE_LOWEST = -87.f;
constexpr int SAMPLE_LIST = 2 * SAMPLE_THREADS;   // keys that are sorted
constexpr double SAMPLE_MASS = 4398046511104.;    // 2^42

struct sample_args {
    const void *logits;
    int64_t row_stride, noise_stride;
    int vocab;
    const float *noise, *temperature, *top_p, *min_p;
    const int32_t *top_k;
    int64_t *tokens;
    float *logprobs;
};

// falling logit, then index: smaller keys come first
__device__ __forceinline__ uint64_t sample_key(float l, int i) { return (uint64_t)(~f32_to_ord(l)) << 32 | (uint32_t)i; }
__device__ __forceinline__ float sample_key_logit(uint64_t key) { return ord_to_f32(~(uint32_t)(key >> 32)); }
__device__ __forceinline__ uint64_t sample_mass(float w) { return (uint64_t)((double)w * SAMPLE_MASS); }

// one row's logits, eight at a time; f(index, logit) for each, NaN read as -inf
template <class T, class F> __device__ __forceinline__ void sample_each(const T *row, int vocab, F f) {
    constexpr int V = 8;
    struct __attribute__((packed, aligned(sizeof(T)))) vec { T v[V]; };
    const int whole = vocab / V * V;
    for (int i = threadIdx.x * V; i < whole; i += SAMPLE_THREADS * V) {
        const vec l = *(const vec *)(row + i);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float x = (float)l.v[e];
            f(i + e, x == x ? x : -INFINITY);
        }
    }
    for (int i = whole + threadIdx.x; i < vocab; i += SAMPLE_THREADS) {
        const float x = (float)row[i];
        f(i, x == x ? x : -INFINITY);
    }
}

struct sample_shared {
    uint32_t count[SAMPLE_BINS];
    uint64_t mass[SAMPLE_BINS];
    uint64_t list[SAMPLE_LIST];
    uint64_t wave64[SAMPLE_THREADS / 64], wave64b[SAMPLE_THREADS / 64];
    uint32_t nlist;
    int bin;
    uint64_t before_count, before_mass, low, high, cut, upto;
};

// x = (logit - max) / T of a row, and its weight
struct sample_scale {
    float top, inv;
    __device__ __forceinline__ float x(float l) const {
        if (!(l > -INFINITY)) return -INFINITY;
        return l == top ? 0.f : (l - top) * inv;   // (max +inf: the infinite ones share the weight)
    }
    __device__ __forceinline__ float weight(float xv) const { return xv >= SAMPLE_LOWEST ? expf(xv) : 0.f; }
    __device__ __forceinline__ int bin(float xv) const { return min(SAMPLE_BINS - 1, (int)(-xv * SAMPLE_BINS_PER_UNIT)); }
};

__device__ __forceinline__ uint64_t wave_min_u64(uint64_t v) {
    for (int d = 32; d > 0; d /= 2) v = min(v, (uint64_t)__shfl_xor((unsigned long long)v, d));
    return v;
}
__device__ __forceinline__ uint64_t wave_sum_u64(uint64_t v) {
    for (int d = 32; d > 0; d /= 2) v += (uint64_t)__shfl_xor((unsigned long long)v, d);
    return v;
}
__device__ uint64_t block_min_u64(sample_shared &sh, uint64_t v) {
    v = wave_min_u64(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh.wave64[threadIdx.x >> 6] = v;
    __syncthreads();
    for (int w = 0; w < SAMPLE_THREADS / 64; ++w) v = min(v, sh.wave64[w]);
    return v;
}
__device__ uint64_t block_sum_u64(sample_shared &sh, uint64_t v) {
    v = wave_sum_u64(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh.wave64[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
    for (int w = 0; w < SAMPLE_THREADS / 64; ++w) v += sh.wave64[w];
    return v;
}

// Sums (count, mass) up to and with this thread's entry, in thread order.
__device__ void block_scan_pair(sample_shared &sh, uint64_t &c, uint64_t &m) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int d = 1; d < 64; d *= 2) {
        const uint64_t cc = __shfl_up((unsigned long long)c, d), mm = __shfl_up((unsigned long long)m, d);
        if (lane >= d) {
            c += cc;
            m += mm;
        }
    }
    __syncthreads();
    if (lane == 63) {
        sh.wave64[wave] = c;
        sh.wave64b[wave] = m;
    }
    __syncthreads();
    for (int w = 0; w < wave; ++w) {
        c += sh.wave64[w];
        m += sh.wave64b[w];
    }
}

// The bin of the histogram in which a limit is reached: the first whose sums, on top of those before the histogram, come to
// `target` tokens (by_count) or weight.  Sets bin, before_count, before_mass; bin = SAMPLE_BINS if the limit is not reached.
__device__ void sample_find_bin(sample_shared &sh, bool by_count, uint64_t target) {
    const int b = 2 * threadIdx.x;
    const uint64_t c0 = sh.count[b], m0 = sh.mass[b], c1 = sh.count[b + 1], m1 = sh.mass[b + 1];
    uint64_t c = c0 + c1, m = m0 + m1;
    block_scan_pair(sh, c, m);
    const uint64_t bc = sh.before_count, bm = sh.before_mass;
    __syncthreads();
    if (threadIdx.x == 0) sh.bin = SAMPLE_BINS;
    __syncthreads();
    c += bc;
    m += bm;
    const uint64_t at = by_count ? c : m, step1 = by_count ? c1 : m1, step0 = by_count ? c0 : m0;
    if (at >= target && at - step1 - step0 < target) {
        const bool second = at - step1 < target;
        sh.bin = b + second;
        sh.before_count = c - c1 - (second ? 0 : c0);
        sh.before_mass = m - m1 - (second ? 0 : m0);
    }
    __syncthreads();
}

// Sorts the list's keys (two per thread), smallest first; those behind n are empty.
__device__ void sample_sort(sample_shared &sh, int n) {
    for (int i = threadIdx.x; i < SAMPLE_LIST; i += SAMPLE_THREADS)
        if (i >= n) sh.list[i] = KEY_EMPTY;
    int size = 2;
    while (size < n) size *= 2;
    __syncthreads();
    for (int k = 2; k <= size; k *= 2)
        for (int j = k / 2; j > 0; j /= 2) {
            for (int p = threadIdx.x; p < size / 2; p += SAMPLE_THREADS) {
                const int i = 2 * p - (p & (j - 1)), o = i + j;   // the pair whose members differ in bit j
                const uint64_t a = sh.list[i], b = sh.list[o];
                if ((a > b) == ((i & k) == 0)) {
                    sh.list[i] = b;
                    sh.list[o] = a;
                }
            }
            __syncthreads();
        }
}

// The cut at which a limit is reached: the key of the `target`-th token, or that of the token at which the weights reach
// `target`.  sh.cut is that key and sh.upto the weights up to and with it; all keys and weights if the limit is not reached.
// The histogram of x is in sh.count, sh.mass.
template <class T> __device__ void sample_find_cut(sample_shared &sh, const T *row, int vocab, const sample_scale &s, bool by_count, uint64_t target,
                                                   uint64_t all_mass) {
    const int tid = threadIdx.x;
    if (tid == 0) {
        sh.before_count = sh.before_mass = 0;
        sh.nlist = 0;
        sh.cut = KEY_EMPTY;
        sh.upto = all_mass;
        sh.low = KEY_EMPTY;
        sh.high = 0;
    }
    __syncthreads();
    sample_find_bin(sh, by_count, target);
    const int bin = sh.bin;
    if (bin >= SAMPLE_BINS) return;
    uint32_t n = sh.count[bin];
    uint64_t low = 0, high = KEY_EMPTY;   // the keys of the bin that are still in question
    if (n > SAMPLE_LIST) {
        // too many for the list: the bin's range of keys is split into 2048 parts, and the part with the limit again, until the
        // rest fits (equal logits are told apart by their indexes, so it ends).  The first histogram is needed again: it goes.
        sample_each(row, vocab, [&](int i, float l) {
            const float x = s.x(l);
            if (x >= SAMPLE_LOWEST && s.bin(x) == bin) {
                const uint64_t key = sample_key(l, i);
                atomicMin((unsigned long long *)&sh.low, key);
                atomicMax((unsigned long long *)&sh.high, key);
            }
        });
        __syncthreads();
        low = sh.low;
        high = sh.high;
        uint32_t keep_count[2];
        uint64_t keep_mass[2];
        for (int e = 0; e < 2; ++e) {
            keep_count[e] = sh.count[2 * tid + e];
            keep_mass[e] = sh.mass[2 * tid + e];
        }
        while (n > SAMPLE_LIST) {
            int shift = 0;
            while ((high - low) >> shift >= SAMPLE_BINS) ++shift;
            __syncthreads();
            for (int e = 0; e < 2; ++e) sh.count[2 * tid + e] = 0, sh.mass[2 * tid + e] = 0;
            __syncthreads();
            sample_each(row, vocab, [&](int i, float l) {
                const uint64_t key = sample_key(l, i);
                const float x = s.x(l);
                if (key < low || key > high || !(x >= SAMPLE_LOWEST) || s.bin(x) != bin) return;
                const int part = (int)((key - low) >> shift);
                atomicAdd(&sh.count[part], 1u);
                atomicAdd((unsigned long long *)&sh.mass[part], (unsigned long long)sample_mass(s.weight(x)));
            });
            __syncthreads();
            sample_find_bin(sh, by_count, target);
            const uint64_t part = sh.bin;
            n = sh.count[part];
            low += part << shift;
            high = min(high, low + ((uint64_t)1 << shift) - 1);
        }
        __syncthreads();
        for (int e = 0; e < 2; ++e) {
            sh.count[2 * tid + e] = keep_count[e];
            sh.mass[2 * tid + e] = keep_mass[e];
        }
        __syncthreads();
    }
    sample_each(row, vocab, [&](int i, float l) {
        const uint64_t key = sample_key(l, i);
        const float x = s.x(l);
        if (key < low || key > high || !(x >= SAMPLE_LOWEST) || s.bin(x) != bin) return;
        sh.list[atomicAdd(&sh.nlist, 1u)] = key;
    });
    __syncthreads();
    sample_sort(sh, (int)n);
    const uint64_t k0 = sh.list[2 * tid], k1 = sh.list[2 * tid + 1];
    const uint64_t m0 = k0 == KEY_EMPTY ? 0 : sample_mass(s.weight(s.x(sample_key_logit(k0))));
    const uint64_t m1 = k1 == KEY_EMPTY ? 0 : sample_mass(s.weight(s.x(sample_key_logit(k1))));
    uint64_t c = (k0 != KEY_EMPTY) + (k1 != KEY_EMPTY), m = m0 + m1;
    block_scan_pair(sh, c, m);
    c += sh.before_count;
    m += sh.before_mass;
    const uint64_t at = by_count ? c : m, step1 = by_count ? k1 != KEY_EMPTY : m1, step0 = by_count ? k0 != KEY_EMPTY : m0;
    if (at >= target && at - step1 - step0 < target) {
        const bool second = at - step1 < target;
        sh.cut = second ? k1 : k0;
        sh.upto = second ? m : m - m1;
    }
    __syncthreads();
}

template <class T> __global__ __launch_bounds__(SAMPLE_THREADS) void sample_kernel(sample_args a) {
    __shared__ sample_shared sh;
    const int r = blockIdx.x, tid = threadIdx.x;
    const T *row = (const T *)a.logits + r * a.row_stride;
    const float *noise = a.noise ? a.noise + r * a.noise_stride : nullptr;

    uint64_t first = KEY_EMPTY;
    sample_each(row, a.vocab, [&](int i, float l) { first = min(first, sample_key(l, i)); });
    first = block_min_u64(sh, first);
    sample_scale s;
    s.top = sample_key_logit(first);
    const float t = a.temperature ? a.temperature[r] : 1.f;
    if (!(s.top > -INFINITY)) {
        if (tid == 0) {
            a.tokens[r] = -1;
            if (a.logprobs) a.logprobs[r] = -INFINITY;
        }
        return;
    }
    const bool greedy = !(t > 0.f);
    if (greedy && (tid == 0)) {
        a.tokens[r] = (int64_t)(uint32_t)first;
        if (a.logprobs) a.logprobs[r] = 0.f;
    }
    if (greedy) return;
    s.inv = fminf(1.f / t, 3.402823466e38f);
    const int64_t top_k = a.top_k ? a.top_k[r] : 0;
    const float top_p = a.top_p ? a.top_p[r] : 1.f, min_p = a.min_p ? a.min_p[r] : 0.f;
    const bool by_k = top_k > 0 && top_k < a.vocab, by_p = top_p < 1.f;

    uint64_t cut = KEY_EMPTY;
    if (by_k || by_p) {
        for (int b = tid; b < SAMPLE_BINS; b += SAMPLE_THREADS) sh.count[b] = 0, sh.mass[b] = 0;
        __syncthreads();
        sample_each(row, a.vocab, [&](int, float l) {
            const float x = s.x(l);
            if (!(x >= SAMPLE_LOWEST)) return;
            const int b = s.bin(x);
            atomicAdd(&sh.count[b], 1u);
            atomicAdd((unsigned long long *)&sh.mass[b], (unsigned long long)sample_mass(s.weight(x)));
        });
        __syncthreads();
        uint64_t all = block_sum_u64(sh, sh.mass[2 * tid] + sh.mass[2 * tid + 1]);
        if (by_k) {
            sample_find_cut(sh, row, a.vocab, s, true, (uint64_t)top_k, all);
            cut = sh.cut;
            all = sh.upto;
            __syncthreads();
        }
        if (by_p) {
            // a token stays while the weights before it are below top_p * all: up to the one that reaches the next whole number
            const double limit = ceil(fmax(0., (double)top_p) * (double)all);
            sample_find_cut(sh, row, a.vocab, s, false, max((uint64_t)1, (uint64_t)limit), all);
            cut = min(cut, sh.cut);
        }
    }

    // the race among the keys up to the cut: the largest score, then the smallest index
    uint64_t best = KEY_EMPTY, mass = 0;
    float drawn = 0.f;
    sample_each(row, a.vocab, [&](int i, float l) {
        const uint64_t key = sample_key(l, i);
        if (key > cut) return;
        const float x = s.x(l);
        const float w = s.weight(x);
        if (!(w > 0.f) || (w < min_p && key != first)) return;
        mass += sample_mass(w);
        const float score = noise ? x - logf(-logf(noise[i])) : x;
        best = min(best, sample_key(score, i));
    });
    // (a score that is NaN, from noise outside 0 ... 1, sorts behind or before the others: some token is drawn all the same)
    const uint64_t all_best = block_min_u64(sh, best);
    mass = block_sum_u64(sh, mass);
    const int token = (int)(uint32_t)all_best;
    if (tid == 0) {
        a.tokens[r] = token;
        drawn = s.x((float)row[token]);
        if (a.logprobs) a.logprobs[r] = (float)((double)drawn - log((double)mass / SAMPLE_MASS));
    }
}

int launch_sample_tokens(pq_ctx *ctx, const void *logits, int elem, int64_t row_stride, int rows, int vocab, const float *noise,
                         int64_t noise_stride, const float *temperature, const int32_t *top_k, const float *top_p,
                         const float *min_p, int64_t *tokens, float *logprobs) {
    const sample_args a = {logits, row_stride, noise_stride, vocab, noise, temperature, top_p, min_p, top_k, tokens, logprobs};
    if (elem == PQ_ELEM_F32) sample_kernel<float><<<rows, SAMPLE_THREADS, 0, ctx->stream>>>(a);
    else if (elem == PQ_ELEM_F16) sample_kernel<_Float16><<<rows, SAMPLE_THREADS, 0, ctx->stream>>>(a);
    else sample_kernel<__bf16><<<rows, SAMPLE_THREADS, 0, ctx->stream>>>(a);
    PQ_HIP(ctx, hipGetLastError());
    return PQ_OK;
}

}  // namespace pq
