// The draw of the next tokens (pq_sample_tokens).
//
// A row's tokens are ordered by key = (falling logit, index), so what the filters leave is always a beginning of that order
// and a cut is one key.  The draw itself is a race: with weights w_i and e_i = -log u_i the token with the largest w_i / e_i
// among those that stay is a sample of their softmax.  It takes one pass without a running sum over the vocabulary, so it
// does not depend on how sums round; and since e_i >= 1 - u_i, a token whose w_i is below (best so far) * (1 - u_i) cannot
// win, which spares nearly all of them the logarithm.
//
// Cuts: one pass puts every token into one of 2048 bins of 1/16 octave of weight, count and weight in one 64-bit word (all
// weights of a bin have the same power of two, so they add up as whole numbers, in any order to the same sum).  The bin in
// which a limit is reached is then known, and the next pass collects the tokens of the bins up to it, or of that bin alone
// where those are too many for the list.  Finer bins of the list end at 256 keys or fewer, which are ranked.  Where the
// list holds all that stay, the draw is from it, else from one more pass over the row.
//
// Weights are relative to a logit that a first look at a part of the row has found, not to the largest: so the pass that fills
// the bins also finds the largest, and the row is read from memory once.  A row whose largest logit lies more than
// SAMPLE_TOP octaves above that look is passed over again, before a bin or a limit is taken from it: these are in the
// reference's octaves, so it is the same from there on to the draw.
//
// 256 rows of 131 072 f32 logits with filters: 64 us (134 MB; 26 us at the rate of a large copy), bound by the adds to the bins and by
// the steps behind that pass, of one block each.  8 rows of 32 000: 17 to 25 us by their filters, all latency: a dozen steps with
// a barrier or a trip to memory each.
//
// A row is one block's work: 256 rows are one for each compute unit.  Only rows of calls without filters, which are one pass,
// are shared by several blocks where they are few (see sample_typed).
#include "elem.h"
#include "pq_internal.h"
#include "topk_device.h"
#include "wave_sums.h"

namespace pq {

constexpr int SAMPLE_THREADS = 1024;
constexpr int SAMPLE_WAVES = SAMPLE_THREADS / 64;
static_assert(SAMPLE_WAVES == 16, "the waves' results are joined by one row of 16 lanes");
constexpr int SAMPLE_V = 8;                // tokens that a thread reads at once
constexpr int SAMPLE_BINS = 2048;
constexpr int SAMPLE_ABOVE = 1024;         // of them above weight 1: 64 octaves, and 64 below
constexpr int SAMPLE_LIST = 4096;
constexpr int SAMPLE_LAST = 256;           // keys among which a cut is found by their ranks
constexpr int SAMPLE_COUNT_BIT = 44;       // a bin: count << 44 | weights in 2^-23 of the bin's power of two
constexpr float SAMPLE_TOP = 60.f;         // octaves above the reference up to which weights and their sums stay in fp32, and in the bins
static_assert(SAMPLE_TOP < SAMPLE_ABOVE / 16, "what is taken lies below the end of the bins");
constexpr int SAMPLE_NONE = 0x7fffffff;

struct sample_args {
    const void *logits;
    int64_t row_stride, noise_stride;
    int vocab;
    const float *noise, *temperature, *top_p, *min_p;
    const int32_t *top_k;
    int64_t *tokens;
    float *logprobs;
};

// falling logit, then index: smaller keys come first (both zeros are equal)
__device__ __forceinline__ uint64_t sample_key(float l, int i) { return (uint64_t)(~f32_to_ord(l + 0.f)) << 32 | (uint32_t)i; }
__device__ __forceinline__ float sample_key_logit(uint64_t key) { return ord_to_f32(~(uint32_t)(key >> 32)); }

struct op_min_u64 {
    template <class V> static __device__ __forceinline__ V none() { return KEY_EMPTY; }
    template <class V> static __device__ __forceinline__ V of(V a, V b) { return min(a, b); }
};
struct op_max {
    template <class V> static __device__ __forceinline__ V none() { return -INFINITY; }
    template <class V> static __device__ __forceinline__ V of(V a, V b) { return fmaxf(a, b); }
};
struct sample_shared {
    unsigned long long bins[SAMPLE_BINS], fine[SAMPLE_BINS];
    unsigned long long list[SAMPLE_LIST], last[SAMPLE_LAST], sorted[SAMPLE_LAST];
    unsigned long long wave64[2][SAMPLE_WAVES];   // two of each, used in turn: one barrier per use
    double wave_d[2][SAMPLE_WAVES];
    uint32_t wave32[2][SAMPLE_WAVES];
    unsigned long long cut;
    double mass;
    uint32_t count, nlist, nlast, best;
    int bin;
};

// what a limit is reached by: so many tokens, or so much weight
struct sample_limit {
    bool by_count;
    uint32_t count;
    double mass;
    __device__ __forceinline__ bool reached(uint32_t c, double m) const { return by_count ? c >= count : m >= mass; }
};

// Weights of a row's logits, as exponents of two: y = log2(w).  What is far below the bins is cut off there, so is what is no
// number (the middle of three is the smallest then), and what is above them at SAMPLE_CAP.
constexpr float SAMPLE_FLOOR = -70.f, SAMPLE_LEAST = -63.f, SAMPLE_CAP = 1e30f;
struct sample_scale {
    float c, ref, low, high;   // y = c * (l - ref), the difference within low ... high
    __device__ __forceinline__ sample_scale(float reference, float inv_t) {
        ref = fminf(reference, 3.402823466e38f);
        c = fminf(fmaxf(inv_t * 1.4426950408889634f, 1e-36f), 1e36f);
        low = SAMPLE_FLOOR / c;
        high = reference < INFINITY ? fminf(SAMPLE_CAP / c, 3.402823466e38f) : 0.f;   // (+inf and the largest number share the weight)
    }
    __device__ __forceinline__ float y(float l) const { return __builtin_amdgcn_fmed3f(l - ref, low, high) * c; }
    static __device__ __forceinline__ float weight(float y) { return __builtin_amdgcn_exp2f(y); }
};
// Bins are sixteenths of an octave, in the order of falling weight; SAMPLE_BINS is what lies below.
__device__ __forceinline__ int bin_of(float y) {
    int k;   // floor
    asm("v_cvt_flr_i32_f32 %0, %1" : "=v"(k) : "v"(y * 16.f));
    return max(SAMPLE_ABOVE - 1 - max(k, SAMPLE_ABOVE - 1 - SAMPLE_BINS), 0);
}
// a weight within its bin, one unit of the count above it
__device__ __forceinline__ unsigned long long bin_word(float y) {
    const uint32_t q = (__float_as_uint(__builtin_amdgcn_exp2f(__builtin_amdgcn_fractf(y))) & 0x7fffffu) | 0x800000u;
    return (unsigned long long)1 << SAMPLE_COUNT_BIT | q;
}
__device__ __forceinline__ uint32_t bin_count(unsigned long long b) { return (uint32_t)(b >> SAMPLE_COUNT_BIT); }
__device__ __forceinline__ double bin_mass(unsigned long long b, int octave) {
    // (2^octave by its exponent bits: octaves are -64 ... 63)
    const double unit = __longlong_as_double((long long)(1023 + octave - 23) << 52);
    return (double)(b & (((unsigned long long)1 << SAMPLE_COUNT_BIT) - 1)) * unit;
}
__device__ __forceinline__ int bin_octave(int bin) { return (SAMPLE_ABOVE - 1 - bin) >> 4; }

// What a part of a row comes to.
struct sample_part {
    uint64_t key;
    double mass;
    float high;
};

template <class T> struct sample_row {
    const sample_args &a;
    sample_shared &sh;
    const T *row;
    const float *noise;
    int64_t r;
    int turn;

    // The row as vectors of eight on 16 bytes and the few logits before and behind them.  A thread keeps its vector of the
    // first 1024 in registers (the first look; empty places hold -inf) until the pass over the rest.
    struct alignas(16) vec { T v[SAMPLE_V]; };
    static constexpr int STEP = SAMPLE_THREADS * SAMPLE_V;
    int before, whole;      // vectors are at before ... whole
    int head, tail;         // the few others before `head` and from `tail` on
    float look[SAMPLE_V];
    __device__ __forceinline__ void whole_row() {
        before = head = min(a.vocab, (int)((16 - ((uintptr_t)row & 15)) % 16 / sizeof(T)));
        whole = tail = before + (a.vocab - before) / SAMPLE_V * SAMPLE_V;
    }
    __device__ __forceinline__ void part_of_row(int part, int parts) {
        whole_row();
        const int64_t n = (whole - before) / SAMPLE_V;
        whole = before + (int)(n * (part + 1) / parts) * SAMPLE_V;
        before += (int)(n * part / parts) * SAMPLE_V;
        if (part > 0) head = 0, tail = a.vocab;
    }
    __device__ __forceinline__ void load_look() {
        const int i = before + threadIdx.x * SAMPLE_V;
        if (i < whole) {
            const vec l = *(const vec *)(row + i);
#pragma unroll
            for (int e = 0; e < SAMPLE_V; ++e) look[e] = (float)l.v[e];
        } else {
#pragma unroll
            for (int e = 0; e < SAMPLE_V; ++e) look[e] = -INFINITY;
        }
    }
    // f(first index, logits) for the vectors, g(index, logit) for the few others; two vectors are on their way at a time.
    // `rest`: without the first look.
    // With `beside`, f's third argument is the noise of the vector, read together with it.
    struct __attribute__((packed, aligned(4))) noises { float v[SAMPLE_V]; };
    template <class F, class G> __device__ __forceinline__ void each_vector(bool rest, bool beside, F f, G g) {
        auto take = [&](const vec &l, const noises &u, int i) {
            float x[SAMPLE_V];
#pragma unroll
            for (int e = 0; e < SAMPLE_V; ++e) x[e] = (float)l.v[e];
            f(i, x, u);
        };
        int i = before + threadIdx.x * SAMPLE_V + (rest ? STEP : 0);
        for (; i + STEP < whole; i += 2 * STEP) {
            const vec p = *(const vec *)(row + i), q = *(const vec *)(row + i + STEP);
            noises up, uq;
            if (beside) {
                up = *(const noises *)(noise + i);
                uq = *(const noises *)(noise + i + STEP);
            }
            take(p, up, i);
            take(q, uq, i + STEP);
        }
        if (i < whole) {
            noises u;
            if (beside) u = *(const noises *)(noise + i);
            take(*(const vec *)(row + i), u, i);
        }
        const int t = (int)threadIdx.x < head ? (int)threadIdx.x : tail + (int)threadIdx.x - head;
        if (t < a.vocab) g(t, (float)row[t]);
    }
    template <class F> __device__ __forceinline__ void each(F f) {
        each_vector(false, false, [&](int i, const float (&l)[SAMPLE_V], const noises &) {
#pragma unroll
            for (int e = 0; e < SAMPLE_V; ++e) f(i + e, l[e]);
        }, f);
    }

    __device__ __forceinline__ uint64_t block_min(uint64_t v) {
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
        turn ^= 1;
        v = wave_scan<op_min_u64>(v);
        if (lane == 63) sh.wave64[turn][wave] = v;
        __syncthreads();
        v = row_scan<op_min_u64>((uint64_t)sh.wave64[turn][lane & 15]);
        return read_lane(v, 15);
    }
    __device__ __forceinline__ float block_max(float v) {
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
        turn ^= 1;
        v = wave_scan<op_max>(v);
        if (lane == 63) sh.wave32[turn][wave] = __float_as_uint(v);
        __syncthreads();
        v = row_scan<op_max>(__uint_as_float(sh.wave32[turn][lane & 15]));
        return read_lane(v, 15);
    }
    __device__ __forceinline__ uint64_t block_sum(uint64_t v) {
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
        turn ^= 1;
        v = wave_scan<op_add>(v);
        if (lane == 63) sh.wave64[turn][wave] = v;
        __syncthreads();
        v = row_scan<op_add>((uint64_t)sh.wave64[turn][lane & 15]);
        return read_lane(v, 15);
    }
    __device__ __forceinline__ double block_sum(double v) {
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
        turn ^= 1;
        v = wave_scan<op_add>(v);
        if (lane == 63) sh.wave_d[turn][wave] = v;
        __syncthreads();
        v = row_scan<op_add>(sh.wave_d[turn][lane & 15]);
        return read_lane(v, 15);
    }
    __device__ __forceinline__ void done(int64_t token, float logprob) {
        if (threadIdx.x != 0) return;
        a.tokens[r] = token;
        if (a.logprobs) a.logprobs[r] = logprob;
    }

    // The key of the largest logit (NaN reads as -inf): vectors that hold nothing larger than before are passed over.
    __device__ __forceinline__ uint64_t first_key() {
        float high = -INFINITY;
        int at = SAMPLE_NONE;
        auto take = [&](int i, float l) {
            if (l > high || (l == high && i < at)) {
                high = l;
                at = i;
            }
        };
        each_vector(false, false, [&](int i, const float (&l)[SAMPLE_V], const noises &) {
            float most = l[0];
#pragma unroll
            for (int e = 1; e < SAMPLE_V; ++e) most = fmaxf(most, l[e]);
            if (!(most > high)) return;
#pragma unroll
            for (int e = 0; e < SAMPLE_V; ++e) take(i + e, l[e]);
        }, take);
        return block_min(sample_key(high, at));
    }

    // the best of a thread's race: largest w / e (logit without noise), then smallest index
    struct race {
        float best = -1.f;
        int token = SAMPLE_NONE;
        __device__ __forceinline__ void enter(float w, float u, int i) {
            const float r = w / fmaxf(-logf(u), 1e-30f);
            if (r > best || (r == best && i < token)) {
                best = r;
                token = i;
            }
        }
        // Without noise: the largest logit.  (Not the largest weight: different logits may round to one.)
        __device__ __forceinline__ void enter_certain(float l, int i) {
            if (token == SAMPLE_NONE || l > best || (l == best && i < token)) {
                best = l;
                token = i;
            }
        }
    };
    // The winner of the block's races as a key, the best first; KEY_EMPTY: none (noise that is no number).
    __device__ __forceinline__ uint64_t winner(const race &x) { return block_min(x.token == SAMPLE_NONE ? KEY_EMPTY : sample_key(x.best, x.token)); }
    // The winner's token, and the log of its share of the weights that stay.
    __device__ __forceinline__ void finish(uint64_t best, const sample_scale &s, double mass) {
        if (best == KEY_EMPTY) best = first_key();
        if (threadIdx.x != 0) return;
        const int token = (int)(uint32_t)best;
        const float octaves = (float)__builtin_amdgcn_frexp_exp(mass);
        done((int64_t)token, (s.y((float)row[token]) - octaves - log2f((float)__builtin_amdgcn_frexp_mant(mass))) * 0.6931471805599453f);
    }

    // Race over the row (or this part): tokens with y of at least `upper` and `least` stay; those from `lower` to below `upper`, which
    // are the bin of the cut, all go into the list (there is room; `cut` KEY_EMPTY), or stay if their key is not behind `cut`
    // (and y at least `least`).  Returns the largest y.
    // many: of most vectors some token stays, so that their noise is read beside them, not after them.
    // A bound on the winner, w / e, is found first, on the first look: e = -log u is at most (1 - u) / u.
    __device__ __forceinline__ float draw(const sample_scale &s, float upper, float lower, float least, uint64_t cut, bool many, race &best, double &mass) {
        const float edge = fmaxf(upper, least);
        float high = -INFINITY, sum[SAMPLE_V] = {};
        auto weight = [&](float y) { return y >= edge ? s.weight(y) : 0.f; };
        auto border = [&](int i) {   // a token of the cut's bin (indexes first, in the place of the keys)
            if (cut == KEY_EMPTY) {
                list_index(i);
                return;
            }
            const float l = (float)row[i], y = s.y(l);
            if (sample_key(l, i) > cut || !(y >= least)) return;
            const float w = s.weight(y);
            sum[0] += w;
            if (noise) best.enter(w, noise[i], i);
            else best.enter_certain(l, i);
        };
        float bounded = 0.f;
        const int first = before + threadIdx.x * SAMPLE_V;
        if (noise && first < whole) {
            const noises u = *(const noises *)(noise + first);
#pragma unroll
            for (int e = 0; e < SAMPLE_V; ++e) bounded = fmaxf(bounded, weight(s.y(look[e])) * u.v[e] * __builtin_amdgcn_rcpf(1.f - u.v[e]));
        }
        bounded = block_max(bounded) * (1.f - 1e-6f);   // (rounded down)
        if (threadIdx.x == 0) {
            sh.best = __float_as_uint(bounded < INFINITY ? bounded : 0.f);
            sh.nlist = 0;
        }
        __syncthreads();
        many = many && noise;
        each_vector(false, many, [&](int i, const float (&l)[SAMPLE_V], noises u) {
            float w[SAMPLE_V], most = -INFINITY;
            uint32_t which = 0;
#pragma unroll
            for (int e = 0; e < SAMPLE_V; ++e) {
                const float y = s.y(l[e]);
                most = fmaxf(most, y);
                w[e] = weight(y);
                sum[e] += w[e];
                which |= (uint32_t)(y >= lower && y < upper) << e;
            }
            high = fmaxf(high, most);
            for (; which; which &= which - 1) border(i + __ffs(which) - 1);
            if (!(most >= edge)) return;
            if (!noise) {
#pragma unroll
                for (int e = 0; e < SAMPLE_V; ++e)
                    if (w[e] > 0.f) best.enter_certain(l[e], i + e);
                return;
            }
            if (!many) u = *(const noises *)(noise + i);
            const float so_far = __uint_as_float(__hip_atomic_load(&sh.best, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP));
            bool wins = false;
#pragma unroll
            for (int e = 0; e < SAMPLE_V; ++e) wins |= w[e] >= so_far * (1.f - u.v[e]);   // (weights of 0 are sorted out below)
            if (!wins) return;
#pragma unroll
            for (int e = 0; e < SAMPLE_V; ++e)
                if (w[e] > 0.f && w[e] >= so_far * (1.f - u.v[e])) best.enter(w[e], u.v[e], i + e);
            // (rounded down, so that the logarithm's last bit decides nothing: the winner is the same whoever passes here first)
            if (best.best > so_far) atomicMax(&sh.best, __float_as_uint(best.best * (1.f - 1e-6f)));
        }, [&](int i, float l) {
            const float y = s.y(l), w = weight(y);
            high = fmaxf(high, y);
            sum[0] += w;
            if (y >= lower && y < upper) border(i);
            if (!(w > 0.f)) return;
            if (noise) best.enter(w, noise[i], i);
            else best.enter_certain(l, i);
        });
#pragma unroll
        for (int e = 0; e < SAMPLE_V; ++e) mass += (double)sum[e];
        high = block_max(high);
        if (cut == KEY_EMPTY) list_keys(list_size());
        return high;
    }
    // Places of the list are given out in any order; what finds none is not listed.
    __device__ __forceinline__ void list_index(int i) {
        const uint32_t at = atomicAdd(&sh.nlist, 1u);
        if (at < SAMPLE_LIST) sh.list[at] = (uint32_t)i;
    }
    __device__ __forceinline__ uint32_t list_size() { return min(sh.nlist, (uint32_t)SAMPLE_LIST); }
    // The list's n indexes become keys.
    __device__ __forceinline__ void list_keys(uint32_t n) {
        for (uint32_t i = threadIdx.x; i < n; i += SAMPLE_THREADS) {
            const int at = (int)sh.list[i];
            sh.list[i] = sample_key((float)row[at], at);
        }
        __syncthreads();
    }
    // The race on the list's keys up to `cut`.  Returns their weights that stay, summed as whole numbers (the keys are in no
    // order); top: the largest y.
    __device__ __forceinline__ double draw_list(const sample_scale &s, int listed, float least, float top, uint64_t cut, race &best) {
        const int shift = (int)ceilf(top);   // weights of at most 2^shift, in 2^-44 of that
        uint64_t mass = 0;
        for (int i = threadIdx.x; i < listed; i += SAMPLE_THREADS) {
            const uint64_t key = sh.list[i];
            const float l = sample_key_logit(key), y = s.y(l), w = s.weight(y);
            const int token = (int)(uint32_t)key;
            if (key > cut || !(y >= least)) continue;
            mass += (uint64_t)ldexp((double)w, 44 - shift);
            if (noise) best.enter(w, noise[token], token);
            else best.enter_certain(l, token);
        }
        return ldexp((double)block_sum(mass), shift - 44);
    }

    // Bins of the whole row; top: the largest y, which has to lie below them.  The bins of the first look at the row say from
    // which bin on about `wanted` tokens are to be expected, and these go into the list on the way: listed = the last bin that
    // the list then holds with all before it, -1 if they were too many.
    __device__ __forceinline__ void fill_bins(const sample_scale &s, uint32_t wanted, float &top, int &listed) {
        const int tid = threadIdx.x;
        for (int b = tid; b < SAMPLE_BINS; b += SAMPLE_THREADS) sh.bins[b] = 0;
        if (tid == 0) sh.nlist = 0;
        __syncthreads();
        float high = -INFINITY;
        auto add = [&](float y) {   // (what lies below the bins may be most of a row: nothing is added to one place for all of it)
            const int b = bin_of(y);
            if (b < SAMPLE_BINS) atomicAdd(&sh.bins[b], bin_word(y));
        };
        const int first = before + tid * SAMPLE_V;
        if (first < whole) {
#pragma unroll
            for (int e = 0; e < SAMPLE_V; ++e) {
                const float y = s.y(look[e]);
                high = fmaxf(high, y);
                add(y);
            }
        }
        __syncthreads();
        uint32_t c = 0;
        double m = 0.;
        wanted = max(1u, (uint32_t)((float)wanted * (float)min(whole - before, STEP) / (float)a.vocab));
        const int last = min(find_bin(sh.bins, sample_limit{true, wanted, 0.}, c, m, bin_octave), SAMPLE_BINS - 1);
        const float lowest = (float)(SAMPLE_ABOVE - 1 - last) * 0.0625f;
        auto list = [&](int i, const float (&y)[SAMPLE_V], float most) {   // (indexes first, in the place of the keys)
            if (!(most >= lowest)) return;
            uint32_t which = 0;
#pragma unroll
            for (int e = 0; e < SAMPLE_V; ++e) which |= (uint32_t)(y[e] >= lowest) << e;
            for (; which; which &= which - 1) list_index(i + __ffs(which) - 1);
        };
        if (first < whole) {
            float y[SAMPLE_V], most = -INFINITY;
#pragma unroll
            for (int e = 0; e < SAMPLE_V; ++e) most = fmaxf(most, y[e] = s.y(look[e]));
            list(first, y, most);
        }
        each_vector(true, false, [&](int i, const float (&l)[SAMPLE_V], const noises &) {
            float y[SAMPLE_V], most = -INFINITY;
#pragma unroll
            for (int e = 0; e < SAMPLE_V; ++e) {
                y[e] = s.y(l[e]);
                most = fmaxf(most, y[e]);
                add(y[e]);
            }
            high = fmaxf(high, most);
            list(i, y, most);
        }, [&](int i, float l) {
            const float y = s.y(l);
            high = fmaxf(high, y);
            add(y);
            if (y >= lowest) list_index(i);
        });
        top = block_max(high);
        listed = sh.nlist <= SAMPLE_LIST ? last : -1;
        if (listed >= 0) list_keys(sh.nlist);
    }

    // The bin in which a limit is reached, counting from c, m before the bins: the bin (SAMPLE_BINS: it is not reached), and
    // in c, m the sums before it.  octave(bin): the power of two of a bin's weights.
    template <class O> __device__ __forceinline__ int find_bin(const unsigned long long *bins, const sample_limit &limit, uint32_t &c0, double &m0, O octave) {
        const int b = 2 * threadIdx.x, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
        const unsigned long long v0 = bins[b], v1 = bins[b + 1];
        const double w0 = bin_mass(v0, octave(b)), w1 = bin_mass(v1, octave(b + 1));
        turn ^= 1;
        uint32_t c = wave_scan<op_add>(bin_count(v0) + bin_count(v1));
        double m = wave_scan<op_add>(w0 + w1);
        if (lane == 63) {
            sh.wave32[turn][wave] = c;
            sh.wave_d[turn][wave] = m;
        }
        __syncthreads();
        const uint32_t wave_count = sh.wave32[turn][lane & 15], cw = row_scan<op_add>(wave_count) + c0;
        const double mw = row_scan<op_add>(sh.wave_d[turn][lane & 15]) + m0;
        if (!limit.reached(read_lane(cw, 15), read_lane(mw, 15))) return SAMPLE_BINS;
        // One wave: of those that hold a token the first whose sum reaches the limit; in it the first bin that does.  An empty one
        // reaches nothing: sums of different waves are added up in different orders, so one may be the last bit above, or below, the
        // sum that it adds nothing to.  Where rounding lets none reach the limit, the last that is not empty.
        const uint32_t holds = (uint32_t)__ballot(wave_count > 0) & 0xffff, reach = (uint32_t)__ballot(limit.reached(cw, mw)) & holds;
        if (holds == 0) return SAMPLE_BINS;
        if (wave == (reach ? __ffs(reach) - 1 : 31 - __clz((int)holds))) {
            const uint32_t cb = wave > 0 ? read_lane(cw, wave - 1) : c0;
            const double mb = wave > 0 ? read_lane(mw, wave - 1) : m0;
            c += cb;
            m += mb;
            const uint32_t n0 = bin_count(v0), n1 = bin_count(v1);
            bool at0 = n0 && limit.reached(c - n1, m - w1), at1 = n1 && limit.reached(c, m);
            uint64_t there = __ballot(at0 || at1);
            if (!there) {
                at0 = !n1;
                there = __ballot(n0 || n1);
                there = there ? 1ull << (63 - __clzll((long long)there)) : 1;
            }
            if (lane == __ffsll((unsigned long long)there) - 1) {
                sh.bin = at0 ? b : b + 1;
                sh.count = c - n1 - (at0 ? n0 : 0);
                sh.mass = m - w1 - (at0 ? w0 : 0.);
            }
        }
        __syncthreads();
        c0 = sh.count;
        m0 = sh.mass;
        return sh.bin;
    }

    // Adds the tokens of bins first ... last with keys low ... high to the list (there is room); returns their number.
    __device__ __forceinline__ int collect(const sample_scale &s, int first, int last, uint64_t low, uint64_t high) {
        if (threadIdx.x == 0) sh.nlist = 0;
        __syncthreads();
        const float lowest = (float)(SAMPLE_ABOVE - 1 - last) * 0.0625f, highest = first == 0 ? INFINITY : (float)(SAMPLE_ABOVE - first) * 0.0625f;
        each([&](int i, float l) {
            const float y = s.y(l);
            if (!(y >= lowest && y < highest)) return;
            const uint64_t key = sample_key(l, i);
            if (key < low || key > high) return;
            const uint32_t at = atomicAdd(&sh.nlist, 1u);
            if (at < SAMPLE_LIST) sh.list[at] = key;
        });
        __syncthreads();
        return (int)list_size();
    }

    // The key in `bin` at which a limit is reached on top of c, m; the weight up to and with it in m.  The bin's keys are split
    // into 2048 parts, the part with the limit again, until 256 or fewer are left, each of which is compared with all (the range of
    // keys shrinks to a 1024th at least, and no two keys are equal, so it ends after six rounds at most).  They come from the list
    // of `listed` keys, or, where the bin has too many for it (listed < 0), from the row until the rest fits.  (201 keys: 4 us, by a
    // round of parts and a sort of 64 by one wave 7 us.)
    __device__ __forceinline__ uint64_t find_cut(const sample_scale &s, int bin, int listed, const sample_limit &limit, uint32_t c, double &m) {
        const int tid = threadIdx.x, octave = bin_octave(bin);
        auto in_bin = [&](float y) { return bin_of(y) == bin; };
        auto from_list = [&](auto f) {
            for (int i = tid; i < listed; i += SAMPLE_THREADS) {
                const uint64_t key = sh.list[i];
                const float y = s.y(sample_key_logit(key));
                if (in_bin(y)) f(key, y);
            }
        };
        auto from_row = [&](auto f) {
            each([&](int i, float l) {
                const float y = s.y(l);
                if (in_bin(y)) f(sample_key(l, i), y);
            });
        };
        uint64_t lo = KEY_EMPTY, hi = 0;
        auto range = [&](uint64_t key, float) {
            lo = min(lo, key);
            hi = max(hi, key);
        };
        uint64_t low = 0, high = KEY_EMPTY;
        uint32_t n = bin_count(sh.bins[bin]);
        if (n > SAMPLE_LAST) {
            if (listed >= 0) from_list(range);
            else from_row(range);
            low = block_min(lo);
            high = ~block_min(~hi);
        }
        while (n > SAMPLE_LAST) {
            int shift = 0;
            while ((high - low) >> shift >= SAMPLE_BINS) ++shift;
            __syncthreads();
            for (int b = tid; b < SAMPLE_BINS; b += SAMPLE_THREADS) sh.fine[b] = 0;
            __syncthreads();
            auto add = [&](uint64_t key, float y) {
                if (key >= low && key <= high) atomicAdd(&sh.fine[(key - low) >> shift], bin_word(y));
            };
            if (listed >= 0) from_list(add);
            else from_row(add);
            __syncthreads();
            const int part = find_bin(sh.fine, limit, c, m, [&](int) { return octave; });
            if (part >= SAMPLE_BINS) {   // reached by the sums of the bins, but not by these, which round differently: the last key
                m = limit.mass;
                return high;
            }
            n = bin_count(sh.fine[part]);
            low += (uint64_t)part << shift;
            high = min(high, low + ((uint64_t)1 << shift) - 1);
            if (listed < 0 && n <= SAMPLE_LIST) listed = collect(s, bin, bin, low, high);
        }
        if (listed < 0) listed = collect(s, bin, bin, low, high);   // (never: such a bin has more keys than the list)
        if (tid == 0) sh.nlast = 0;
        __syncthreads();
        from_list([&](uint64_t key, float) {
            if (key < low || key > high) return;
            const uint32_t at = atomicAdd(&sh.nlast, 1u);
            if (at < SAMPLE_LAST) sh.last[at] = key;
        });
        __syncthreads();
        // ranks: of a few keys by the wave that goes on with them, else by as many lanes for each key as there are
        const int left = (int)min(sh.nlast, (uint32_t)SAMPLE_LAST);
        if (left <= 16) {
            if (tid < 64) {
                const uint64_t mine = sh.last[tid & 15];
                int rank = 0;
                for (int i = 0; i < left; ++i) rank += read_lane(mine, i) < mine;
                __builtin_amdgcn_wave_barrier();
                if (tid < left) sh.sorted[rank] = mine;
                __builtin_amdgcn_wave_barrier();
            }
        } else {
            const int lanes = left <= 64 ? 16 : 4, at = tid / lanes;
            if (at < left) {   // (the lanes of a key together)
                const uint64_t mine = sh.last[at];
                int rank = 0;
                for (int i = tid & (lanes - 1); i < left; i += lanes) rank += sh.last[i] < mine;
                for (int d = lanes / 2; d > 0; d /= 2) rank += __shfl_xor(rank, d);
                if ((tid & (lanes - 1)) == 0) sh.sorted[rank] = mine;
            }
            __syncthreads();
        }
        if (tid < 64) {
            // (a lane has one key, or some one after the other)
            constexpr int EACH = SAMPLE_LAST / 64;
            const int each = left <= 64 ? 1 : EACH;
            double upto[EACH], sum = 0.;
#pragma unroll
            for (int e = 0; e < EACH; ++e) {
                if (e < each && each * tid + e < left) sum += (double)s.weight(s.y(sample_key_logit(sh.sorted[each * tid + e])));
                upto[e] = sum;
            }
            const double before_lane = wave_scan<op_add>(sum) - sum + m;
            int reached = EACH;
#pragma unroll
            for (int e = EACH - 1; e >= 0; --e)
                if (e < each && each * tid + e < left && limit.reached(c + each * tid + e + 1, before_lane + upto[e])) reached = e;
            const uint64_t there = __ballot(reached < EACH);
            if (!there) reached = (left - 1) % each;   // (not reached: rounding, the last one)
            if (tid == (there ? __ffsll((unsigned long long)there) - 1 : (left - 1) / each)) {
                sh.cut = sh.sorted[each * tid + reached];
                double all = upto[0];
#pragma unroll
                for (int e = 1; e < EACH; ++e)
                    if (e <= reached) all = upto[e];
                sh.mass = before_lane + all;
            }
        }
        __syncthreads();
        m = sh.mass;
        const uint64_t cut = sh.cut;
        return cut;
    }

    // the reference: the largest of a first look, or of all where that is needed
    __device__ __forceinline__ float largest_of_look() {
        float high = -INFINITY;
#pragma unroll
        for (int e = 0; e < SAMPLE_V; ++e) high = fmaxf(high, look[e]);
        return block_max(high);
    }
    __device__ __forceinline__ float largest() {
        float high = -INFINITY;
        each([&](int, float l) { high = fmaxf(high, l); });
        return block_max(high);
    }

    // The whole row by this block.
    __device__ __forceinline__ void run() {
        const int tid = threadIdx.x;
        const float t = a.temperature ? a.temperature[r] : 1.f;
        const int64_t top_k = a.top_k ? a.top_k[r] : 0;
        const float top_p = a.top_p ? a.top_p[r] : 1.f, min_p = a.min_p ? a.min_p[r] : 0.f;
        const bool greedy = !(t > 0.f) || min_p > 1.f;   // (the first token alone stays)
        const bool by_k = top_k > 0 && top_k < a.vocab, by_p = top_p < 1.f;
        whole_row();
        load_look();
        if (greedy) {
            const uint64_t first = first_key();
            return sample_key_logit(first) > -INFINITY ? done((int64_t)(uint32_t)first, 0.f) : done(-1, -INFINITY);
        }
        float ref = -INFINITY, top = 0.f;
        if (!(min_p > 0.f && !by_k && !by_p)) ref = largest_of_look();
        if (!(ref > -INFINITY)) ref = largest();
        if (!(ref > -INFINITY)) return done(-1, -INFINITY);
        const float inv = 1.f / t;
        sample_scale s(ref, inv);
        // (without limits, min_p takes the largest logit for the reference: of weight 1)
        float least = min_p > 0.f ? fmaxf(log2f(min_p), SAMPLE_LEAST) : SAMPLE_LEAST;
        uint64_t cut = KEY_EMPTY;
        sample_limit limit = {};
        uint32_t c = 0;       // tokens and weight before the bin of the cut
        double m = 0.;
        int listed = 0;       // keys in the list
        int cut_bin = SAMPLE_BINS;
        bool on_list = false, later = false;   // the list holds all that stay; the cut is to be found after the pass over the row

        if (by_k || by_p) {
            // (half as many again as top_k asks for, or some, for top_p, which may ask for any number)
            const uint32_t wanted = by_k ? (uint32_t)min((int64_t)(SAMPLE_LIST / 2), top_k + top_k / 2 + 64) : SAMPLE_LIST / 4;
            int complete;   // the list holds the tokens of all bins up to this one; -1: of none
            for (int round = 0; round < 2; ++round) {   // (the second with the largest logit for the reference)
                fill_bins(s, wanted, top, complete);
                if (top <= SAMPLE_TOP || round == 1) break;
                ref = largest();
                s = sample_scale(ref, inv);
            }
            least = min_p > 0.f ? fmaxf(top + log2f(min_p), SAMPLE_LEAST) : SAMPLE_LEAST;
            listed = complete >= 0 ? (int)sh.nlist : 0;
            // each limit in turn: its bin, the list if it is not there, its cut
            double all = block_sum(bin_mass(sh.bins[2 * tid], bin_octave(2 * tid)) + bin_mass(sh.bins[2 * tid + 1], bin_octave(2 * tid + 1)));
            for (int step = 0; step < 2; ++step) {
                if (step == 0 ? !by_k : !by_p) continue;
                limit.by_count = step == 0;
                limit.count = (uint32_t)top_k;
                limit.mass = fmax((double)top_p * all, 1e-300);   // a token stays while the weights before it are below: up to the one that reaches it
                c = 0;
                m = 0.;
                const int bin = find_bin(sh.bins, limit, c, m, bin_octave);
                if (bin >= SAMPLE_BINS) continue;   // not reached: all stay
                cut_bin = bin;
                int have = listed;
                if (bin > complete) {
                    const uint32_t n = bin_count(sh.bins[bin]);
                    const bool fits = c + n <= SAMPLE_LIST;
                    if (!fits && n <= SAMPLE_LIST && (step == 1 || !by_p)) {
                        later = true;
                        break;
                    }
                    have = n > SAMPLE_LIST ? -1 : collect(s, fits ? 0 : bin, bin, 0, KEY_EMPTY);
                    listed = fits ? have : 0;
                    complete = fits ? bin : -1;
                }
                cut = min(cut, find_cut(s, bin, have, limit, c, m));
                all = m;
            }
            on_list = complete >= 0 && cut != KEY_EMPTY;
        }
        race best;
        double mass = 0.;
        if (!on_list) {
            // from the row: what lies before the bin of the cut stays, the bin itself is listed for later, or the cut is there
            const float lower = cut_bin < SAMPLE_BINS ? (float)(SAMPLE_ABOVE - 1 - cut_bin) * 0.0625f : -INFINITY;
            const float upper = cut_bin < SAMPLE_BINS ? lower + 0.0625f : -INFINITY;
            // (without limits, the second round with the largest logit for the reference; limits hold for the reference that they have)
            for (int round = 0; round < 2; ++round) {
                const float high = draw(s, upper, lower, least, later ? KEY_EMPTY : cut, cut_bin >= SAMPLE_BINS || c > (uint32_t)a.vocab / 32, best, mass);
                if (high <= SAMPLE_TOP || by_k || by_p || round == 1) break;
                s = sample_scale(largest(), inv);
                best = race();
                mass = 0.;
            }
            mass = block_sum(mass);
            if (later) {
                listed = (int)list_size();
                cut = min(cut, find_cut(s, cut_bin, listed, limit, c, m));
            }
        }
        if (on_list || later) mass += draw_list(s, listed, least, top, cut, best);
        finish(winner(best), s, mass);
    }

    // One part of a row without filters.
    __device__ __forceinline__ void run_part(int part, int parts, sample_part *results) {
        const int tid = threadIdx.x;
        sample_part &result = results[r * parts + part];
        race best;
        double mass = 0.;
        const float t = a.temperature ? a.temperature[r] : 1.f;
        if (!(t > 0.f)) {
            part_of_row(part, parts);
            const uint64_t key = first_key();
            if (tid == 0) result = {key, 0., 0.f};
            return;
        }
        // every part looks at the same beginning of the row, for the same reference
        whole_row();
        load_look();
        float ref = largest_of_look();
        if (!(ref > -INFINITY)) ref = largest();
        float high = -INFINITY;
        if (ref > -INFINITY) {
            part_of_row(part, parts);
            load_look();
            high = draw(sample_scale(ref, 1.f / t), -INFINITY, -INFINITY, SAMPLE_LEAST, 0, true, best, mass);
        }
        mass = block_sum(mass);
        const uint64_t key = winner(best);
        if (tid == 0) result = {key, mass, high};
    }

    // Joins the parts of a row.
    __device__ __forceinline__ void join(int parts, const sample_part *results) {
        uint64_t best = KEY_EMPTY;
        double mass = 0.;
        bool far = false;   // a part's largest logit lies too far above the reference
        for (int part = 0; part < parts; ++part) {
            const sample_part &x = results[r * parts + part];
            best = min(best, x.key);
            mass += x.mass;
            far |= x.high > SAMPLE_TOP;
        }
        if (far) return run();
        whole_row();
        const float t = a.temperature ? a.temperature[r] : 1.f;
        if (!(t > 0.f)) return sample_key_logit(best) > -INFINITY ? done((int64_t)(uint32_t)best, 0.f) : done(-1, -INFINITY);
        load_look();
        float ref = largest_of_look();
        if (!(ref > -INFINITY)) ref = largest();
        if (!(ref > -INFINITY)) return done(-1, -INFINITY);
        finish(best, sample_scale(ref, 1.f / t), mass);
    }
};

template <class T> __device__ __forceinline__ sample_row<T> row_of(const sample_args &a, sample_shared &sh, int64_t r) {
    return {a, sh, (const T *)a.logits + r * a.row_stride, a.noise ? a.noise + r * a.noise_stride : nullptr, r, 0, 0, 0, 0, 0, {}};
}
template <class T> __global__ __launch_bounds__(SAMPLE_THREADS) void sample_kernel(sample_args a) {
    __shared__ sample_shared sh;
    row_of<T>(a, sh, blockIdx.x).run();
}
template <class T> __global__ __launch_bounds__(SAMPLE_THREADS) void sample_parts_kernel(sample_args a, sample_part *results) {
    __shared__ sample_shared sh;
    row_of<T>(a, sh, blockIdx.y).run_part(blockIdx.x, gridDim.x, results);
}
template <class T> __global__ __launch_bounds__(SAMPLE_THREADS) void sample_join_kernel(sample_args a, int parts, const sample_part *results) {
    __shared__ sample_shared sh;
    row_of<T>(a, sh, blockIdx.x).join(parts, results);
}

template <class T> static int sample_typed(pq_ctx *ctx, const sample_args &a, int rows) {
    // Rows without filters that leave half of the compute units idle are drawn in parts of 8192 tokens or more (33 rows of 50 021:
    // 11.8 us in parts, 14.1 us by a block each; 8 rows of 131 072: 12.1 and 22.9 us).  Sharing the last pass of rows with
    // filters was no gain: 256 rows of 131 072 took 97 us with it, 73 us without.
    if (!a.top_k && !a.top_p && !a.min_p && 2 * rows <= ctx->num_cu && a.vocab > 8192) {
        const int most = (a.vocab + 8191) / 8192, room = ctx->num_cu / rows;
        const int parts = most < room ? most : room;
        if (const int rc = buf_reserve(ctx, &ctx->read_ws, (size_t)rows * parts * sizeof(sample_part), "the draw of tokens")) return rc;
        sample_part *const results = (sample_part *)ctx->read_ws.p;
        sample_parts_kernel<T><<<dim3(parts, rows), SAMPLE_THREADS, 0, ctx->stream>>>(a, results);
        sample_join_kernel<T><<<rows, SAMPLE_THREADS, 0, ctx->stream>>>(a, parts, results);
    } else {
        sample_kernel<T><<<rows, SAMPLE_THREADS, 0, ctx->stream>>>(a);
    }
    PQ_HIP(ctx, hipGetLastError());
    return PQ_OK;
}

int launch_sample_tokens(pq_ctx *ctx, const void *logits, int elem, int64_t row_stride, int rows, int vocab, const float *noise,
                         int64_t noise_stride, const float *temperature, const int32_t *top_k, const float *top_p,
                         const float *min_p, int64_t *tokens, float *logprobs) {
    const sample_args a = {logits, row_stride, noise_stride, vocab, noise, temperature, top_p, min_p, top_k, tokens, logprobs};
    if (elem == PQ_ELEM_F32) return sample_typed<float>(ctx, a, rows);
    if (elem == PQ_ELEM_F16) return sample_typed<_Float16>(ctx, a, rows);
    return sample_typed<__bf16>(ctx, a, rows);
}

}  // namespace pq
