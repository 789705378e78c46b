// The append to a paged cache of 8 bits (pq_kv_append8).
#include <limits.h>

#include "e4m3.h"
#include "kv_append.h"

namespace pq {

struct append8_args {
    append_args in;       // (its cache: sizes alone)
    pq_kv_cache8 cache;
};

// The slot of a token that is written, -1 for others.
__device__ __forceinline__ int64_t append8_slot(const append8_args &a, int64_t t) {
    const int32_t p = a.in.positions[t];
    const int64_t slot = a.in.slots[t];
    return p >= 0 && (a.in.rot == 0 || p < a.in.max_positions) && slot >= 0 && slot < a.cache.nblocks * a.cache.block_size ? slot : -1;
}

// A run: tokens one after the other whose slots follow each other within a block.
struct append8_run {
    int64_t block;
    int place, count;   // of its first token; its tokens (0: token t does not begin a run)
};
// by a whole wave
__device__ __forceinline__ append8_run append8_find(const append8_args &a, int64_t t) {
    const int lane = threadIdx.x & 63;
    append8_run r = {0, 0, 0};
    const int64_t slot = append8_slot(a, t);
    if (slot < 0) return r;
    r.block = slot / a.cache.block_size;
    r.place = (int)(slot - r.block * a.cache.block_size);
    if (r.place > 0 && t > 0 && append8_slot(a, t - 1) == slot - 1) return r;
    const int most = (int)min((int64_t)(a.cache.block_size - r.place), a.in.ntokens - t);
    while (r.count < most) {
        const int i = r.count + lane;
        const uint64_t no = ~__ballot(i < most && append8_slot(a, t + i) == slot + i);
        if (no) {
            r.count += __ffsll((unsigned long long)no) - 1;
            break;
        }
        r.count += 64;
    }
    return r;
}

// ---- any layout ---------------------------------------------------------------------------------------
//
// One wave for each token and head (of the cache: one for keys, one for values), which holds the run that begins there.  It goes over
// the run's rows twice, for the largest element and to write them; no row is kept between.
template <class T, bool PAIRS> __device__ __forceinline__ void append8_general_head(const append8_args &a, int64_t t, int h, bool is_key) {
    const append8_run run = append8_find(a, t);
    if (run.count == 0) return;
    const int lane = threadIdx.x & 63, dim = a.cache.dim, rot = is_key ? a.in.rot : 0;
    const pq_heads &from = is_key ? a.in.k : a.in.v;
    const int64_t *strides = is_key ? a.cache.key_strides : a.cache.value_strides;
    uint8_t *const block = (uint8_t *)(is_key ? a.cache.keys : a.cache.values) + run.block * strides[0] + h * strides[2];
    float *const scale = (is_key ? a.cache.key_scales : a.cache.value_scales) + run.block * a.cache.heads + h;

    // f(place, unit's first, unit's second, values) for all pairs of elements of the run
    auto each = [&](auto f) {
        for (int i = 0; i < run.count; ++i) {
            const T *const row = (const T *)from.p + (t + i) * from.token_stride + h * from.head_stride;
            double r = 1.0;
            if (is_key && a.in.norm) {
                double sum = 0.0;
                for (int e = lane; e < dim; e += 64) sum += (double)(float)row[e] * (double)(float)row[e];
                for (int d = 32; d > 0; d /= 2) sum += __shfl_xor(sum, d);
                r = 1.0 / sqrt(sum / (double)dim + (double)a.in.eps);
            }
            for (int u = lane; u < dim / 2; u += 64) {
                const append_unit<1, PAIRS> unit(u, rot);
                double x[1] = {(double)(float)row[unit.first]}, y[1] = {(double)(float)row[unit.second]};
                if (is_key && a.in.norm) {
                    x[0] = x[0] * r * (a.in.k_weight ? (double)a.in.k_weight[unit.first] : 1.0);
                    y[0] = y[0] * r * (a.in.k_weight ? (double)a.in.k_weight[unit.second] : 1.0);
                }
                if (unit.angle >= 0) {
                    const int64_t at = (int64_t)a.in.positions[t + i] * (rot / 2) + unit.angle;
                    const double c[1] = {(double)a.in.cos_table[at]}, s[1] = {(double)a.in.sin_table[at]};
                    append_turn<1, PAIRS>(x, y, c, s);
                }
                f(run.place + i, unit.first, unit.second, (float)x[0], (float)y[0]);
            }
        }
    };
    float amax = 0.f;
    each([&](int, int, int, float x, float y) { amax = fmaxf(amax, fmaxf(finite_size(x), finite_size(y))); });
    for (int d = 32; d > 0; d /= 2) amax = fmaxf(amax, __shfl_xor(amax, d));
    const int before = run.place > 0 ? scale_exponent(*scale) : LEAST_EXPONENT, e = max(before, exponent_for(amax));
    if (run.place > 0 && e > before)
        for (int p = 0; p < run.place; ++p)
            for (int i = lane; i < dim; i += 64) {
                uint8_t *const at = block + p * strides[1] + i;
                *at = (uint8_t)e4m3_of(ldexpf((float)e4m3{*at}, before - e), 0.f);
            }
    each([&](int place, int first, int second, float x, float y) {
        const uint32_t codes = e4m3_of(ldexpf(x, -e), ldexpf(y, -e));
        block[place * strides[1] + first] = (uint8_t)codes;
        block[place * strides[1] + second] = (uint8_t)(codes >> 8);
    });
    if (lane == 0) *scale = scale_of(e);
}

template <class T, bool PAIRS> __global__ __launch_bounds__(APPEND_THREADS) void kv_append8_general_kernel(append8_args a, unsigned query_blocks) {
    if (blockIdx.x < query_blocks) {
        append_rows_general<T, PAIRS>(a.in, blockIdx.x);
        return;
    }
    const int64_t item = ((int64_t)(blockIdx.x - query_blocks) * APPEND_THREADS + threadIdx.x) / 64;
    const int heads = 2 * a.cache.heads;
    const int64_t t = item / heads;
    const int row = (int)(item - t * heads);
    if (t < a.in.ntokens) append8_general_head<T, PAIRS>(a, t, row % a.cache.heads, row < a.cache.heads);
}

template <class T, bool PAIRS> static int append8_typed(pq_ctx *ctx, const append8_args &a) {
    constexpr int WAVES = APPEND_THREADS / 64;
    const int64_t queries = (a.in.ntokens * a.in.q_heads + WAVES - 1) / WAVES, items = (a.in.ntokens * 2 * a.cache.heads + WAVES - 1) / WAVES;
    if (queries + items > INT_MAX) return fail(ctx, PQ_EUNSUPPORTED, "kv_append8: %lld tokens in one call", (long long)a.in.ntokens);
    kv_append8_general_kernel<T, PAIRS><<<(unsigned)(queries + items), APPEND_THREADS, 0, ctx->stream>>>(a, (unsigned)queries);
    PQ_HIP(ctx, hipGetLastError());
    return PQ_OK;
}

int launch_kv_append8(pq_ctx *ctx, const pq_kv_cache8 *cache, int elem, const pq_heads *q, int q_heads, const pq_heads *k, const pq_heads *v,
                      int64_t ntokens, const int32_t *positions, const int64_t *slots, const float *cos_table, const float *sin_table,
                      int64_t max_positions, int rot, int pairs, int norm, const float *q_weight, const float *k_weight, float eps,
                      void *q_out) {
    append8_args a = {};
    if (q_heads > 0) a.in.q = *q;
    a.in.k = *k;
    a.in.v = *v;
    a.in.cache.dim = cache->dim;
    a.in.positions = positions;
    a.in.slots = slots;
    a.in.cos_table = cos_table;
    a.in.sin_table = sin_table;
    a.in.q_weight = q_weight;
    a.in.k_weight = k_weight;
    a.in.q_out = q_out;
    a.in.ntokens = ntokens;
    a.in.max_positions = max_positions;
    a.in.eps = eps;
    a.in.q_heads = q_heads;
    a.in.rot = rot;
    a.in.norm = norm;
    a.in.rows = q_heads;   // (of a token, those that go to q_out)
    a.cache = *cache;
    switch (elem) {
    case PQ_ELEM_F32: return pairs ? append8_typed<float, true>(ctx, a) : append8_typed<float, false>(ctx, a);
    case PQ_ELEM_F16: return pairs ? append8_typed<_Float16, true>(ctx, a) : append8_typed<_Float16, false>(ctx, a);
    default: return pairs ? append8_typed<__bf16, true>(ctx, a) : append8_typed<__bf16, false>(ctx, a);
    }
}

}  // namespace pq
