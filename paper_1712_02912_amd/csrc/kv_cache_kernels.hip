// The paged cache of the reading step: the plan (pq_kv_plan) and the append (pq_kv_append).
#include <limits.h>

#include "kv_append.h"
#include "wave_sums.h"

namespace pq {

// ---- plan -------------------------------------------------------------------------------------------
//
// Two prefix sums over the requests (new tokens, needed blocks), then one thread per new token that finds its request by
// bisection.  A fresh block begins with a new token, so the thread of that token also writes the block's entry in the
// table; tokens of fresh blocks take the block from free_blocks, never from the table, so no thread reads what another
// one writes.  There is next to nothing to move (12 bytes a token); what counts is that it is one launch: every block
// forms the sums for itself (PLAN_MAX requests: four rounds of its threads), rather than wait for another kernel.
// Bound by latency: lengths, two sums over the block, a bisection in shared memory, a table's entry, one after the other.  64
// requests of one token 3.3 us (a launch of nothing: about 2.5), 1777 requests of 1 to 611 tokens 8.4 us.
constexpr int PLAN_THREADS = 1024;
constexpr int PLAN_MAX = 4096;   // requests whose sums a block keeps in shared memory
static_assert(PLAN_THREADS / 64 == 16, "the waves' sums are joined by one row of 16 lanes");

struct plan_args {
    const int32_t *new_lens, *cached_lens;
    int32_t *tables;
    const int32_t *free_blocks;
    int nreq, width, nfree;
    fast_div by_block;
    int64_t ntokens;
    int32_t *cu, *kv, *positions;
    int64_t *slots;
    int32_t *taken;
};
// of every request: tokens and needed blocks before it (one more of each behind the last), its cached tokens or -1 (refused)
struct plan_sums {
    int32_t *tokens, *blocks, *cached;
};

__device__ __forceinline__ int32_t clamp_i32(uint64_t x) { return (int32_t)min(x, (uint64_t)INT_MAX); }
// ceil(n / block) for 0 <= n < 2^31
__device__ __forceinline__ uint32_t plan_blocks(const plan_args &a, uint32_t n) {
    const uint32_t q = a.by_block.div(n);
    return q + (q * a.by_block.d < n);
}

// The sums, by one block; the block that `writes` also writes the results that belong to requests.
__device__ __forceinline__ void plan_add_up(const plan_args &a, const plan_sums &x, bool writes) {
    __shared__ uint64_t wave_sum[2][2][16];
    __shared__ int taken;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    uint64_t carry_t = 0, carry_b = 0;
    int mine = 0, turn = 0;
    if (tid == 0) x.tokens[0] = x.blocks[0] = taken = 0;
    for (int base = 0; base < a.nreq; base += PLAN_THREADS, turn ^= 1) {
        const int r = base + tid;
        uint32_t fresh = 0, cached = 0, need = 0;
        bool fits = false;
        if (r < a.nreq) {
            fresh = (uint32_t)max(a.new_lens[r], 0);
            const int32_t held = a.cached_lens[r];   // (negative: refused before, and again)
            cached = (uint32_t)max(held, 0);
            const uint32_t all = fresh + cached;   // (below 2^32)
            const uint32_t full = all <= INT_MAX ? plan_blocks(a, all) : UINT_MAX;
            fits = held >= 0 && full <= (uint32_t)a.width;
            need = fits ? full - plan_blocks(a, cached) : 0;
        }
        uint64_t t = wave_scan<op_add>((uint64_t)fresh), b = wave_scan<op_add>((uint64_t)need);
        if (lane == 63) {
            wave_sum[turn][0][wave] = t;
            wave_sum[turn][1][wave] = b;
        }
        __syncthreads();
        const uint64_t tw = row_scan<op_add>(wave_sum[turn][0][lane & 15]) + carry_t, bw = row_scan<op_add>(wave_sum[turn][1][lane & 15]) + carry_b;
        t += wave > 0 ? read_lane(tw, wave - 1) : carry_t;
        b += wave > 0 ? read_lane(bw, wave - 1) : carry_b;
        carry_t = read_lane(tw, 15);
        carry_b = read_lane(bw, 15);
        if (r < a.nreq) {
            const bool served = fits && b <= (uint64_t)a.nfree && t <= (uint64_t)a.ntokens;
            x.tokens[r + 1] = clamp_i32(t);
            x.blocks[r + 1] = clamp_i32(b);
            x.cached[r] = served ? (int32_t)cached : -1;
            if (writes) {
                if (a.cu != x.tokens) a.cu[r + 1] = clamp_i32(t);
                a.kv[r] = served ? (int32_t)(cached + fresh) : -1;
                if (served) mine += (int)need;
            }
        }
    }
    __syncthreads();
    if (writes) {
        if (mine) atomicAdd(&taken, mine);   // (whole numbers: the order does not matter)
        __syncthreads();
        if (tid == 0) {
            if (a.cu != x.tokens) a.cu[0] = 0;
            *a.taken = taken;
        }
    }
}

__device__ __forceinline__ void plan_token(const plan_args &a, const plan_sums &x, int64_t t) {
    int32_t position = -1;
    int64_t slot = -1;
    if (t < x.tokens[a.nreq]) {
        int low = 0, high = a.nreq;   // the request with tokens[low] <= t < tokens[low + 1]
        while (high - low > 1) {
            const int mid = (low + high) >> 1;
            if (x.tokens[mid] <= t) low = mid;
            else high = mid;
        }
        const int32_t cached = x.cached[low];
        if (cached >= 0) {
            position = cached + (int32_t)(t - x.tokens[low]);
            const int b = (int)a.by_block.d, column = (int)a.by_block.div((uint32_t)position), have = (int)plan_blocks(a, (uint32_t)cached);
            int32_t *entry = a.tables + (size_t)low * a.width + column;
            int32_t block;
            if (column < have) {
                block = *entry;
            } else {
                block = a.free_blocks[x.blocks[low] + column - have];
                if (position == column * b) *entry = block;
            }
            slot = (int64_t)block * b + (position - column * b);
        }
    }
    a.positions[t] = position;
    a.slots[t] = slot;
}

__global__ __launch_bounds__(PLAN_THREADS) void kv_plan_kernel(plan_args a) {
    __shared__ int32_t tokens[PLAN_MAX + 1], blocks[PLAN_MAX + 1], cached[PLAN_MAX];
    const plan_sums x = {tokens, blocks, cached};
    plan_add_up(a, x, blockIdx.x == 0);
    const int64_t step = (int64_t)gridDim.x * PLAN_THREADS;
    for (int64_t t = (int64_t)blockIdx.x * PLAN_THREADS + threadIdx.x; t < a.ntokens; t += step) plan_token(a, x, t);
}

// more requests: the sums by one block first, then the tokens
__global__ __launch_bounds__(PLAN_THREADS) void kv_plan_sums_kernel(plan_args a, plan_sums x) { plan_add_up(a, x, true); }
__global__ __launch_bounds__(PLAN_THREADS) void kv_plan_tokens_kernel(plan_args a, plan_sums x) {
    const int64_t step = (int64_t)gridDim.x * PLAN_THREADS;
    for (int64_t t = (int64_t)blockIdx.x * PLAN_THREADS + threadIdx.x; t < a.ntokens; t += step) plan_token(a, x, t);
}

int launch_kv_plan(pq_ctx *ctx, const int32_t *new_lens, const int32_t *cached_lens, int nreq, int32_t *tables, int width,
                   const int32_t *free_blocks, int nfree, int block_size, int64_t ntokens, int32_t *cu, int32_t *kv,
                   int32_t *positions, int64_t *slots, int32_t *taken) {
    const plan_args a = {new_lens, cached_lens, tables, free_blocks, nreq, width, nfree, fast_div((uint32_t)block_size), ntokens, cu, kv, positions, slots, taken};
    // one token per thread up to two blocks per compute unit, each of which forms the sums
    const int64_t wanted = (ntokens + PLAN_THREADS - 1) / PLAN_THREADS;
    const int grid = (int)(wanted < 1 ? 1 : wanted > 2 * ctx->num_cu ? 2 * ctx->num_cu : wanted);
    if (nreq <= PLAN_MAX) {
        kv_plan_kernel<<<grid, PLAN_THREADS, 0, ctx->stream>>>(a);
    } else {
        const int rc = buf_reserve(ctx, &ctx->read_ws, 2 * ((size_t)nreq + 1) * sizeof(int32_t), "the plan of a paged cache");
        if (rc) return rc;
        const plan_sums x = {cu, (int32_t *)ctx->read_ws.p, (int32_t *)ctx->read_ws.p + nreq + 1};
        kv_plan_sums_kernel<<<1, PLAN_THREADS, 0, ctx->stream>>>(a, x);
        kv_plan_tokens_kernel<<<grid, PLAN_THREADS, 0, ctx->stream>>>(a, x);
    }
    PQ_HIP(ctx, hipGetLastError());
    return PQ_OK;
}

// ---- append -----------------------------------------------------------------------------------------
//
// By groups of lanes that hold a head each (kv_append.h).  Bound by memory: 16 384 tokens of
// 32 + 8 + 8 heads of 128 dimensions, bf16, 411 MB in 76.5 us = 5.4 TB/s (a large copy on this card: 5.1); 4099 tokens of 36 heads
// of 80 dimensions, f32, 95 MB in 24 us = 3.9 TB/s.  Four heads one after the other in a group of lanes, all read before the first
// is written and the rotation's row read once for them, were slower (93 us).
template <class T, int V, bool PAIRS> __global__ __launch_bounds__(APPEND_THREADS) void kv_append_kernel(append_args a, int gl) {
    append_rows<T, V, PAIRS>(a, gl, (int64_t)blockIdx.x * APPEND_THREADS + threadIdx.x);
}
template <class T, bool PAIRS> __global__ __launch_bounds__(APPEND_THREADS) void kv_append_general_kernel(append_args a) {
    append_rows_general<T, PAIRS>(a, blockIdx.x);
}

template <class T, int V, bool PAIRS> static int append_vector(pq_ctx *ctx, const append_args &a) {
    int gl = 1;
    while (gl < a.cache.dim / (2 * V)) gl *= 2;
    const int64_t grid = (a.ntokens * a.rows * gl + APPEND_THREADS - 1) / APPEND_THREADS;
    if (!grid_fits(grid, APPEND_THREADS)) return fail(ctx, PQ_EUNSUPPORTED, "kv_append: %lld tokens in one call", (long long)a.ntokens);
    kv_append_kernel<T, V, PAIRS><<<(int)grid, APPEND_THREADS, 0, ctx->stream>>>(a, gl);
    PQ_HIP(ctx, hipGetLastError());
    return PQ_OK;
}

// elements per access that every row's address, the pairs and the rest of the head allow
static int append_width(const append_args &a, int most) {
    const pq_kv_cache &c = a.cache;
    const size_t e = elem_bytes(c.elem);
    uint64_t bits = (uint64_t)(a.rot / 2) * e | (uint64_t)((c.dim - a.rot) / 2) * e | (uint64_t)(uintptr_t)c.keys | (uint64_t)(uintptr_t)c.values;
    for (int i = 0; i < 3; ++i) bits |= (uint64_t)c.key_strides[i] * e | (uint64_t)c.value_strides[i] * e;
    for (const pq_heads *h : {&a.q, &a.k, &a.v})
        if (h != &a.q || a.q_heads > 0) bits |= (uint64_t)(uintptr_t)h->p | (uint64_t)h->token_stride * e | (uint64_t)h->head_stride * e;
    if (a.q_heads > 0) bits |= (uint64_t)(uintptr_t)a.q_out | (uint64_t)c.dim * e;
    // the tables and weights are read by the same number of fp32 elements
    uint64_t wide = (uint64_t)(uintptr_t)a.q_weight | (uint64_t)(uintptr_t)a.k_weight;
    if (a.rot > 0) wide |= (uint64_t)(uintptr_t)a.cos_table | (uint64_t)(uintptr_t)a.sin_table | (uint64_t)(a.rot / 2) * 4;
    int v = most;
    while (v > 1 && (bits % (v * e) != 0 || wide % (v * 4) != 0)) v /= 2;
    return v;
}

template <class T, bool PAIRS> static int append_typed(pq_ctx *ctx, const append_args &a) {
    constexpr int most = 16 / sizeof(T);
    const int v = append_width(a, most);
    if (a.cache.dim <= 64 * 2 * v) {   // the units of a head fit a wave
        if (v == 8 && most == 8) return append_vector<T, most, PAIRS>(ctx, a);
        if (v >= 4) return append_vector<T, 4, PAIRS>(ctx, a);
    }
    const int64_t grid = (a.ntokens * a.rows + APPEND_THREADS / 64 - 1) / (APPEND_THREADS / 64);
    if (!grid_fits(grid, APPEND_THREADS)) return fail(ctx, PQ_EUNSUPPORTED, "kv_append: %lld tokens in one call", (long long)a.ntokens);
    kv_append_general_kernel<T, PAIRS><<<(int)grid, APPEND_THREADS, 0, ctx->stream>>>(a);
    PQ_HIP(ctx, hipGetLastError());
    return PQ_OK;
}

int launch_kv_append(pq_ctx *ctx, const pq_kv_cache *cache, const pq_heads *q, int q_heads, const pq_heads *k, const pq_heads *v,
                     int64_t ntokens, const int32_t *positions, const int64_t *slots, const float *cos_table,
                     const float *sin_table, int64_t max_positions, int rot, int pairs, int norm, const float *q_weight,
                     const float *k_weight, float eps, void *q_out) {
    append_args a = {};
    if (q_heads > 0) a.q = *q;
    a.k = *k;
    a.v = *v;
    a.cache = *cache;
    a.positions = positions;
    a.slots = slots;
    a.cos_table = cos_table;
    a.sin_table = sin_table;
    a.q_weight = q_weight;
    a.k_weight = k_weight;
    a.q_out = q_out;
    a.ntokens = ntokens;
    a.max_positions = max_positions;
    a.eps = eps;
    a.q_heads = q_heads;
    a.rot = rot;
    a.norm = norm;
    a.rows = q_heads + 2 * cache->heads;
    switch (cache->elem) {
    case PQ_ELEM_F32: return pairs ? append_typed<float, true>(ctx, a) : append_typed<float, false>(ctx, a);
    case PQ_ELEM_F16: return pairs ? append_typed<_Float16, true>(ctx, a) : append_typed<_Float16, false>(ctx, a);
    default: return pairs ? append_typed<__bf16, true>(ctx, a) : append_typed<__bf16, false>(ctx, a);
    }
}

}  // namespace pq
