// Attention of few rows per head of the cache (single tokens, and short chunks): at most 16 rows, which is one tile of the
// matrix cores.  Bound by memory: every key and value is read once and used for at most 16 rows.
//
// Scores are formed transposed, S^T = K Q^T: keys are rows of the first operand, which lanes load straight from the cache, 16
// bytes each, and a lane holds scores of one row of queries only.  The weights then are the second operand of
// O^T = V^T P^T as they lie in the registers (the order of the keys within a product is free, so V's keys are read in the
// order that the scores have).  V^T needs columns of what the cache holds in rows: values go through shared memory, each
// wave's through its own part, and are read back transposed.
//
// Work is cut by what it is, not by request: all keys of all requests and heads form one line of units of 128 keys, and every
// block takes an equal stretch of it, so contexts of any lengths fill the chip evenly.  A (request, head) that lies
// within one block is finished there; of others each block leaves a part (maximum, sum, weighted values), and a second kernel
// joins the parts, always in the same order.  (The block that leaves the last part could join them, without a second launch;
// but what makes the parts visible across the chip's eight caches writes these back and empties them, in every block: 364 us instead
// of 164 for the 64 tokens below.)
//
// 64 tokens over up to 8192 keys, 32 heads of 128 dimensions on 8, bf16: 823 MB in 160 us = 5.1 TB/s, and 6.6 us to join parts.
// One token over 131 038 keys: 537 MB in 108 us = 5.0 TB/s, and 6.6 us.  Two blocks for each compute unit, as many as registers
// allow (of 256 dimensions one): with one the 64 tokens take 175 us.  Short contexts are bound by latency: lengths, sums, the table's
// entry, keys, values one after the other, about 8 us before the first result.
//
// Over a cache of 8 bits (C = e4m3) lanes hold codes until they are multiplied or written to shared memory, four vector instructions for
// eight of them.  The same 64 tokens: 403 MB in 89 us = 4.5 TB/s, and 6 us to join parts; one token over 131 038 keys: 55 us, and
// 6.  Half the bytes are on their way at a time, and the chain of a tile (products, powers, transposed values) shows: waves wait 69 % of
// their cycles.  Two tiles at a time instead of one took 103 us, not 95: what they add to the chain is more than the bytes.
#pragma once
#include "kv_attention.h"

namespace pq {

constexpr int FEW_TILE = 32;     // keys that a wave takes at a time
constexpr int FEW_MAX = 1024;    // requests whose line a block adds up in shared memory

struct few_line {
    int unit;                // keys of a unit: FEW_TILE for each wave of a block
    bool each;               // a block for each (request, head), no line
    const int64_t *starts;   // [nreq + 1] units of one head before each request, where the block does not add them up itself
    int64_t *starts_out;     // the same, for the kernel that joins the parts
    float *parts, *stats;    // [blocks][2][rows][D], [blocks][2][rows][2]
    int blocks;
    int row_waves;           // waves that join the parts of a row
};

struct few_range {
    int fresh, held, keys, from;   // new tokens, those of them whose rows are computed
    int64_t units;
};
// Keys that the rows of a request see; a request without any that still has rows is one unit (its rows are written).
__device__ __forceinline__ few_range few_load(const attention_args &a, int unit, int r) {
    few_range x;
    x.fresh = a.cu[r + 1] - a.cu[r];
    x.held = attention_held(a, r);
    const int kv = attention_length(a, r);
    x.keys = max(0, attention_keys(a, r));
    x.from = a.window > 0 ? (int)max((int64_t)0, (int64_t)kv - x.fresh - a.window + 1) : 0;
    x.units = x.held <= 0 || !attention_is_few(a, x.held) ? 0 : max((int64_t)1, (int64_t)(((uint32_t)max(x.keys - x.from, 0) + unit - 1) / (uint32_t)unit));
    return x;
}

// Units of one head before every request, by one block of THREADS; starts: [nreq + 1].
template <int THREADS> __device__ __forceinline__ void few_starts(const attention_args &a, int unit, int64_t *starts) {
    __shared__ int64_t wave_sum[THREADS / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int64_t carry = 0;
    if (tid == 0) starts[0] = 0;
    for (int base = 0; base < a.nreq; base += THREADS) {
        int64_t u = base + tid < a.nreq ? few_load(a, unit, base + tid).units : 0;
        for (int d = 1; d < 64; d *= 2) {
            const int64_t v = __shfl_up((long long)u, d);
            if (lane >= d) u += v;
        }
        if (lane == 63) wave_sum[wave] = u;
        __syncthreads();
        u += carry;
        for (int w = 0; w < THREADS / 64; ++w) {
            if (w < wave) u += wave_sum[w];
            carry += wave_sum[w];
        }
        if (base + tid < a.nreq) starts[base + tid + 1] = u;
        __syncthreads();
    }
}
// The stretches of the line: the first total % blocks of them are one unit longer.
struct few_cut {
    int64_t each, longer;
    __device__ __forceinline__ few_cut(int64_t total, int blocks) {
        each = (uint64_t)total >> 32 ? total / blocks : (int64_t)((uint32_t)total / (uint32_t)blocks);
        longer = total - each * blocks;
    }
    __device__ __forceinline__ int64_t begin(int b) const { return each * b + min((int64_t)b, longer); }
    __device__ __forceinline__ int block_of(int64_t unit) const {   // the block that holds it
        const int64_t in_longer = longer * (each + 1);
        const uint64_t n = unit < in_longer ? unit : unit - in_longer, d = unit < in_longer ? each + 1 : each;
        return (int)((unit < in_longer ? 0 : longer) + (int64_t)(n >> 32 | d >> 32 ? n / d : (uint32_t)n / (uint32_t)d));
    }
};

// where keys and values of a lane's two places of a tile are, in elements (and their blocks, of which a cache of 8 bits has the scales)
struct few_places {
    int64_t k[2], v[2];
    int64_t block[2];
};

// A lane's share of a row in registers: of the queries' type D / 4 elements, eight at 8 g + 32 t for each product t; of 8 bits
// sixteen at 16 g + 64 u for two products, so that they come 16 bytes at a time, too, and eight at 8 g behind the last whole 64 (the
// order of the dimensions within the products is free, and the queries' is the same).
template <class C, int D> struct few_row {
    static constexpr int STEPS = D / 32;
    u32x4 x[STEPS];
    static __device__ __forceinline__ int dim(int t, int g) { return 32 * t + 8 * g; }
    __device__ __forceinline__ void load(const C *row, int g) {
#pragma unroll
        for (int t = 0; t < STEPS; ++t) x[t] = *(const u32x4 *)(row + dim(t, g));
    }
    template <class T> __device__ __forceinline__ u32x4 step(int t, float) const { return x[t]; }
};
template <int D> struct few_row<e4m3, D> {
    static constexpr int STEPS = D / 32;
    uint32_t x[2 * STEPS];
    static __device__ __forceinline__ int dim(int t, int g) { return t < STEPS / 2 * 2 ? 64 * (t / 2) + 16 * g + 8 * (t % 2) : 32 * t + 8 * g; }
    __device__ __forceinline__ void load(const e4m3 *row, int g) {
#pragma unroll
        for (int u = 0; u < STEPS / 2; ++u) {
            const u32x4 c = *(const u32x4 *)(row + 64 * u + 16 * g);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[4 * u + i] = c[i];
        }
        if constexpr (STEPS % 2 != 0) {
            const uint2 c = *(const uint2 *)(row + dim(STEPS - 1, g));
            x[2 * STEPS - 2] = c.x;
            x[2 * STEPS - 1] = c.y;
        }
    }
    template <class T> __device__ __forceinline__ u32x4 step(int t, float scale) const { return from_e4m3<T>(x[2 * t], x[2 * t + 1], scale); }
};

template <int D, int WAVES> constexpr int FEW_POOL = WAVES * FEW_TILE * lds_row<D>::bytes;

// The block's stretch of the line; pool: FEW_POOL bytes of shared memory.
template <class T, class C, int D, int WAVES> __device__ __forceinline__ void few_block(const attention_args &a, const few_line &line, int block, unsigned char *pool) {
    typedef lds_row<D> row;
    constexpr int THREADS = 64 * WAVES, UNIT = WAVES * FEW_TILE;
    constexpr int STEPS = D / 32;   // products over the dimensions
    constexpr int OUTS = D / 16;    // tiles of the result
    static_assert(FEW_TILE * row::bytes >= FEW_ROWS * D * 4, "results of a wave fit its part");
    __shared__ float stat[WAVES][FEW_ROWS][2];
    __shared__ int64_t own_starts[FEW_MAX + 1];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 15, g = lane >> 4;
    unsigned char *const mine = pool + wave * FEW_TILE * row::bytes;

    const int heads = a.cache.heads;
    const int64_t *starts = line.starts;
    int64_t begin = 0, end = 1;
    if (!line.each) {
        if (!starts) {
            few_starts<THREADS>(a, UNIT, own_starts);
            starts = own_starts;
            if (block == 0)
                for (int i = tid; i <= a.nreq; i += THREADS) line.starts_out[i] = own_starts[i];
        }
        const few_cut cut(starts[a.nreq] * heads, line.blocks);
        begin = cut.begin(block);
        end = cut.begin(block + 1);
    }

    for (int64_t at = begin; at < end;) {
        // the request and head at this place of the line, or of this block
        const int r = line.each ? block / heads : wave_search(a.nreq, [&](int i) { return starts[i] * heads <= at; });
        const few_range x = few_load(a, UNIT, r);
        if (x.units == 0) return;   // (of a block of its own)
        const int64_t in_request = line.each ? (block - r * heads) * x.units : at - starts[r] * heads;
        const int h = (int)(in_request / x.units);
        const int64_t first = in_request - h * x.units, count = line.each ? x.units : min(x.units - first, end - at);
        const bool whole = count == x.units;
        const int part = at == begin ? 0 : 1;
        at += count;

        // rows: token n / group, head n % group of the group
        const int kv = attention_length(a, r);
        const int rows = (int)min((int64_t)FEW_ROWS, (int64_t)x.held * a.group);
        const int token = (int)a.by_group.div((uint32_t)n), sub = n - token * a.group;
        // the keys that this lane's row sees: `seen` of them from first_seen on
        const int last = kv - x.fresh + token, first_seen = a.window > 0 ? (int)max((int64_t)0, (int64_t)last - a.window + 1) : 0;
        const uint32_t seen = (uint32_t)max(0, min(last, x.keys - 1) - first_seen + 1);
        const int all_upto = min(kv - x.fresh, x.keys - 1);   // the last key that all rows see
        const int64_t qrow = a.cu[r] + (n < rows ? token : 0);
        u32x4 q[STEPS];
        {
            const T *p = (const T *)a.q.p + qrow * a.q.token_stride + (h * a.group + (n < rows ? sub : 0)) * a.q.head_stride;
#pragma unroll
            for (int t = 0; t < STEPS; ++t) q[t] = *(const u32x4 *)(p + few_row<C, D>::dim(t, g));
        }
        f32x4 out[OUTS];
#pragma unroll
        for (int f = 0; f < OUTS; ++f) out[f] = f32x4{0.f, 0.f, 0.f, 0.f};
        float ref = NO_SCORE, sum = 0.f;
        bool taken_out = false;

        const int tile0 = x.from + (int)first * UNIT + wave * FEW_TILE;   // this wave's first key; the next ones follow by units
        const int tiles = x.keys > tile0 ? (int)min(count, (int64_t)(x.keys - tile0 + UNIT - 1) / UNIT) : 0;
        const C *const keys = (const C *)a.cache.keys + h * a.cache.key_strides[2];
        const C *const values = (const C *)a.cache.values + h * a.cache.value_strides[2];
        auto places = [&](int i) {
            few_places p;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                int64_t page;
                int place;
                attention_place(a, r, min(tile0 + i * UNIT + 16 * s + n, x.keys - 1), page, place);
                p.k[s] = (int64_t)attention_key_at(a, page, place);
                p.v[s] = (int64_t)attention_value_at(a, page, place);
                p.block[s] = page;
            }
            return p;
        };
        few_row<C, D> k[2], v[2];
        float k_scale[2] = {1.f, 1.f}, v_scale[2] = {1.f, 1.f};
        auto load_k = [&](const few_places &p) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                k[s].load(keys + p.k[s], g);
                if constexpr (__is_same(C, e4m3)) k_scale[s] = e4m3_scale<T>(a, a.k_scales, p.block[s], h);
            }
        };
        auto load_v = [&](const few_places &p) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                v[s].load(values + p.v[s], g);
                if constexpr (__is_same(C, e4m3)) v_scale[s] = e4m3_scale<T>(a, a.v_scales, p.block[s], h);
            }
        };
        few_places next;
        if (tiles > 0) {
            next = places(0);
            load_k(next);
            load_v(next);
            next = places(min(1, tiles - 1));
        }
        for (int i = 0; i < tiles; ++i) {
            const int tile = tile0 + i * UNIT;
            f32x4 s[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                s[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int t = 0; t < STEPS; ++t) s[j] = mfma_of<T>::m16(k[j].template step<T>(t, k_scale[j]), q[t], s[j]);
            }
            if (i + 1 < tiles) load_k(next);
            // a lane's scores: keys 16 j + 4 g + e of the tile for row n
            float p[8], high_score = NO_SCORE;
            const bool all_seen = tile + FEW_TILE - 1 <= all_upto && (a.window == 0 || tile >= (int64_t)kv - a.window);
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int key = tile + 16 * j + 4 * g + e;
                    float y = s[j][e] * a.scale_log2;
                    if (!all_seen && (uint32_t)(key - first_seen) >= seen) y = -INFINITY;
                    p[4 * j + e] = y;
                    high_score = fmaxf(high_score, y);
                }
            // The reference of a row moves only when a score passes it by 2^8: that much neither the sums nor the weights' type
            // minds, and nearly no tile scales the results.
            if (__any(high_score > ref + (8.f + WEIGHT_ROOM<T>))) {
                high_score = fmaxf(high_score, __shfl_xor(high_score, 16));
                high_score = fmaxf(high_score, __shfl_xor(high_score, 32));
                const float moved = fmaxf(ref, high_score - WEIGHT_ROOM<T>), shrink = exp2f(ref - moved);
                ref = moved;
                sum *= shrink;
#pragma unroll
                for (int f = 0; f < OUTS; ++f) out[f] *= shrink;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                p[e] = __builtin_amdgcn_exp2f(p[e] - ref);
                sum += p[e];
            }
            const u32x4 weights = pack8<T>(p);
            // values: rows of the tile into shared memory
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int t = 0; t < STEPS; ++t)
                    *(u32x4 *)(mine + (16 * j + n) * row::bytes + 16 * row::chunk(16 * j + n, few_row<C, D>::dim(t, g) / 8)) = v[j].template step<T>(t, v_scale[j]);
            // zeros for places that hold no key; what is not finite and not seen by all rows is taken out, see kv_attention_chunk.h
            if (!all_seen) {
                bool found = false;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const bool held = tile + 16 * j + n < x.keys;
#pragma unroll
                    for (int t = 0; t < STEPS; ++t) {
                        const u32x4 x = v[j].template step<T>(t, v_scale[j]);
                        if (held && !any_not_finite<T>(x)) continue;
                        found |= held;
                        *(u32x4 *)(mine + (16 * j + n) * row::bytes + 16 * row::chunk(16 * j + n, few_row<C, D>::dim(t, g) / 8)) = held ? finite_only<T>(x) : u32x4{0, 0, 0, 0};
                    }
                }
                taken_out |= __any(found);
            }
            if (i + 1 < tiles) {
                load_v(next);
                next = places(min(i + 2, tiles - 1));
            }
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int f = 0; f < OUTS; ++f) {
                u32x4 vt;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int key = 16 * j + 4 * g + (n >> 2);
                    const uint2 c = read_transposed(mine + key * row::bytes + 16 * row::chunk(key, 2 * f + ((n >> 1) & 1)) + 8 * (n & 1));
                    vt[2 * j] = c.x;
                    vt[2 * j + 1] = c.y;
                }
                out[f] = mfma_of<T>::m16(vt, weights, out[f]);
            }
            __builtin_amdgcn_wave_barrier();
        }
        if (taken_out) {
            for (int i = 0; i < tiles; ++i) {
                const int tile = tile0 + i * UNIT;
                if (tile + FEW_TILE - 1 <= all_upto && (a.window == 0 || tile >= (int64_t)kv - a.window)) continue;
                for (int key = tile; key < min(tile + FEW_TILE, x.keys); ++key) {
                    if ((uint32_t)(key - first_seen) >= seen) continue;
                    int64_t page;
                    int place;
                    attention_place(a, r, key, page, place);
                    const C *const row_v = values + attention_value_at(a, page, place);
#pragma unroll
                    for (int f = 0; f < OUTS; ++f) add_not_finite<T>(row_v + 16 * f + 4 * g, out[f], 0);
                }
            }
        }
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);

        // the four waves' results: dimensions 16 f + 4 g + e of row n
#pragma unroll
        for (int f = 0; f < OUTS; ++f) *(f32x4 *)(mine + (n * D + 16 * f + 4 * g) * 4) = out[f];
        if (g == 0) {
            stat[wave][n][0] = ref;
            stat[wave][n][1] = sum;
        }
        __syncthreads();
        for (int i = tid; i < rows * D; i += THREADS) {
            const int m = i / D, d = i % D;
            float top = NO_SCORE, all = 0.f, o = 0.f;
            for (int w = 0; w < WAVES; ++w) top = fmaxf(top, stat[w][m][0]);
            for (int w = 0; w < WAVES; ++w) {
                const float share = __builtin_amdgcn_exp2f(stat[w][m][0] - top);
                all += share * stat[w][m][1];
                o += share * ((const float *)(pool + w * FEW_TILE * row::bytes))[m * D + d];
            }
            if (whole) {
                const int tok = (int)a.by_group.div((uint32_t)m);
                const int64_t at_row = (int64_t)(a.cu[r] + tok) * a.q_heads + h * a.group + (m - tok * a.group);
                ((T *)a.out)[at_row * D + d] = (T)(all != 0.f ? o * VALUE_UNIT<T, C> / all : 0.f);
                if (d == 0 && a.lse) a.lse[at_row] = all != 0.f ? (top + log2f(all)) * LN2 : -INFINITY;
            } else {
                const int64_t at_row = ((int64_t)block * 2 + part) * FEW_ROWS + m;
                line.parts[at_row * D + d] = o;
                if (d == 0) {
                    line.stats[2 * at_row] = top;
                    line.stats[2 * at_row + 1] = all;
                }
            }
        }
        __syncthreads();
    }
}

// Joins the parts of rows of one (request, head), WAVES / row_waves of them: a row's waves sum up every so many-th part, and
// their sums are added in the same order always.
template <class T, class C, int D, int WAVES> __device__ __forceinline__ void few_join_block(const attention_args &a, const few_line &line, int block, int slice) {
    __shared__ float sums[WAVES][D], alls[WAVES], tops[WAVES];
    constexpr int E = (D + 63) / 64;
    const int heads = a.cache.heads, r = block / heads, h = block - r * heads, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t start = line.starts_out[r], units = line.starts_out[r + 1] - start;
    if (units == 0) return;
    const few_cut cut(line.starts_out[a.nreq] * heads, line.blocks);
    const int64_t from = start * heads + h * units, to = from + units;
    const int first = cut.block_of(from), last = cut.block_of(to - 1);
    if (first == last) return;   // all in one block: done there
    const int row_waves = line.row_waves, first_row = slice * (WAVES / row_waves);
    const int rows = min(WAVES / row_waves, (int)min((int64_t)FEW_ROWS, (int64_t)few_load(a, line.unit, r).held * a.group) - first_row);
    if (rows <= 0) return;
    const int mine = wave / row_waves, way = wave - mine * row_waves, m = first_row + mine;
    float top = NO_SCORE, all = 0.f, o[E] = {};
    if (mine < rows) {
        // the part of block b: its first one, but where the (request, head) begins inside the block
        auto slot = [&](int b) { return ((int64_t)b * 2 + (cut.begin(b) >= from ? 0 : 1)) * FEW_ROWS + m; };
        for (int b = first + lane; b <= last; b += 64) top = fmaxf(top, line.stats[2 * slot(b)]);
        for (int d = 32; d > 0; d /= 2) top = fmaxf(top, __shfl_xor(top, d));
#pragma unroll 4
        for (int b = first + way; b <= last; b += row_waves) {
            const int64_t at = slot(b);
            const float share = __builtin_amdgcn_exp2f(line.stats[2 * at] - top);
            all += share * line.stats[2 * at + 1];
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (D % 64 == 0 || e * 64 + lane < D) o[e] += share * line.parts[at * D + e * 64 + lane];
        }
    }
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (D % 64 == 0 || e * 64 + lane < D) sums[wave][e * 64 + lane] = o[e];
    if (lane == 0) {
        alls[wave] = all;
        tops[wave] = top;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < rows * D; i += 64 * WAVES) {
        const int at = i / D, d = i % D, row = first_row + at;
        float total = 0.f, sum = 0.f;
        for (int w = at * row_waves; w < (at + 1) * row_waves; ++w) {
            total += alls[w];
            sum += sums[w][d];
        }
        const int tok = (int)a.by_group.div((uint32_t)row);
        const int64_t at_row = (int64_t)(a.cu[r] + tok) * a.q_heads + h * a.group + (row - tok * a.group);
        ((T *)a.out)[at_row * D + d] = (T)(total != 0.f ? sum * VALUE_UNIT<T, C> / total : 0.f);
        if (d == 0 && a.lse) a.lse[at_row] = total != 0.f ? (tops[at * row_waves] + log2f(total)) * LN2 : -INFINITY;
    }
}

// The line's memory in read_ws (from its start on), its blocks and the waves that join a row; grows the buffer to hold `more` bytes
// behind it.
int few_prepare(pq_ctx *ctx, const attention_args &a, int waves, size_t more, few_line *line, size_t *ws_used);
// Slices of the rows of a (request, head) for the kernel that joins, of `waves` waves.
static inline int few_slices(const few_line &line, int most_rows, int waves) { return (most_rows * line.row_waves + waves - 1) / waves; }

}  // namespace pq
