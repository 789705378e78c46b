// The append to a paged cache of 8 bits (pq_kv_append8).
#include "e4m3.h"
#include "kv_append.h"
#include "wave_sums.h"

namespace pq {

struct append8_args {
    append_args in;       // (its cache: sizes alone)
    pq_kv_cache8 cache;
    fast_div by_block;
    double of_dim;        // 1 / dim
};

// The slot of a token that is written, -1 for others.
__device__ __forceinline__ int64_t append8_slot(const append8_args &a, int64_t t) {
    const int32_t p = a.in.positions[t];
    const int64_t slot = a.in.slots[t];
    return p >= 0 && (a.in.rot == 0 || p < a.in.max_positions) && slot >= 0 && slot < a.cache.nblocks * a.cache.block_size ? slot : -1;
}
__device__ __forceinline__ int64_t append8_block(const append8_args &a, int64_t slot) {
    return slot >> 31 ? slot / a.cache.block_size : (int64_t)a.by_block.div((uint32_t)slot);
}

// A run: tokens one after the other whose slots follow each other within a block.
struct append8_run {
    int64_t token, block;
    int place, count;   // of its first token; its tokens
};
// Whether a token begins one (slot: its own, slot_before: that of the token before it).
__device__ __forceinline__ bool append8_begins(const append8_args &a, int64_t slot, int64_t slot_before) {
    return slot >= 0 && (slot_before != slot - 1 || append8_block(a, slot) * a.cache.block_size == slot);
}
// The run of a token that begins one and has so many tokens.
__device__ __forceinline__ append8_run append8_known(const append8_args &a, int64_t t, int64_t slot, int count) {
    const int64_t block = append8_block(a, slot);
    return {t, block, (int)(slot - block * a.cache.block_size), count};
}
// The same with the tokens behind these that belong to it, by a whole wave.
__device__ __forceinline__ append8_run append8_find(const append8_args &a, append8_run r) {
    const int lane = threadIdx.x & 63;
    const int64_t t = r.token, slot = r.block * a.cache.block_size + r.place;
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

// Where a run's keys or values of a head go, and its scale.
struct append8_place {
    uint8_t *rows;     // place 0 of the block
    int64_t stride;    // from place to place
    float *scale;
};
__device__ __forceinline__ append8_place append8_locate(const append8_args &a, const append8_run &run, int h, bool is_key) {
    const int64_t *strides = is_key ? a.cache.key_strides : a.cache.value_strides;
    return {(uint8_t *)(is_key ? a.cache.keys : a.cache.values) + run.block * strides[0] + h * strides[2], strides[1],
            (is_key ? a.cache.key_scales : a.cache.value_scales) + run.block * a.cache.heads + h};
}

// ---- any layout ---------------------------------------------------------------------------------------
//
// One wave for each token and head (of the cache: one for keys, one for values), which holds the run that begins there.  It goes over
// the run's rows twice, for the largest element and to write them; no row is kept between.  (The 16 384 tokens below take 1430 us here.)
template <class T, bool PAIRS> __device__ __forceinline__ void append8_general_head(const append8_args &a, int64_t t, int h, bool is_key) {
    const int64_t slot = append8_slot(a, t);
    if (!append8_begins(a, slot, t > 0 ? append8_slot(a, t - 1) : -1)) return;
    const append8_run run = append8_find(a, append8_known(a, t, slot, 1));
    const int lane = threadIdx.x & 63, dim = a.cache.dim, rot = is_key ? a.in.rot : 0;
    const pq_heads &from = is_key ? a.in.k : a.in.v;
    const append8_place to = append8_locate(a, run, h, is_key);

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
    const int before = run.place > 0 ? scale_exponent(*to.scale) : LEAST_EXPONENT, e = max(before, exponent_for(amax));
    if (run.place > 0 && e > before)
        for (int p = 0; p < run.place; ++p)
            for (int i = lane; i < dim; i += 64) {
                uint8_t *const at = to.rows + p * to.stride + i;
                *at = (uint8_t)e4m3_of(ldexpf((float)e4m3{*at}, before - e), 0.f);
            }
    each([&](int place, int first, int second, float x, float y) {
        const uint32_t codes = e4m3_of(ldexpf(x, -e), ldexpf(y, -e));
        to.rows[place * to.stride + first] = (uint8_t)codes;
        to.rows[place * to.stride + second] = (uint8_t)(codes >> 8);
    });
    if (lane == 0) *to.scale = scale_of(e);
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

// ---- by groups of lanes ---------------------------------------------------------------------------------
//
// A block looks at a chunk of tokens and takes the runs that begin among them, as many side by side as it has rows for (gl lanes
// hold a row, kv_append.h), head by head, keys or values.  A row stays in registers from the norm over the largest
// element to the codes, what the rows of a run need of a scale they tell each other in shared memory; the next head's rows are on their
// way meanwhile, and a token's rotation is read once for all its heads.  Rows of a run that is longer than the block holds are read
// a second time.
//
// Scales are powers of two: a scale that grows moves the exponents of what is there, and only what falls below the least exponent is
// rounded again; a number's own exponent makes a finer scale of little use.  fp64 up to a key's x costs 2 us of 40 (below) and makes
// its code a matter of the definition, not of the order in which a norm is summed: next to a border of e4m3 the last bit of x decides
// over a sixteenth of it.
//
// 16 384 tokens of 32 + 8 + 8 heads of 128 dimensions, bf16: 378 MB in 97 us, 44 us keys and values (101 MB; bound by vector instructions
// and by their meetings: a list of 16 rows takes a wave about 250 to 350 of them) and 53 us queries (268 MB = 5.0 TB/s); 4099 tokens of 36 heads of
// 80 dimensions, f16, 25 us; 64 single tokens 8.6 us a call, a chain of slots, rows and rotations, scales.
constexpr int APPEND8_V = 4;       // of keys (eight elements a lane: sixteen, in fp64, leave registers for two waves of a SIMD)
constexpr int APPEND8_MOST = 1024; // threads of a block
constexpr int APPEND8_ROWS = APPEND8_MOST;

// Runs side by side: tokens t ... t + n - 1.  begins: those of 64 tokens from t - i0 on that begin a run; one: there is one run.
struct append8_tile {
    int64_t t;
    int n, i0;
    uint64_t begins;
    bool one;
    append8_run run;   // the first
};
// The run of a thread's row: its block, its first place there, its rows of the tile.
struct append8_row {
    int64_t block;
    int place, begin, end;
};
__device__ __forceinline__ append8_row append8_row_of(const append8_args &a, const append8_tile &tile, int row, int rows) {
    append8_row mine = {tile.run.block, tile.run.place, 0, min(tile.n, rows)};
    if (!tile.one && row < tile.n) {
        const int i = tile.i0 + row;
        const uint64_t behind = i < 63 ? tile.begins >> (i + 1) : 0;
        mine.begin = 63 - __clzll((long long)(tile.begins & (~0ull >> (63 - i)))) - tile.i0;
        mine.end = behind ? min(tile.n, row + __ffsll((unsigned long long)behind)) : tile.n;
        const int64_t slot = a.in.slots[tile.t + mine.begin];
        mine.block = append8_block(a, slot);
        mine.place = (int)(slot - mine.block * a.cache.block_size);
    }
    return mine;
}

// 1 / sqrt(x), to the last bits: the processor's, which has about half of them, and two steps of Newton's method
__device__ __forceinline__ double inverse_root(double x) {
    double r = __builtin_amdgcn_rsq(x);
#pragma unroll
    for (int i = 0; i < 2; ++i) r = fma(r * 0.5, fma(-x * r, r, 1.0), r);
    return x < INFINITY ? r : 1.0 / x;   // (0: of numbers whose squares are no number any more)
}

// Exponents of the scales that a list's runs need, in the place of a run's first row.  Three lists' in turn: while one is written, that
// before it is read, and that before is cleared.
struct append8_shared {
    int exponent[3][APPEND8_ROWS];
};

// The keys or the values of heads first ... end - 1, from head `at` on.
template <class T, int V, bool PAIRS, bool KEYS, bool LONG>
__device__ __forceinline__ void append8_heads(const append8_args &a, int gl, const append8_tile &tile, const append8_row &mine, int first, int end, int at, append8_shared &shared, int &turn) {
    typedef elem_vec<T, V> vec;
    typedef elem_vec<float, V> fvec;
    typedef elem_vec<uint32_t, V / 4> codes;
    const int u = threadIdx.x & (gl - 1), rows = blockDim.x / gl, row = threadIdx.x / gl;
    const bool active = u < a.cache.dim / (2 * V), normed = KEYS && a.in.norm, weighted = normed && a.in.k_weight;
    const append_unit<V, PAIRS> unit(active ? u : 0, KEYS ? a.in.rot : 0);
    const int second = unit.second - unit.first, parts = LONG ? (tile.n + rows - 1) / rows : 1;

    const pq_heads &from = KEYS ? a.in.k : a.in.v;
    const T *const in = (const T *)from.p + (tile.t + row) * from.token_stride + unit.first;
    const int64_t *const strides = KEYS ? a.cache.key_strides : a.cache.value_strides;
    uint8_t *const block = (uint8_t *)(KEYS ? a.cache.keys : a.cache.values) + mine.block * strides[0] + unit.first;
    uint8_t *const out = block + (mine.place + row - mine.begin) * strides[1];
    float *const scales = (KEYS ? a.cache.key_scales : a.cache.value_scales) + mine.block * a.cache.heads;

    fvec wx, wy, c, s;
    if (weighted) {
        wx = *(const fvec *)(a.in.k_weight + unit.first);
        wy = *(const fvec *)(a.in.k_weight + unit.first + second);
    }
    vec next_x, next_y;
    float next_scale = 0.f;
    auto fetch = [&](int h, int begin) {
        if (!active || begin + row >= tile.n) return;
        if (mine.place > 0) next_scale = scales[h];
        const T *const p = in + begin * from.token_stride + h * from.head_stride;
        next_x = *(const vec *)p;
        next_y = *(const vec *)(p + second);
    };
    auto angles = [&](int begin) {
        if (!KEYS || unit.angle < 0 || !active || begin + row >= tile.n) return;
        const int64_t i = (int64_t)a.in.positions[tile.t + begin + row] * (a.in.rot / 2) + unit.angle;
        c = *(const fvec *)(a.in.cos_table + i);
        s = *(const fvec *)(a.in.sin_table + i);
    };

    fetch(at, 0);
    angles(0);
#pragma unroll 1
    for (int left = end - first, h = at; left > 0; --left) {
        const int next_h = h + 1 < end ? h + 1 : first;
        if (parts > 1 && left < end - first) {   // (of one part they are on their way since the head before)
            fetch(h, 0);
            angles(0);
        }
        const int before = mine.place > 0 ? scale_exponent(next_scale) : LEAST_EXPONENT;
        float amax = 0.f;
        int e8 = before;
        bool odd = false;   // some number is none
        // (a run of more than one part first for the largest element, then to be written)
#pragma unroll 1
        for (int n = 0; n < (parts > 1 ? 2 * parts : 1); ++n) {
            const int begin = (n < parts ? n : n - parts) * rows;
            const bool there = active && begin + row < tile.n;
            if (n > 0) {
                fetch(h, begin);
                angles(begin);
            }
            float x[V], y[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                x[e] = there ? (float)next_x.v[e] : 0.f;
                y[e] = there ? (float)next_y.v[e] : 0.f;
            }
            if (parts == 1 && left > 1) fetch(next_h, 0);
            if constexpr (KEYS) {
                double r = 1.0;
                if (normed) {
                    double sum = 0.0;
#pragma unroll
                    for (int e = 0; e < V; ++e) sum += (double)x[e] * (double)x[e] + (double)y[e] * (double)y[e];
                    r = inverse_root(group_total<op_add>(sum, gl) * a.of_dim + (double)a.in.eps);
                }
                if (there) {   // (what is not there is zero: a norm of it might be none)
                    double dx[V], dy[V];
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        dx[e] = (double)x[e] * r;
                        dy[e] = (double)y[e] * r;
                    }
                    if (weighted)
#pragma unroll
                        for (int e = 0; e < V; ++e) {
                            dx[e] *= (double)wx.v[e];
                            dy[e] *= (double)wy.v[e];
                        }
                    if (unit.angle >= 0) {
                        double dc[V], ds[V];
#pragma unroll
                        for (int e = 0; e < V; ++e) {
                            dc[e] = (double)c.v[e];
                            ds[e] = (double)s.v[e];
                        }
                        append_turn<V, PAIRS>(dx, dy, dc, ds);
                    }
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        x[e] = (float)dx[e];
                        y[e] = (float)dy[e];
                    }
                }
            }
            if (n < parts) {
                uint32_t largest = 0;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const uint32_t bx = __builtin_bit_cast(uint32_t, x[e]) & 0x7fffffffu, by = __builtin_bit_cast(uint32_t, y[e]) & 0x7fffffffu;
                    largest = max(largest, max(bx, by));
                }
                if (__any(largest >= 0x7f800000u)) {
                    odd = true;
                    largest = 0;
#pragma unroll
                    for (int e = 0; e < V; ++e) largest = max(largest, __builtin_bit_cast(uint32_t, fmaxf(finite_size(x[e]), finite_size(y[e]))));
                }
                amax = fmaxf(amax, __builtin_bit_cast(float, largest));
                if (n + 1 < parts) continue;
                const int needed = exponent_for(group_total<op_larger>(amax, gl));
                if (row < tile.n && u == 0) atomicMax(&shared.exponent[turn][mine.begin], needed);
                __syncthreads();
                e8 = max(e8, shared.exponent[turn][mine.begin]);
                if (u == 0) shared.exponent[turn == 0 ? 2 : turn - 1][row] = LEAST_EXPONENT;
                turn = turn == 2 ? 0 : turn + 1;
                if (parts > 1) continue;
            }
            if (!there) continue;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                x[e] = __builtin_amdgcn_ldexpf(x[e], -e8);
                y[e] = __builtin_amdgcn_ldexpf(y[e], -e8);
            }
            uint8_t *const p = out + begin * strides[1] + h * strides[2];
            codes cx, cy;
#pragma unroll
            for (int e = 0; e < V / 4; ++e) {
                cx.v[e] = odd ? e4m3_of(x + 4 * e) : e4m3_of_held(x + 4 * e);
                cy.v[e] = odd ? e4m3_of(y + 4 * e) : e4m3_of_held(y + 4 * e);
            }
            *(codes *)p = cx;
            *(codes *)(p + second) = cy;
        }
        const bool there = active && row < tile.n;
        // The scale has grown: what the block held before, rounded anew.
        if (there && e8 > before)
            for (int p = row - mine.begin; p < mine.place; p += mine.end - mine.begin)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    codes *const at_codes = (codes *)(block + p * strides[1] + h * strides[2] + half * second);
                    codes held = *at_codes;
#pragma unroll
                    for (int e = 0; e < V / 4; ++e) {
                        float f[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) f[i] = __builtin_amdgcn_ldexpf((float)e4m3{(uint8_t)(held.v[e] >> 8 * i)}, before - e8);
                        held.v[e] = e4m3_of_held(f);
                    }
                    *at_codes = held;
                }
        if (there && u == 0 && row == mine.begin) scales[h] = scale_of(e8);
        h = next_h;
    }
}

// The runs that begin in a chunk, of as many tokens as the block has rows (64 at most): heads first ... end - 1 of their keys or values.
template <class T, int V, bool PAIRS, bool KEYS, bool LONG>
__device__ __forceinline__ void append8_chunk(const append8_args &a, int gl, int64_t chunk, int first, int end, append8_shared &shared) {
    const int lane = threadIdx.x & 63, rows = blockDim.x / gl, tokens = min(rows, 64);
    const int64_t t0 = chunk * tokens, t = t0 + lane;
    // the slots of 64 tokens, and of those before them
    const int64_t slot = t < a.in.ntokens ? append8_slot(a, t) : -1, slot_before = t > 0 && t < a.in.ntokens ? append8_slot(a, t - 1) : -1;
    const bool is_first = append8_begins(a, slot, slot_before);
    const uint64_t begins = __ballot(is_first), follows = __ballot(slot >= 0 && !is_first);
    // tokens of the run that token i begins, so far as it lies among the 64
    auto length = [&](int i) {
        const uint64_t behind = i == 63 ? 0 : ~(follows >> (i + 1));
        return 1 + (behind ? min(__ffsll((unsigned long long)behind) - 1, 63 - i) : 63 - i);
    };
    if ((threadIdx.x & (gl - 1)) == 0)
        for (int i = 0; i < 3; ++i) shared.exponent[i][threadIdx.x / gl] = LEAST_EXPONENT;
    __syncthreads();
    int turn = 0;
    for (uint64_t todo = begins & (~0ull >> (64 - tokens)); todo;) {
        const int i = __ffsll((unsigned long long)todo) - 1;
        append8_tile tile = {t0 + i, length(i), i, begins, true, {}};
        tile.run = append8_known(a, t0 + i, read_lane(slot, i), tile.n);
        todo &= todo - 1;
        if (i + tile.n >= 64) {
            tile.run = append8_find(a, tile.run);
            tile.n = tile.run.count;
        } else {
            // the runs that begin right behind it, so long as there are rows for them
            while (i + tile.n < tokens && (todo >> (i + tile.n) & 1)) {
                const int more = length(i + tile.n);
                if (i + tile.n + more >= 64 || tile.n + more > rows) break;
                todo &= todo - 1;
                tile.n += more;
                tile.one = false;
            }
        }
        const append8_row mine = append8_row_of(a, tile, threadIdx.x / gl, rows);
        append8_heads<T, V, PAIRS, KEYS, LONG>(a, gl, tile, mine, first, end, first, shared, turn);
    }
}

// The blocks of one side, keys or values: `groups` of them share a chunk's heads, `each` of these a block.
struct append8_side {
    int64_t blocks;
    int gl, groups, each;
};
// Blocks of keys, of values, and of queries, W elements of both of which are accessed at once.  LONG: blocks of the cache have more
// places than there are rows.
template <class T, int W, bool PAIRS, int THREADS, bool LONG>
__global__ __launch_bounds__(THREADS) void kv_append8_kernel(append8_args a, append8_side keys, append8_side values) {
    __shared__ append8_shared shared;
    unsigned block = blockIdx.x;
    if (block < keys.blocks) {
        const unsigned chunk = block / keys.groups, first = (block - chunk * keys.groups) * keys.each;
        append8_chunk<T, APPEND8_V, PAIRS, true, LONG>(a, keys.gl, chunk, first, min(a.cache.heads, (int)first + keys.each), shared);
        return;
    }
    block -= keys.blocks;
    if (block < values.blocks) {
        const unsigned chunk = block / values.groups, first = (block - chunk * values.groups) * values.each;
        append8_chunk<T, W, PAIRS, false, LONG>(a, values.gl, chunk, first, min(a.cache.heads, (int)first + values.each), shared);
        return;
    }
    append_rows<T, W, PAIRS>(a.in, values.gl, (int64_t)(block - values.blocks) * blockDim.x + threadIdx.x);
}

template <class T, int W, bool PAIRS> __global__ __launch_bounds__(APPEND_THREADS) void kv_append8_queries_kernel(append_args a, int gl) {
    append_rows<T, W, PAIRS>(a, gl, (int64_t)blockIdx.x * APPEND_THREADS + threadIdx.x);
}

static int lanes_of(int units) {
    int gl = 1;
    while (gl < units) gl *= 2;
    return gl;
}

template <class T, int W, bool PAIRS> static int append8_vector(pq_ctx *ctx, const append8_args &a) {
    const int key_gl = lanes_of(a.cache.dim / (2 * APPEND8_V)), gl = lanes_of(a.cache.dim / (2 * W)), heads = a.cache.heads;
    int threads = APPEND_THREADS;
    while (threads < APPEND8_MOST && threads / key_gl < a.cache.block_size) threads *= 2;
    auto side = [&](int lanes) {
        const int tokens = threads / lanes < 64 ? threads / lanes : 64;
        // (as many blocks as the chip holds, four waves on a SIMD, half of them for keys: fewer heads each begin more often)
        const int64_t chunks = (a.in.ntokens + tokens - 1) / tokens, held = ctx->num_cu * (1024 / threads) / 2, most = (held + chunks - 1) / chunks;
        const int each = most >= heads ? 1 : most <= 1 ? heads : (int)((heads + most - 1) / most), groups = (heads + each - 1) / each;
        return append8_side{chunks * groups, lanes, groups, each};
    };
    const append8_side keys = side(key_gl), values = side(gl);
    const int64_t queries = (a.in.ntokens * a.in.q_heads * gl + APPEND_THREADS - 1) / APPEND_THREADS;
    // Up to 64 MiB of queries in the same launch, which saves one: 32 + 8 + 8 heads of 128 dimensions, bf16, 34 MB of queries 30 us, 33 with a
    // launch of their own, 67 MB 55 and 60; 12 heads each of 80, f16, 8 MB 25 and 30, 58 MB 147 and 147.  More of them want the waves that
    // this kernel's registers do not leave: 98 MB of the former 79 and 74 us, 134 MB 106 and 97; 96 MB in f32 (28 + 4 + 4 heads) 60 and 57.
    const bool merged = a.in.ntokens * a.in.q_heads * a.cache.dim * (int64_t)sizeof(T) <= (int64_t)64 << 20;
    const int64_t all = keys.blocks + values.blocks + (merged ? (queries * APPEND_THREADS + threads - 1) / threads : 0);
    if (!grid_fits(all, threads) || !grid_fits(queries, APPEND_THREADS)) return fail(ctx, PQ_EUNSUPPORTED, "kv_append8: %lld tokens in one call", (long long)a.in.ntokens);
    const unsigned grid = (unsigned)all;
    if (a.cache.block_size > threads / key_gl) kv_append8_kernel<T, W, PAIRS, APPEND8_MOST, true><<<grid, threads, 0, ctx->stream>>>(a, keys, values);
    else if (threads > APPEND_THREADS) kv_append8_kernel<T, W, PAIRS, APPEND8_MOST, false><<<grid, threads, 0, ctx->stream>>>(a, keys, values);
    else kv_append8_kernel<T, W, PAIRS, APPEND_THREADS, false><<<grid, threads, 0, ctx->stream>>>(a, keys, values);
    if (!merged && queries > 0) kv_append8_queries_kernel<T, W, PAIRS><<<(unsigned)queries, APPEND_THREADS, 0, ctx->stream>>>(a.in, gl);
    PQ_HIP(ctx, hipGetLastError());
    return PQ_OK;
}

// whether rows, pairs and the rest of the head allow accesses of v elements: of keys, or of queries and values, whose codes they are too
static bool append8_fits(const append8_args &a, int v, size_t e, bool of_keys) {
    const pq_kv_cache8 &c = a.cache;
    uint64_t elems = 0, codes = (uint64_t)(uintptr_t)(of_keys ? c.keys : c.values), tables = (uint64_t)(uintptr_t)(of_keys ? a.in.k_weight : a.in.q_weight);
    for (int i = 0; i < 3; ++i) codes |= (uint64_t)(of_keys ? c.key_strides[i] : c.value_strides[i]);
    auto rows = [&](const pq_heads &h) { elems |= (uint64_t)(uintptr_t)h.p | (uint64_t)h.token_stride * e | (uint64_t)h.head_stride * e; };
    rows(of_keys ? a.in.k : a.in.v);
    if (!of_keys && a.in.q_heads > 0) {
        rows(a.in.q);
        elems |= (uint64_t)(uintptr_t)a.in.q_out;   // (dim is a multiple of v, as its parts are)
    }
    if (a.in.rot > 0) tables |= (uint64_t)(uintptr_t)a.in.cos_table | (uint64_t)(uintptr_t)a.in.sin_table;
    return a.in.rot / 2 % v == 0 && (c.dim - a.in.rot) / 2 % v == 0 && c.dim <= 64 * 2 * v && elems % (v * e) == 0 && codes % v == 0 && tables % (v * 4) == 0;
}

template <class T, bool PAIRS> static int append8_typed(pq_ctx *ctx, const append8_args &a) {
    constexpr int most = 16 / sizeof(T);
    if (append8_fits(a, APPEND8_V, sizeof(T), true)) {
        if (append8_fits(a, most, sizeof(T), false)) return append8_vector<T, most, PAIRS>(ctx, a);
        if (append8_fits(a, 4, sizeof(T), false)) return append8_vector<T, 4, PAIRS>(ctx, a);
    }
    constexpr int WAVES = APPEND_THREADS / 64;
    const int64_t queries = (a.in.ntokens * a.in.q_heads + WAVES - 1) / WAVES, items = (a.in.ntokens * 2 * a.cache.heads + WAVES - 1) / WAVES;
    if (!grid_fits(queries + items, APPEND_THREADS)) return fail(ctx, PQ_EUNSUPPORTED, "kv_append8: %lld tokens in one call", (long long)a.in.ntokens);
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
    a.by_block = fast_div((uint32_t)cache->block_size);
    a.of_dim = 1.0 / cache->dim;
    switch (elem) {
    case PQ_ELEM_F32: return pairs ? append8_typed<float, true>(ctx, a) : append8_typed<float, false>(ctx, a);
    case PQ_ELEM_F16: return pairs ? append8_typed<_Float16, true>(ctx, a) : append8_typed<_Float16, false>(ctx, a);
    default: return pairs ? append8_typed<__bf16, true>(ctx, a) : append8_typed<__bf16, false>(ctx, a);
    }
}

}  // namespace pq
