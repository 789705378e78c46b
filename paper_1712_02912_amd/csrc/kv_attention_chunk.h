// Attention of chunks of new tokens: bound by the matrix cores.
//
// A block holds 32 rows of queries per wave in registers (rows: token, head of the group, so the heads that share keys
// share them here too) and walks over the keys in tiles of 64 (32), which its waves read from shared memory.  Scores are formed
// transposed, S^T = K Q^T, so a lane holds scores of one row only, its maximum and sum need no exchange between lanes in most
// tiles, and the weights are, as they lie, the second operand of O^T = V^T P^T (the order of the keys within a product is
// free: V's are read in the order that the scores have, transposed by the reads from shared memory).
//
// Keys and values go through registers into one of two buffers while the other one is computed on, so one barrier per tile is
// enough and loads have a tile's time to arrive.  Places that hold no key become zeros on that way.
//
// Two chunks of 2048 over 14 336 keys, 32 heads of 128 dimensions on 8, bf16: 736 GFLOP in 690 to 730 us, by the card = 1.01 to 1.06
// PFLOP/s (a large product: 1.23).  Matrix instructions take 52 % of the cycles there, vector instructions (a quarter of them the powers of
// two, at a quarter of the rate) 48 %: the waves of a block meet at every tile and do the same at the same time, and giving half of
// them priority did not change that.  64 dimensions: 0.75 PFLOP/s (as many powers for half the products); 256: 0.48, where a SIMD
// has registers for one wave only.
//
// Over a cache of 8 bits (C = e4m3) a tile's codes become 16-bit elements on their way into shared memory, once for all waves of a block
// (products of 8 bits at twice the rate would need queries and weights in two halves each, twice the products, and instructions for every
// weight of every row, where a converted element serves all rows): the two chunks take 715 us a call, 722 over 16 bits.  33 requests of 2 to 6
// tokens, 7 heads on each of 4, up to 5009 keys: 46 us, and 9 us to join parts; a tile of 128 rows has 14 to 42 there, so one wave or two
// carry the chain of every tile of keys (1.3 TB/s, 73 TFLOP/s) and the others only move keys.  (Parts of equal length instead of equal shares of a
// request: 63 rows 46 us, not 64, but equal contexts 43 to 53 us; tiles of 32 rows in kv_attention_few.h: 28 rows 57 us, not 49.)
#pragma once
#include <type_traits>

#include "kv_attention_few.h"

namespace pq {

struct chunk_split {
    int splits;            // blocks that share the keys of a tile of rows
    bool without_few;      // requests of few rows are left to the blocks of kv_attention_few.h
    float *parts, *stats;  // [ntokens * q_heads][splits][D], [..][splits][2]
};

// The tiles of rows, one index each: request after request, the empty indexes behind the last one.  Every wave adds up the
// requests before its own, 64 at a time.  (Blocks without work between the others are not free: they take their turn in the
// order in which blocks are dealt to the parts of the chip, so with every second index empty half of the compute units got all
// the work, and 448 tiles of 128 rows over 1152 keys of 64 dimensions took 51 us, 33 us without.)  Adding up is for
// CHUNK_ADDED requests; where there are more, request r owns the indexes from cu[r] * group / M + r on, at least as many as it
// has tiles.
constexpr int CHUNK_ADDED = 512;
struct chunk_place {
    int r, tiles;     // the request (-1: none), its tiles of rows
    int64_t index;    // among them
};
template <int M> __device__ __forceinline__ chunk_place chunk_locate(const attention_args &a, bool without_few, int64_t index) {
    auto tiles_of = [&](int r) {
        const int held = attention_held(a, r);
        return held <= 0 || (without_few && attention_is_few(a, held)) ? 0 : (int)(((int64_t)held * a.group + M - 1) / M);
    };
    if (a.nreq > CHUNK_ADDED) {
        const int r = wave_search(a.nreq, [&](int i) { return (int64_t)a.cu[i] * a.group / M + i <= index; });
        const int tiles = tiles_of(r);
        index -= (int64_t)a.cu[r] * a.group / M + r;
        return {index < tiles ? r : -1, tiles, index};
    }
    const int lane = threadIdx.x & 63;
    int64_t before = 0;
    for (int base = 0; base < a.nreq; base += 64) {
        const int mine = base + lane < a.nreq ? tiles_of(base + lane) : 0;
        int upto = mine;
        for (int d = 1; d < 64; d *= 2) {
            const int v = __shfl_up(upto, d);
            if (lane >= d) upto += v;
        }
        const uint64_t there = __ballot(before + upto > index);
        if (there) {
            const int at = __ffsll((unsigned long long)there) - 1, tiles = __shfl(mine, at);
            return {__builtin_amdgcn_readfirstlane(base + at), tiles, index - before - (__shfl(upto, at) - tiles)};
        }
        before += __shfl(upto, 63);
    }
    return {-1, 0, 0};
}

// What one load moves: eight elements of the queries' type, or 16 codes (eight where a row has fewer than 16 for each of `lanes`), which
// become elements of the queries' type where they are stored.
template <class C, int LANES, int D> struct chunk_of {
    static constexpr int ELEMS = 8;
    u32x4 x;
    __device__ __forceinline__ void load(const C *p) { x = *(const u32x4 *)p; }
    template <class T> __device__ __forceinline__ u32x4 eight(int, float) const { return x; }
};
template <int LANES, int D> struct chunk_of<e4m3, LANES, D> {
    static constexpr int ELEMS = D >= 16 * LANES ? 16 : 8;
    uint32_t x[ELEMS / 4];
    __device__ __forceinline__ void load(const e4m3 *p) {
        const elem_vec<uint32_t, ELEMS / 4> c = *(const elem_vec<uint32_t, ELEMS / 4> *)p;
#pragma unroll
        for (int i = 0; i < ELEMS / 4; ++i) x[i] = c.v[i];
    }
    template <class T> __device__ __forceinline__ u32x4 eight(int e, float scale) const { return from_e4m3<T>(x[2 * e], x[2 * e + 1], scale); }
};

// keys of a tile (of 256 dimensions, registers and shared memory hold half as many)
template <int D> constexpr int CHUNK_TILE = D > 128 ? 32 : 64;
template <int D> constexpr int CHUNK_POOL = 4 * CHUNK_TILE<D> * lds_row<D>::bytes;

// One block's tile of rows (block: index * heads + head) and part of its keys; pool: CHUNK_POOL bytes of shared memory.
template <class T, class C, int D, int WAVES> __device__ __forceinline__ void chunk_block(const attention_args &a, const chunk_split &split, int block, int part, unsigned char *pool) {
    constexpr int TILE = CHUNK_TILE<D>;
    typedef lds_row<D> row;
    constexpr int M = 32 * WAVES, THREADS = 64 * WAVES;
    constexpr int STEPS = D / 16, OUTS = D / 32;
    // (Alone on its SIMD, a wave waits for every read of shared memory unless it reads ahead: 8 requests of 1024 tokens over 1024 to
    // 8192 keys, 8 heads of 256 dimensions: 599 us, 663 without.  Where there are two waves it is no gain and costs registers.)
    constexpr int AT_ONCE = D > 128 ? 4 : 1;
    // a thread moves chunks of one key (and value) of a tile, every LANES-th from its own on: 16 bytes each, or 8 where eight-bit rows are
    // shorter than that for all lanes
    constexpr int LANES = THREADS / TILE;
    typedef chunk_of<C, LANES, D> piece;
    constexpr int CHUNKS = D / piece::ELEMS, MOVES = (CHUNKS + LANES - 1) / LANES;
    unsigned char *const lds_k[2] = {pool, pool + TILE * row::bytes}, *const lds_v[2] = {pool + 2 * TILE * row::bytes, pool + 3 * TILE * row::bytes};
    __shared__ int taken_out;   // values were (see below)
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 31, g = lane >> 5;

    // heads vary fastest: blocks that read the same head's keys are on the same XCD where the heads are a multiple of eight
    const int heads = a.cache.heads, h = block % heads;
    const chunk_place at = chunk_locate<M>(a, split.without_few, block / heads);
    if (at.r < 0) return;
    const int r = at.r, fresh = a.cu[r + 1] - a.cu[r], held = attention_held(a, r);
    const int64_t rows = (int64_t)held * a.group, mine = at.tiles - 1 - at.index;   // the last rows see the most keys: they come first

    const int kv = attention_length(a, r), nkeys = attention_keys(a, r);
    // this lane's row
    const int64_t my_row = mine * M + wave * 32 + n;
    const bool valid = my_row < rows;
    const int token = valid ? (int)a.by_group.div((uint32_t)my_row) : 0, sub = valid ? (int)(my_row - (int64_t)token * a.group) : 0;
    // the keys that it sees: `seen` of them from first_seen on
    const int last = kv - fresh + token, first_seen = a.window > 0 ? (int)max((int64_t)0, (int64_t)last - a.window + 1) : 0;
    const uint32_t seen = (uint32_t)max(0, min(last, nkeys - 1) - first_seen + 1);
    // the keys that the tile's rows see, and those that all of them see
    const int token0 = (int)a.by_group.div((uint32_t)(mine * M)), token1 = (int)a.by_group.div((uint32_t)(min(rows, (mine + 1) * M) - 1));
    const int to = min(nkeys, kv - fresh + token1 + 1);
    const int from = a.window > 0 ? (int)max((int64_t)0, (int64_t)kv - fresh + token0 - a.window + 1) : 0;
    const int all_from = a.window > 0 ? (int)max((int64_t)0, (int64_t)kv - fresh + token1 - a.window + 1) : 0, all_to = min(nkeys, kv - fresh + token0 + 1);
    const int tiles_all = to > from ? (to - from + TILE - 1) / TILE : 0;
    const int tile_begin = (int)((int64_t)tiles_all * part / split.splits), tile_end = (int)((int64_t)tiles_all * (part + 1) / split.splits);

    // (a negative scale is the queries' sign: scores are compared before they are scaled)
    const uint32_t sign = a.scale_log2 < 0.f ? 0x80008000u : 0u;
    const float scale_log2 = fmaxf(fabsf(a.scale_log2), 1e-37f);   // (0 times the -inf of a key that is not seen is no number)
    u32x4 q[STEPS];
    {
        const T *p = (const T *)a.q.p + (a.cu[r] + token) * a.q.token_stride + (h * a.group + sub) * a.q.head_stride + 8 * g;
#pragma unroll
        for (int t = 0; t < STEPS; ++t) q[t] = *(const u32x4 *)(p + 16 * t) ^ sign;
    }
    f32x16 out[OUTS];
#pragma unroll
    for (int f = 0; f < OUTS; ++f)
#pragma unroll
        for (int i = 0; i < 16; ++i) out[f][i] = 0.f;
    float ref = NO_SCORE, sum = 0.f;   // ref: of the scaled scores

    // the tiles that some row of this wave sees: the others it only helps to move
    const int64_t row0 = mine * M + wave * 32, row1 = min(rows, row0 + 32) - 1;
    int wave_begin = tile_end, wave_end = tile_end;
    if (row0 < rows) {
        const int wave_to = min(nkeys, kv - fresh + (int)a.by_group.div((uint32_t)row1) + 1);
        const int wave_from = a.window > 0 ? (int)max((int64_t)0, (int64_t)kv - fresh + (int)a.by_group.div((uint32_t)row0) - a.window + 1) : 0;
        wave_begin = (wave_from - from) / TILE;
        wave_end = wave_to > from ? (wave_to - from + TILE - 1) / TILE : 0;
    }

    // this thread's chunks of a tile
    const int my_key = tid / LANES, my_chunk = tid % LANES;
    const C *const keys = (const C *)a.cache.keys + h * a.cache.key_strides[2] + piece::ELEMS * my_chunk;
    const C *const values = (const C *)a.cache.values + h * a.cache.value_strides[2] + piece::ELEMS * my_chunk;
    const int32_t *const table = a.tables + (int64_t)r * a.width;
    piece mk[MOVES], mv[MOVES];
    float k_scale = 1.f, v_scale = 1.f;
    // (a tile's entry of the block table is read a tile before its keys are, so that nothing waits for it)
    int32_t entry = 0, place = 0;
    auto look_up = [&](int tile) {
        const uint32_t j = (uint32_t)min(from + tile * TILE + my_key, to - 1), column = a.by_block.div(j);
        place = (int)(j - column * a.cache.block_size);
        entry = table[column];
    };
    auto load = [&]() {
        const int64_t block = attention_block(a, entry);
        const C *const k = keys + attention_key_at(a, block, place);
        const C *const v = values + attention_value_at(a, block, place);
        if constexpr (__is_same(C, e4m3)) {
            k_scale = e4m3_scale<T>(a, a.k_scales, block, h);
            v_scale = e4m3_scale<T>(a, a.v_scales, block, h);
        }
#pragma unroll
        for (int i = 0; i < MOVES; ++i) {
            if (CHUNKS % LANES != 0 && my_chunk + LANES * i >= CHUNKS) continue;
            mk[i].load(k + piece::ELEMS * LANES * i);
            mv[i].load(v + piece::ELEMS * LANES * i);
        }
    };
    auto store = [&](int tile, int buffer) {
        const int key0 = from + tile * TILE;
#pragma unroll
        for (int i = 0; i < MOVES; ++i) {
            const int chunk = my_chunk + LANES * i;
            if (CHUNKS % LANES != 0 && chunk >= CHUNKS) continue;
#pragma unroll
            for (int e = 0; e < piece::ELEMS / 8; ++e) {
                const int at = my_key * row::bytes + 16 * row::chunk(my_key, chunk * (piece::ELEMS / 8) + e);
                *(u32x4 *)(lds_k[buffer] + at) = mk[i].template eight<T>(e, k_scale);
                *(u32x4 *)(lds_v[buffer] + at) = mv[i].template eight<T>(e, v_scale);
            }
        }
        // Values that some row does not see must not reach it as 0 times inf: where a tile has rows that do not see all of it,
        // what is not finite is taken out, and added in the end to the rows that see it.  Places behind the last key become zeros.
        if (key0 < all_from || key0 + TILE > all_to) {
            const bool held = key0 + my_key < to;
#pragma unroll
            for (int i = 0; i < MOVES; ++i) {
                const int chunk = my_chunk + LANES * i;
                if (CHUNKS % LANES != 0 && chunk >= CHUNKS) continue;
#pragma unroll
                for (int e = 0; e < piece::ELEMS / 8; ++e) {
                    const u32x4 x = mv[i].template eight<T>(e, v_scale);
                    if (held && !any_not_finite<T>(x)) continue;
                    *(u32x4 *)(lds_v[buffer] + my_key * row::bytes + 16 * row::chunk(my_key, chunk * (piece::ELEMS / 8) + e)) = held ? finite_only<T>(x) : u32x4{0, 0, 0, 0};
                    if (held) taken_out = 1;
                }
            }
        }
    };
    // Where this lane reads: key n of 32 and chunk g, key 4 g + (lane / 4) % 4 of 16 and its part of chunk pair 0.  Other chunks
    // differ in bits that the row's swizzle only turns over, so their places are one exclusive or away.
    const int k_at = n * row::bytes + 16 * row::chunk(n, g);
    const int v_key = 4 * g + ((lane >> 2) & 3);
    const int v_at = v_key * row::bytes + 16 * row::chunk(v_key, 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1)) + 8 * (lane & 1);

    auto compute = [&](int tile, auto buffer_of) {
        constexpr int buffer = decltype(buffer_of)::value;
        if (tile < wave_begin || tile >= wave_end) return;
        const int key0 = from + tile * TILE;
        f32x16 s[TILE / 32];
#pragma unroll
        for (int j = 0; j < TILE / 32; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[j][i] = 0.f;
        constexpr int KS = STEPS * (TILE / 32), VS = (TILE / 16) * OUTS;   // products of either kind
        u32x4 kf[2][AT_ONCE], vf[2][AT_ONCE];
        auto read_k = [&](int group) {
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                const int u = group * AT_ONCE + i, t = u / (TILE / 32), j = u % (TILE / 32);
                if (u < KS) kf[group & 1][i] = *(const u32x4 *)(lds_k[buffer] + (k_at ^ (32 * t)) + 32 * j * row::bytes);
            }
        };
        auto read_v = [&](int group) {
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                const int u = group * AT_ONCE + i, b = u / OUTS, f = u % OUTS;
                if (u >= VS) continue;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    // (keys 8 on change the swizzle's last bit, but in rows of 128 bytes, too)
                    const uint2 c = read_transposed(lds_v[buffer] + (v_at ^ (64 * f) ^ (16 * e)) + (16 * b + 8 * e) * row::bytes);
                    vf[group & 1][i][2 * e] = c.x;
                    vf[group & 1][i][2 * e + 1] = c.y;
                }
            }
        };
        read_k(0);
#pragma unroll
        for (int group = 0; group * AT_ONCE < KS; ++group) {
            if ((group + 1) * AT_ONCE < KS) read_k(group + 1);
            if (AT_ONCE > 1) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                const int u = group * AT_ONCE + i, t = u / (TILE / 32), j = u % (TILE / 32);
                if (u < KS) s[j] = mfma_of<T>::m32(kf[group & 1][i], q[t], s[j]);
            }
            if (AT_ONCE > 1) __builtin_amdgcn_sched_barrier(0);
        }
        read_v(0);
        // scores of this lane: keys 32 j + 8 (i / 4) + 4 g + i % 4 of the tile
        if (key0 < all_from || key0 + TILE > all_to) {   // some row does not see some key
#pragma unroll
            for (int j = 0; j < TILE / 32; ++j)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int key = key0 + 32 * j + 8 * (i / 4) + 4 * g + i % 4;
                    if ((uint32_t)(key - first_seen) >= seen) s[j][i] = -INFINITY;
                }
        }
        float high_score = -INFINITY;
#pragma unroll
        for (int j = 0; j < TILE / 32; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) high_score = fmaxf(high_score, s[j][i]);
        // (the reference moves only when a score passes it by 2^8, see kv_attention_few.h)
        if (__any(high_score * scale_log2 > ref + (8.f + WEIGHT_ROOM<T>))) {
            high_score = fmaxf(high_score, __shfl_xor(high_score, 32));
            const float moved = fmaxf(ref, high_score * scale_log2 - WEIGHT_ROOM<T>), shrink = __builtin_amdgcn_exp2f(ref - moved);
            ref = moved;
            sum *= shrink;
#pragma unroll
            for (int f = 0; f < OUTS; ++f) out[f] *= shrink;
        }
        float p[TILE / 2];
#pragma unroll
        for (int i = 0; i < TILE / 2; ++i) {
            p[i] = __builtin_amdgcn_exp2f(fmaf(s[i / 16][i % 16], scale_log2, -ref));
            sum += p[i];
        }
        u32x4 weights[TILE / 16];
#pragma unroll
        for (int b = 0; b < TILE / 16; ++b) weights[b] = pack8<T>(p + 8 * b);
#pragma unroll
        for (int group = 0; group * AT_ONCE < VS; ++group) {
            if ((group + 1) * AT_ONCE < VS) read_v(group + 1);
            if (AT_ONCE > 1) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                const int u = group * AT_ONCE + i, b = u / OUTS, f = u % OUTS;
                if (u < VS) out[f] = mfma_of<T>::m32(vf[group & 1][i], weights[b], out[f]);
            }
            if (AT_ONCE > 1) __builtin_amdgcn_sched_barrier(0);
        }
    };

    if (tid == 0) taken_out = 0;
    __syncthreads();
    if (tile_begin < tile_end) {
        look_up(tile_begin);
        load();
        look_up(min(tile_begin + 1, tile_end - 1));
        store(tile_begin, 0);
        load();
        look_up(min(tile_begin + 2, tile_end - 1));
    }
    // (behind the last tile that one is loaded once more, and not stored)
    auto step = [&](int tile, auto buffer_of) {
        constexpr int buffer = decltype(buffer_of)::value;
        __syncthreads();   // this tile is written, and the one before it read
        if (tile + 1 < tile_end) {
            store(tile + 1, buffer ^ 1);
            load();
            look_up(min(tile + 3, tile_end - 1));
        }
        compute(tile, buffer_of);
    };
    for (int tile = tile_begin; tile < tile_end; tile += 2) {
        step(tile, std::integral_constant<int, 0>());
        if (tile + 1 < tile_end) step(tile + 1, std::integral_constant<int, 1>());
    }
    if (__builtin_amdgcn_readfirstlane(taken_out)) {
        // (rare, and so without marks: all values of the tiles that some row does not see all of)
        for (int tile = max(tile_begin, wave_begin); tile < min(tile_end, wave_end); ++tile) {
            const int key0 = from + tile * TILE;
            if (key0 >= all_from && key0 + TILE <= all_to) continue;
            for (int key = key0; key < min(key0 + TILE, to); ++key) {
                if ((uint32_t)(key - first_seen) >= seen) continue;
                int64_t block;
                int at;
                attention_place(a, r, key, block, at);
                const C *const v = (const C *)a.cache.values + h * a.cache.value_strides[2] + attention_value_at(a, block, at);
#pragma unroll
                for (int f = 0; f < OUTS; ++f)
#pragma unroll
                    for (int i = 0; i < 4; ++i) add_not_finite<T>(v + 32 * f + 8 * i + 4 * g, out[f], 4 * i);
            }
        }
    }
    sum += __shfl_xor(sum, 32);
    if (!valid) return;
    const int64_t at_row = (int64_t)(a.cu[r] + token) * a.q_heads + h * a.group + sub;
    // dimensions 32 f + 8 (i / 4) + 4 g + i % 4 of this lane's row
    if (split.splits > 1) {
        const int64_t slot = at_row * split.splits + part;
#pragma unroll
        for (int f = 0; f < OUTS; ++f)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *(f32x4 *)(split.parts + slot * D + 32 * f + 8 * i + 4 * g) = f32x4{out[f][4 * i], out[f][4 * i + 1], out[f][4 * i + 2], out[f][4 * i + 3]};
        if (g == 0) {
            split.stats[2 * slot] = ref;
            split.stats[2 * slot + 1] = sum;
        }
        return;
    }
    const float scale = sum != 0.f ? VALUE_UNIT<T, C> / sum : 0.f;
    T *const to_row = (T *)a.out + at_row * D;
#pragma unroll
    for (int f = 0; f < OUTS; ++f)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            elem_vec<T, 4> v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v.v[e] = (T)(sum != 0.f ? out[f][4 * i + e] * scale : 0.f);
            *(elem_vec<T, 4> *)(to_row + 32 * f + 8 * i + 4 * g) = v;
        }
    if (g == 0 && a.lse) a.lse[at_row] = sum != 0.f ? (ref + log2f(sum)) * LN2 : -INFINITY;
}

// Joins the parts of rows, a wave for each row, in the order of the keys.
constexpr int JOIN_ROWS = 4;
template <class T, class C, int D> __device__ __forceinline__ void chunk_join_block(const attention_args &a, const chunk_split &split, int block) {
    constexpr int E = (D + 63) / 64;
    const int64_t row = (int64_t)block * JOIN_ROWS + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (row >= min(a.ntokens, (int64_t)a.cu[a.nreq]) * a.q_heads) return;
    const int64_t t = row / a.q_heads;
    const int r = wave_search(a.nreq, [&](int i) { return a.cu[i] <= t; });
    if (t - a.cu[r] >= a.max_new || (split.without_few && attention_is_few(a, attention_held(a, r)))) return;   // it has no parts
    const float *const stats = split.stats + 2 * row * split.splits, *const parts = split.parts + row * split.splits * D;
    float top = NO_SCORE, all = 0.f, o[E] = {};
    for (int s = lane; s < split.splits; s += 64) top = fmaxf(top, stats[2 * s]);
    for (int d = 32; d > 0; d /= 2) top = fmaxf(top, __shfl_xor(top, d));
#pragma unroll 4
    for (int s = 0; s < split.splits; ++s) {
        const float share = __builtin_amdgcn_exp2f(stats[2 * s] - top);
        all += share * stats[2 * s + 1];
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (D % 64 == 0 || e * 64 + lane < D) o[e] += share * parts[s * D + e * 64 + lane];
    }
    T *const out = (T *)a.out + row * D;
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (D % 64 == 0 || e * 64 + lane < D) out[e * 64 + lane] = (T)(all != 0.f ? o[e] * VALUE_UNIT<T, C> / all : 0.f);
    if (lane == 0 && a.lse) a.lse[row] = all != 0.f ? (top + log2f(all)) * LN2 : -INFINITY;
}

}  // namespace pq
