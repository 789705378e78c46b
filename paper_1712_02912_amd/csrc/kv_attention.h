// What the attention kernels share (kv_attention_kernels.hip, kv_attention_few.h, kv_attention_chunk.h).
#pragma once
#include <limits.h>
#include <math.h>

#include "e4m3.h"
#include "elem.h"
#include "pq_internal.h"
#include "wave_sums.h"

namespace pq {

struct attention_args {
    pq_kv_cache cache;   // (elem: the queries'; a cache of 8 bits has the same layout in its own elements, and scales)
    const float *k_scales, *v_scales;   // [blocks][heads], of a cache of 8 bits
    pq_heads q;
    const int32_t *cu, *kv_lens, *tables;
    void *out;
    float *lse;
    int64_t ntokens;
    int q_heads, nreq, width, window, max_new;
    int group;          // query heads that read one head of the cache
    uint32_t k_strides[2], v_strides[2];   // of blocks and places of the cache, where the matrix cores are taken
    fast_div by_block, by_group;
    float scale_log2;   // scale * log2(e): softmax in powers of two
};

constexpr float LN2 = 0.6931471805599453f;
// Reference of a running softmax that has seen no key: below every score, and finite, so that no -inf - -inf is formed.
constexpr float NO_SCORE = -3e38f;

// A request's length (refused requests have -1; so has what lies below, that no difference leaves 32 bits) and its keys as its
// table can hold them (kv_lens is the caller's: memory is read by it).
__device__ __forceinline__ int attention_length(const attention_args &a, int r) { return max(a.kv_lens[r], -1); }
__device__ __forceinline__ int attention_keys(const attention_args &a, int r) { return min(attention_length(a, r), a.width * a.cache.block_size); }
// New tokens of a request whose rows are computed: of all, those that have a row, up to max_new.
__device__ __forceinline__ int attention_held(const attention_args &a, int r) {
    return (int)min((int64_t)min(a.cu[r + 1] - a.cu[r], a.max_new), a.ntokens - a.cu[r]);
}

// A block table's entry; blocks outside the cache read as block 0 (memory stays in bounds, see pq_read.h).
__device__ __forceinline__ int64_t attention_block(const attention_args &a, int32_t entry) { return (unsigned)entry < (uint64_t)a.cache.nblocks ? entry : 0; }
// Position j of a request as (block, place).
__device__ __forceinline__ void attention_place(const attention_args &a, int r, int j, int64_t &block, int &place) {
    const int column = (int)a.by_block.div((uint32_t)j);
    place = j - column * a.cache.block_size;
    block = attention_block(a, a.tables[(int64_t)r * a.width + column]);
}

// Where a place's keys and values are, in elements (one multiply-add of 32 by 32 bits for each stride).
__device__ __forceinline__ uint64_t attention_key_at(const attention_args &a, int64_t block, int place) {
    return (uint64_t)(uint32_t)block * a.k_strides[0] + (uint64_t)(uint32_t)place * a.k_strides[1];
}
__device__ __forceinline__ uint64_t attention_value_at(const attention_args &a, int64_t block, int place) {
    return (uint64_t)(uint32_t)block * a.v_strides[0] + (uint64_t)(uint32_t)place * a.v_strides[1];
}

// ---- the matrix cores on 16-bit elements ---------------------------------------------------------------
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));   // eight elements, as they are moved
typedef short s16x4 __attribute__((ext_vector_type(4)));

template <class T> struct mfma_of;
template <> struct mfma_of<_Float16> {
    typedef _Float16 v8 __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ f32x4 m16(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x16 m32(u32x4 a, u32x4 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
};
template <> struct mfma_of<__bf16> {
    typedef __bf16 v8 __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ f32x4 m16(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x16 m32(u32x4 a, u32x4 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
};

// Whether one of eight elements is inf or NaN (the exponent's bits are all set).
template <class T> __device__ __forceinline__ bool any_not_finite(u32x4 x) {
    constexpr uint32_t e = __is_same(T, _Float16) ? 0x7c00u : 0x7f80u;
    bool found = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) found |= (x[i] & e) == e || (x[i] >> 16 & e) == e;
    return found;
}
// The same eight with those as zeros.
template <class T> __device__ __forceinline__ u32x4 finite_only(u32x4 x) {
    constexpr uint32_t e = __is_same(T, _Float16) ? 0x7c00u : 0x7f80u;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = ((x[i] & e) == e ? 0u : x[i] & 0xffffu) | ((x[i] >> 16 & e) == e ? 0u : x[i] & 0xffff0000u);
    return x;
}

// Adds those of four elements of a row of values that are inf or NaN.
template <class T, class V> __device__ __forceinline__ void add_not_finite(const T *v, V &out, int at) {
    const elem_vec<T, 4> x = *(const elem_vec<T, 4> *)v;
#pragma unroll
    for (int e = 0; e < 4; ++e) out[at + e] += !(fabsf((float)x.v[e]) < INFINITY) ? (float)x.v[e] : 0.f;
}

// four elements of a column: lane 4 r + c of 16 gives the address of part c of row r, lane n gets column n of the four rows
__device__ __forceinline__ uint2 read_transposed(const void *lds) {
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)lds));
}

// Weights are rounded to the cache's type for the product with the values: at most half a unit in the last place each, which
// is what the values themselves were rounded by, where a product in fp32 would take sixteen times as long.  Their sum is of
// those before the rounding.  Those of f16, whose least is 2^-24, are scaled by 2^7 (the sum with them): with the 2^8 by which
// a score may pass the reference the largest is 2^15, and weights of 2^-32 of a row's first still count.
template <class T> constexpr float WEIGHT_ROOM = __is_same(T, _Float16) ? 7.f : 0.f;
template <class T> __device__ __forceinline__ u32x4 pack8(const float *p) {
    typename mfma_of<T>::v8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (T)p[i];
    return __builtin_bit_cast(u32x4, v);
}

// Rows of keys or values in shared memory: bytes from row to row, and the 16-byte chunk of a row that chunk c of row k lies
// in.  Sixteen rows' equal chunks lie in different banks (rows written by a lane each, columns of keys read), and so do the
// even pairs of chunks of four rows that one transposing read takes.
template <int D> struct lds_row {
    static constexpr int bytes = D <= 64 ? 128 : D <= 128 ? 256 : 512;
    static __device__ __forceinline__ int chunk(int k, int c) {
        return c ^ (bytes == 128 ? ((k >> 1) & 3) << 1 | ((k >> 3) & 1) : (k & 7) << 1 | ((k >> 3) & 1));
    }
};

// ---- what the cache holds ---------------------------------------------------------------------------------
//
// The kernels on the matrix cores are built for caches of the queries' type T (C = T) and for e4m3 numbers (C = e4m3), which become
// elements of T on their way from the cache: two a conversion, times a power of two, and exact, but for f16 at the ends of its range.
// There a number times its scale may be 2^16, just above f16's largest, so f16 gets half of it, and twice the scale of the
// scores (from the host) and twice the result.
template <class T, class C> constexpr bool HALVED = __is_same(C, e4m3) && __is_same(T, _Float16);
template <class T, class C> constexpr float VALUE_UNIT = HALVED<T, C> ? 2.f : 1.f;

// Eight elements of two words of codes; scale: a power of two (only its exponent counts).
template <class T> __device__ __forceinline__ u32x4 from_e4m3(uint32_t low, uint32_t high, float scale) {
    if constexpr (__is_same(T, _Float16)) {
        return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)low, scale, false)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)low, scale, true)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)high, scale, false)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)high, scale, true))};
    } else {
        return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)low, scale, false)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)low, scale, true)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)high, scale, false)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)high, scale, true))};
    }
}
// A head's scale in a block, as the conversion takes it.
template <class T> __device__ __forceinline__ float e4m3_scale(const attention_args &a, const float *scales, int64_t block, int head) {
    return scales[block * a.cache.heads + head] * (HALVED<T, e4m3> ? 0.5f : 1.f);
}

// Adds those of four elements of a row of values that are NaN.
template <class T, class V> __device__ __forceinline__ void add_not_finite(const e4m3 *v, V &out, int at) {
    const elem_vec<e4m3, 4> x = *(const elem_vec<e4m3, 4> *)v;
#pragma unroll
    for (int e = 0; e < 4; ++e) out[at + e] += (x.v[e].bits & 0x7f) == 0x7f ? NAN : 0.f;
}

// Requests of so few rows per head of the cache have a kernel of their own.
constexpr int FEW_ROWS = 16;
__device__ __forceinline__ bool attention_is_few(const attention_args &a, int held) { return (int64_t)held * a.group <= FEW_ROWS; }

// The last of 0 ... n - 1 for which f holds; f holds from 0 up to there.  By a whole wave, 64 places at once, so that a
// search of a few hundred takes two loads one after the other, not nine.
template <class F> __device__ __forceinline__ int wave_search(int n, F f) {
    const int lane = threadIdx.x & 63;
    int low = 0;
    while (n > 1) {
        const int step = (n + 63) / 64, i = lane * step;
        const int last = __popcll(__ballot(i < n && f(low + i))) - 1;
        low += max(last, 0) * step;
        n = min(step, n - max(last, 0) * step);
    }
    return __builtin_amdgcn_readfirstlane(low);
}

// The request whose rows hold token t; -1 behind the last one.
__device__ __forceinline__ int attention_request(const int32_t *cu, int nreq, int64_t t) {
    if (t >= cu[nreq]) return -1;
    int low = 0, high = nreq;
    while (high - low > 1) {
        const int mid = (low + high) >> 1;
        if (cu[mid] <= t) low = mid;
        else high = mid;
    }
    return low;
}

// All requests, none of more than most_rows <= FEW_ROWS rows per head.
int launch_kv_attention_few(pq_ctx *ctx, const attention_args &a, int most_rows);
// All requests; some_few: those of few rows by the blocks of their own kind.
int launch_kv_attention_chunk(pq_ctx *ctx, const attention_args &a, bool some_few);
// The same over a cache of 8 bits.
int launch_kv_attention8_few(pq_ctx *ctx, const attention_args &a, int most_rows);
int launch_kv_attention8_chunk(pq_ctx *ctx, const attention_args &a, bool some_few);

}  // namespace pq
