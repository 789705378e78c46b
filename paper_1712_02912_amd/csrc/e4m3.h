// Elements of a cache of 8 bits (pq_kv_cache8): e4m3 numbers and their scales.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace pq {

struct e4m3 {
    uint8_t bits;
    __device__ __forceinline__ explicit operator float() const { return __builtin_amdgcn_cvt_pk_f32_fp8(bits, false)[0]; }
};
constexpr float E4M3_LARGEST = 448.f;   // 1.75 * 2^8

// Two numbers, to the nearest, ties to the even one, in the lower half of a word; those above the largest become it.
__device__ __forceinline__ uint32_t e4m3_of(float x, float y) {
    // (comparisons, not minima: NaN stays)
    x = x > E4M3_LARGEST ? E4M3_LARGEST : x < -E4M3_LARGEST ? -E4M3_LARGEST : x;
    y = y > E4M3_LARGEST ? E4M3_LARGEST : y < -E4M3_LARGEST ? -E4M3_LARGEST : y;
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x, y, 0, false) & 0xffffu;
}

// Four numbers in a word.
__device__ __forceinline__ uint32_t e4m3_of(const float *x) { return e4m3_of(x[0], x[1]) | e4m3_of(x[2], x[3]) << 16; }

// The same of numbers that are 448 at most, or NaN.
__device__ __forceinline__ uint32_t e4m3_of_held(const float *x) {
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false), true);
}

// Scales are handled by their exponents, from -126 on.
constexpr int LEAST_EXPONENT = -126;
__device__ __forceinline__ int scale_exponent(float scale) {
    const int e = (int)(__builtin_bit_cast(uint32_t, scale) >> 23 & 255u) - 127;
    return min(max(e, LEAST_EXPONENT), 127);
}
__device__ __forceinline__ float scale_of(int exponent) { return __builtin_bit_cast(float, (uint32_t)(exponent + 127) << 23); }
// The least exponent whose scale puts amax at 448 or below (amax >= 0, finite).
__device__ __forceinline__ int exponent_for(float amax) {
    const uint32_t bits = __builtin_bit_cast(uint32_t, amax);
    return max((int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0), LEAST_EXPONENT);
}
// |x| if it is finite, else 0
__device__ __forceinline__ float finite_size(float x) { return fabsf(x) < INFINITY ? fabsf(x) : 0.f; }

}  // namespace pq
