// Sums and the like over the lanes of a wave, in registers (lanes exchange by the data-parallel primitives, a few cycles a step).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace pq {

template <int CTRL, int ROWS, class V> __device__ __forceinline__ V from_lane(V none, V v) {
    if constexpr (sizeof(V) == 4) {
        return __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, none), __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false));
    } else {
        const int2 n = __builtin_bit_cast(int2, none), x = __builtin_bit_cast(int2, v);
        return __builtin_bit_cast(V, int2{__builtin_amdgcn_update_dpp(n.x, x.x, CTRL, ROWS, 0xf, false),
                                          __builtin_amdgcn_update_dpp(n.y, x.y, CTRL, ROWS, 0xf, false)});
    }
}
template <class V> __device__ __forceinline__ V read_lane(V v, int lane) {
    if constexpr (sizeof(V) == 4) {
        return __builtin_bit_cast(V, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
    } else {
        const int2 x = __builtin_bit_cast(int2, v);
        return __builtin_bit_cast(V, int2{__builtin_amdgcn_readlane(x.x, lane), __builtin_amdgcn_readlane(x.y, lane)});
    }
}
struct op_add {
    template <class V> static __device__ __forceinline__ V none() { return V(0); }
    template <class V> static __device__ __forceinline__ V of(V a, V b) { return a + b; }
};
// every lane gets what the lanes up to and with it come to, within its row of 16
template <class OP, class V> __device__ __forceinline__ V row_scan(V v) {
    v = OP::template of<V>(v, from_lane<0x111, 0xf>(OP::template none<V>(), v));
    v = OP::template of<V>(v, from_lane<0x112, 0xf>(OP::template none<V>(), v));
    v = OP::template of<V>(v, from_lane<0x114, 0xf>(OP::template none<V>(), v));
    return OP::template of<V>(v, from_lane<0x118, 0xf>(OP::template none<V>(), v));
}
template <class OP, class V> __device__ __forceinline__ V wave_scan(V v) {
    v = row_scan<OP>(v);
    v = OP::template of<V>(v, from_lane<0x142, 0xa>(OP::template none<V>(), v));
    return OP::template of<V>(v, from_lane<0x143, 0xc>(OP::template none<V>(), v));
}

// n / d for 0 <= n < 2^31, as a product
struct fast_div {
    uint32_t d, mul, shift;
    fast_div() = default;
    explicit fast_div(uint32_t by) : d(by), shift(0) {
        while (((uint64_t)1 << shift) < by) ++shift;
        mul = (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << shift) - by)) / by + 1);
    }
    __device__ __forceinline__ uint32_t div(uint32_t n) const { return (__umulhi(mul, n) + n) >> shift; }
};

}  // namespace pq
