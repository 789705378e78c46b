// Sums and the like over the lanes of a wave, in registers (lanes exchange by the data-parallel primitives, a few cycles a step).
#pragma once
#include <hip/hip_runtime.h>
#include <math.h>
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
struct op_larger {
    template <class V> static __device__ __forceinline__ V none() {
        if constexpr (__is_same(V, float)) return -INFINITY;
        else return V(0);   // (of whole numbers from 0 on)
    }
    template <class V> static __device__ __forceinline__ V of(V a, V b) { return a > b ? a : b; }
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

// what all lanes come to
template <class OP, class V> __device__ __forceinline__ V wave_total(V v) { return read_lane(wave_scan<OP>(v), 63); }

// what the lanes of a group come to, each of them; lanes: of a group, a power of two (all lanes of the wave are here)
template <class OP, class V> __device__ __forceinline__ V group_total(V v, int lanes) {
    if (lanes > 1) v = OP::template of<V>(v, from_lane<0xb1, 0xf>(v, v));    // neighbours
    if (lanes > 2) v = OP::template of<V>(v, from_lane<0x4e, 0xf>(v, v));    // pairs of four
    if (lanes > 4) v = OP::template of<V>(v, from_lane<0x141, 0xf>(v, v));   // fours of eight, mirrored
    if (lanes > 8) v = OP::template of<V>(v, from_lane<0x140, 0xf>(v, v));   // eights of sixteen, mirrored
    if (lanes > 16) v = OP::template of<V>(v, __shfl_xor(v, 16));
    if (lanes > 32) v = OP::template of<V>(v, __shfl_xor(v, 32));
    return v;
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
