// Values of other lanes of a wavefront, without the LDS crossbar (whose answers take some 130 cycles). Workgroups are one-dimensional.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dppo {

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true); }

// Both values of the pair of lanes X (16 or 32) apart, the one of the lane with bit X clear first.
template <int X>
__device__ __forceinline__ void pair_values(uint32_t v, uint32_t& low, uint32_t& high) {
    static_assert(X == 16 || X == 32, "rows of 16 lanes, halves");
    if constexpr (X == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        low = r[0]; high = r[1];
    } else {
        const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        low = r[0]; high = r[1];
    }
}
template <int X>
__device__ __forceinline__ float pair_max(float v) {
    uint32_t a, b;
    pair_values<X>(__float_as_uint(v), a, b);
    return fmaxf(__uint_as_float(a), __uint_as_float(b));
}
template <int X>
__device__ __forceinline__ float pair_sum(float v) {
    uint32_t a, b;
    pair_values<X>(__float_as_uint(v), a, b);
    return __uint_as_float(a) + __uint_as_float(b);
}

// The value of lane (own lane ^ X).
template <int X>
__device__ __forceinline__ uint32_t xor_lane(uint32_t v) {
    if constexpr (X == 1) return dpp<0xB1>(v);               // quad_perm 1 0 3 2
    else if constexpr (X == 2) return dpp<0x4E>(v);          // quad_perm 2 3 0 1
    else if constexpr (X == 3) return dpp<0x1B>(v);          // quad_perm 3 2 1 0
    else if constexpr (X == 7) return dpp<0x141>(v);         // row_half_mirror
    else if constexpr (X == 8) return dpp<0x128>(v);         // row_ror 8
    else if constexpr (X == 15) return dpp<0x140>(v);        // row_mirror
    else if constexpr (X == 4) return xor_lane<3>(xor_lane<7>(v));
    else if constexpr (X == 31) return xor_lane<16>(xor_lane<15>(v));
    else if constexpr (X == 63) return xor_lane<32>(xor_lane<31>(v));
    else {
        uint32_t a, b;
        pair_values<X>(v, a, b);
        return threadIdx.x & X ? a : b;
    }
}
template <int X>
__device__ __forceinline__ uint64_t xor_lane(uint64_t v) {
    return ((uint64_t)xor_lane<X>((uint32_t)(v >> 32)) << 32) | xor_lane<X>((uint32_t)v);
}
template <int X>
__device__ __forceinline__ float xor_lane(float v) { return __uint_as_float(xor_lane<X>(__float_as_uint(v))); }

}  // namespace dppo
