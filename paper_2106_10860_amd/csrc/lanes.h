// Values exchanged and reduced between the lanes of a wavefront, without memory.
#pragma once

#include "device_common.h"

namespace maddness {

// The value that lane (l + D) mod 16 of the row of 16 lanes has (D = 8, 4, 2, 1), lane l ^ 16, lane l ^ 32.
template <int D>
__device__ __forceinline__ uint32_t from_lane(uint32_t x)
{
    if constexpr (D < 16) {
        return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x120 + D, 0xf, 0xf, true);
    } else if constexpr (D == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        return threadIdx.x & 16 ? r[0] : r[1];
    } else {
        const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        return threadIdx.x & 32 ? r[0] : r[1];
    }
}

template <int D>
__device__ __forceinline__ float from_lane(float x) { return __uint_as_float(from_lane<D>(__float_as_uint(x))); }

template <int D>
__device__ __forceinline__ double from_lane(double x)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    return __builtin_bit_cast(double, from_lane<D>((uint32_t)b) | ((uint64_t)from_lane<D>((uint32_t)(b >> 32)) << 32));
}

// f over the LANES (16 or 64) lanes that share a token, in all of them.
template <int LANES, typename T, typename F>
__device__ __forceinline__ T over_lanes(T x, F f)
{
    x = f(x, from_lane<8>(x));
    x = f(x, from_lane<4>(x));
    x = f(x, from_lane<2>(x));
    x = f(x, from_lane<1>(x));
    if constexpr (LANES == 64) {
        x = f(x, from_lane<16>(x));
        x = f(x, from_lane<32>(x));
    }
    return x;
}

constexpr auto plus = [](auto a, auto b) INLINE_LAMBDA { return a + b; };

}  // namespace maddness
