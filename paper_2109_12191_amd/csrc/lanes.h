// Sums and maxima over the lanes of a wave, or over the lanes of it that share a row.  gfx950 only.
#pragma once

#include "internal.h"

namespace dp {

// Sum and largest of a wave's values, in every lane, by data-parallel-primitive moves.
__device__ __forceinline__ float wave_all_sum(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, wave_sum_last_lane(v)), 63));
}
__device__ __forceinline__ float wave_all_max(float v)
{
    auto step = [](float x, auto ctrl, auto rows) {              // lanes without a source keep their own value
        const int bits = __builtin_bit_cast(int, x);
        return fmaxf(x, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(bits, bits, decltype(ctrl)::value, decltype(rows)::value, 0xf, false)));
    };
    typedef std::integral_constant<int, 0xf> all_rows;
    v = step(v, std::integral_constant<int, 0x111>{}, all_rows{});
    v = step(v, std::integral_constant<int, 0x112>{}, all_rows{});
    v = step(v, std::integral_constant<int, 0x114>{}, all_rows{});
    v = step(v, std::integral_constant<int, 0x118>{}, all_rows{});
    v = step(v, std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});
    v = step(v, std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

// Sum or largest of the TPR lanes of a row, in each of them.
template <int TPR, bool MAX>
__device__ __forceinline__ float lanes_reduce(float v)
{
    auto step = [](float x, auto ctrl) {
        const float y = __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xf, 0xf, true));
        return MAX ? fmaxf(x, y) : x + y;
    };
    v = step(v, std::integral_constant<int, 0xB1>{});              // lane ^ 1
    v = step(v, std::integral_constant<int, 0x4E>{});              // lane ^ 2
    v = step(v, std::integral_constant<int, 0x141>{});             // the other four of eight
    if constexpr (TPR >= 16) v = step(v, std::integral_constant<int, 0x140>{});    // the other eight of sixteen
    if constexpr (TPR >= 32) {
        const float y = __shfl_xor(v, 16, 64);
        v = MAX ? fmaxf(v, y) : v + y;
    }
    return v;
}

}  // namespace dp
