// Sums over a wave on the vector ALU.
#pragma once
#include <type_traits>

#include "common.h"

namespace vpe {

// Sum over the 64 lanes in every lane, by row permutations and half exchanges (an exchange through the LDS crossbar takes ~100 clocks, six of
// them per sum and four sums per row are what a single row waits for).
__device__ __forceinline__ float wave_total(float v) {
    auto dpp = [](float x, auto ctrl) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(ctrl)::value, 0xF, 0xF, true)); };
    v += dpp(v, std::integral_constant<int, 0xB1>{});         // quad_perm [1,0,3,2]
    v += dpp(v, std::integral_constant<int, 0x4E>{});         // quad_perm [2,3,0,1]
    v += dpp(v, std::integral_constant<int, 0x141>{});        // mirror within eight
    v += dpp(v, std::integral_constant<int, 0x140>{});        // mirror within sixteen
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

}  // namespace vpe
