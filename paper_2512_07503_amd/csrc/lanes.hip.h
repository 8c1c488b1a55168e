// Sums and maxima over lanes of a wavefront.
#pragma once
#include "common.hip.h"

// f of a team of lanes' x (TEAM = 1, 2, .. 64, aligned), in every one of them.  Within 16 lanes by moves that are part of f's instruction: neighbours, pairs, then mirror images of 8 and of
// 16 lanes, whose halves hold one number each by then; beyond by exchanging halves of 32 and of 64.
template <int CTRL> SJD_D float lanes_moved(float x) { return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xF, 0xF, true)); }
template <int TEAM, typename F> SJD_D float lanes_all(float x, F f) {
    if constexpr (TEAM > 1) x = f(x, lanes_moved<0xB1>(x));        // lanes 1 0 3 2
    if constexpr (TEAM > 2) x = f(x, lanes_moved<0x4E>(x));        // 2 3 0 1
    if constexpr (TEAM > 4) x = f(x, lanes_moved<0x141>(x));       // 7 6 .. 0
    if constexpr (TEAM > 8) x = f(x, lanes_moved<0x140>(x));       // 15 14 .. 0
    if constexpr (TEAM > 16) {
        const auto y = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(int, x), __builtin_bit_cast(int, x), false, false);
        x = f(__builtin_bit_cast(float, (int)y[0]), __builtin_bit_cast(float, (int)y[1]));
    }
    if constexpr (TEAM > 32) {
        const auto y = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(int, x), __builtin_bit_cast(int, x), false, false);
        x = f(__builtin_bit_cast(float, (int)y[0]), __builtin_bit_cast(float, (int)y[1]));
    }
    return x;
}
template <int TEAM> SJD_D float lanes_sum(float x) {
    return lanes_all<TEAM>(x, [](float a, float b) { return a + b; });
}
template <int TEAM> SJD_D float lanes_max(float x) {
    return lanes_all<TEAM>(x, [](float a, float b) { return fmaxf(a, b); });
}
