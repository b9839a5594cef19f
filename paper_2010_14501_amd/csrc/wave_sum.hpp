// Sums and maxima over a wave, in every lane, without LDS: neighbours, fours, eights, 16 lanes, then the four rows of 16 through their last lanes.
#pragma once
#include <hip/hip_runtime.h>

namespace monet {

// v joined with the lane that CTRL names; lanes without one, and rows outside ROWS, with `none`
template <int CTRL, int ROWS, class F>
__device__ __forceinline__ float dpp_join(float v, float none, F &&f) {
    return f(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, none), __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false)));
}
template <class F>
__device__ __forceinline__ float wave_join(float v, float none, F &&f) {
    v = dpp_join<0xb1, 0xf>(v, none, f);       // quad_perm 1 0 3 2
    v = dpp_join<0x4e, 0xf>(v, none, f);       // quad_perm 2 3 0 1
    v = dpp_join<0x141, 0xf>(v, none, f);      // row_half_mirror
    v = dpp_join<0x140, 0xf>(v, none, f);      // row_mirror
    v = dpp_join<0x142, 0xa>(v, none, f);      // row_bcast15
    v = dpp_join<0x143, 0xc>(v, none, f);      // row_bcast31
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}
__device__ __forceinline__ float wave_sum(float v) {
    return wave_join(v, 0.f, [](float a, float b) { return a + b; });
}
// over four and over 16 neighbouring lanes, in all of them
__device__ __forceinline__ float quad_sum(float v) {
    const auto add = [](float a, float b) { return a + b; };
    v = dpp_join<0xb1, 0xf>(v, 0.f, add);
    return dpp_join<0x4e, 0xf>(v, 0.f, add);
}
__device__ __forceinline__ float row_sum(float v) {
    const auto add = [](float a, float b) { return a + b; };
    v = dpp_join<0x141, 0xf>(quad_sum(v), 0.f, add);
    return dpp_join<0x140, 0xf>(v, 0.f, add);
}
__device__ __forceinline__ float wave_max(float v) {
    return wave_join(v, -INFINITY, [](float a, float b) { return fmaxf(a, b); });
}

}  // namespace monet
