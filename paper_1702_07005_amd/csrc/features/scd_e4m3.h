// scd_e4m3.h -- 8-bit values (e4m3: 4 bits of exponent, 3 of mantissa, no infinity) and the largest magnitudes that their
// scales come from.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "scd_device.h"

namespace scd {
namespace feat {

constexpr float kTop = 448.0f;          // the largest value
constexpr float kLeast = 0x1p-9f;        // the least above 0
constexpr float kLeastScale = 0x1p-126f;

// The scale of values up to `most`: they become at most 448 (1 + 2^-21), which rounds to 448.  Its least value keeps its
// inverse finite.
__device__ __forceinline__ float e4m3_scale(float most) { return fmaxf(most * (1.0f / kTop), kLeastScale); }

// To the nearest, ties to even.
__device__ __forceinline__ uint32_t e4m3_pack4(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// max |x| over groups of G lanes, 0 where all are NaN; every lane of a group gets it.  `w` (uniform, a power of two up to G)
// makes the groups smaller.
template <int G>
__device__ __forceinline__ float group_max(float x, int w) {
    if (G >= 2 && w >= 2) x = fmaxf(x, dpp_f<0xB1>(x));   // lane ^ 1
    if (G >= 4 && w >= 4) x = fmaxf(x, dpp_f<0x4E>(x));   // lane ^ 2
    if (G >= 8 && w >= 8) x = fmaxf(x, dpp_f<0x141>(x));  // other quad of 8
    if (G >= 16 && w >= 16) x = fmaxf(x, dpp_f<0x140>(x));
    if (G >= 32 && w >= 32) x = fmaxf(x, __int_as_float(__builtin_amdgcn_ds_swizzle(__float_as_int(x), 0x401F)));
    if (G >= 64 && w >= 64)
        x = fmaxf(__int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 0)), __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 32)));
    return x;
}

}  // namespace feat
}  // namespace scd
