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

// The scale of values up to `most`: a product with 1/448 as 32 bits hold it, half of whose results are a unit off the
// quotient, so that it and not the quotient is what the header states.  Values become at most 448 (1 + 2^-21), which rounds
// to 448.  Its least value keeps its inverse finite.
__device__ __forceinline__ float e4m3_scale(float most) { return fmaxf(most * (1.0f / kTop), kLeastScale); }

// 1 / scale, rounded once: the instruction's result is a unit off at most, and the remainder corrects it (on gfx950 to what a
// division gives, for each of the 2^23 mantissas).
__device__ __forceinline__ float inverse(float scale) {
    const float q = __builtin_amdgcn_rcpf(scale);
    return fmaf(fmaf(-q, scale, 1.0f), q, q);
}

// x / scale, rounded once: the product with the rounded inverse is off by less than two units, and the remainder corrects it
// to 2^-22 of a unit before the rounding.  (The 180 million quotients of 24-bit numbers that lie within 2^-20 of a unit of the
// middle between two results all come out as a division gives them.)  The signs are such that -0 stays -0.
__device__ __forceinline__ float scaled(float x, float scale, float inverse) {
    const float q = x * inverse;
    return fmaf(-fmaf(q, scale, -x), inverse, q);
}

// Vectors of a lane by their scale.  Below 2^-64 both are multiplied by 2^64 first, so that the remainder of a quotient that 8
// bits tell from 0 is a number of 32 bits; an infinite scale gives 0 or NaN.  16,384 x 4,096 (bf16) into 8 bits with a scale
// for each row takes 49 us so, 56 with a division where one is small or infinite (8 registers more), and 47 multiplied by the
// inverse, which is one rounding more.
template <int NV, int V>
__device__ __forceinline__ void divide(float (&x)[NV][V], float scale) {
    constexpr float kSmall = 0x1p-64f;
    if (__any(scale < kSmall)) {
        const float up = scale < kSmall ? 1.0f / kSmall : 1.0f;
        scale *= up;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) x[j][i] *= up;
    }
    const bool finite = scale < __builtin_inff();
    const float inv = finite ? inverse(scale) : 0.0f;
    scale = finite ? scale : 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) x[j][i] = scaled(x[j][i], scale, inv);
}

template <int V>
__device__ __forceinline__ void divide(float (&x)[V], float scale) {
    divide(reinterpret_cast<float(&)[1][V]>(x), scale);
}

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
