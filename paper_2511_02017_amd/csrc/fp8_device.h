// 8-bit floating point (E4M3: four exponent bits, three of the mantissa, largest value 448, no infinities) with a binary32 scale for 128 elements.
#pragma once

#include "head.h"

namespace tapout {

// The scale of a block whose largest magnitude has these bits: that magnitude times 1/448 (448: the type's largest value; both rounded to binary32).  A NaN or an infinity anywhere
// in the block (bits from 0x7f800000 on: magnitudes' bits order like the magnitudes) makes the scale, and with it every value, NaN.  Magnitudes
// below 448 times the smallest normal number share that one's scale, which keeps the quotients exact down there.
__device__ __forceinline__ float fp8_scale(uint32_t top)
{
    return top >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : fmaxf(__uint_as_float(top), 448.f * 0x1p-126f) * (1.f / 448.f);
}

// Four values over the scale, to nearest, ties to even.
__device__ __forceinline__ uint32_t fp8_pack(float a, float b, float c, float d, float scale)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a / scale, b / scale, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c / scale, d / scale, w, true);
}

// Largest of the bits that 2^LOG neighbouring lanes hold, in every one of them.
template <int LOG> __device__ __forceinline__ uint32_t fp8_top(uint32_t v)
{
    return (uint32_t)lanes_reduce_i((int)v, 0, LOG, [](int x, int y) { return max(x, y); });
}

}  // namespace tapout
