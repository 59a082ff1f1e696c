// Codes and scales of the pools in 8 bits: e4m3 codes, powers of two as the exponent byte of an fp32 number.
#pragma once
#include "tr_internal.h"

namespace {

constexpr int Q8_LEAST = -117, Q8_MOST = 120; // exponents of scales: 2^-9 2^-117 is normal, 448 2^120 is beyond the largest fp32 number

// The smallest e with top <= 448 * 2^e = 1.75 * 2^(e + 8), for the bits of a finite top >= 0.
__device__ __forceinline__ int q8_exponent(int top)
{
    const int e = (top >> 23) - (127 + 8) + ((top & 0x7fffff) > 0x600000);
    return min(max(e, Q8_LEAST), Q8_MOST);
}
__device__ __forceinline__ float q8_power(int e) { return __builtin_amdgcn_ldexpf(1.0f, e); }

// Four codes from four values, to nearest even; NaN and infinite ones become NaN.
__device__ __forceinline__ uint32_t q8_encode(float a, float b, float c, float d)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
// Their values.
__device__ __forceinline__ void q8_decode(uint32_t w, float (&x)[4])
{
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    x[0] = lo[0], x[1] = lo[1], x[2] = hi[0], x[3] = hi[1];
}

} // namespace
