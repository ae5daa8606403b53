// Codes of 8 bits (e4m3) and their scales (include/etc.h, etc_serving_append_codes), on the device.
#pragma once
#include "serving_rt.hip.h"

namespace etc {

// Four codes, nearest even, of values that are at most 448, or NaN.
__device__ __forceinline__ uint32_t to_f8x4(float a, float b, float c, float d)
{
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}
__device__ __forceinline__ f32x4 from_f8x4(uint32_t w)
{
    const auto x = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), y = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    return f32x4{x[0], x[1], y[0], y[1]};
}
__device__ __forceinline__ float finite_or_nan(float x) { return __builtin_fmaf(x, 0.f, x); }
// The scale of values up to `most` as its byte, `least` at least: the smallest E with most <= 1.75 * 2^(8 + E).
__device__ __forceinline__ int scale_byte(float most, int least)
{
    const uint32_t u = __float_as_uint(most);
    return max((int)(u >> 23) - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0), least);
}
__device__ __forceinline__ float one_over_scale(int byte) { return __uint_as_float((uint32_t)(254 - byte) << 23); }
// Eight codes as bf16, times a power of two: exact.
__device__ __forceinline__ u32x4 codes_to_bf16x8(uint32_t a, uint32_t b, float scale)
{
    return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true))};
}
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

}  // namespace etc
