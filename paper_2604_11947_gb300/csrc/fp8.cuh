// fp8.cuh -- e4m3 values in units of a shared fp32 scale (the 8-bit form of include/resbm_train.h).
#pragma once

#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <stdint.h>

namespace resbm {

constexpr float kE4m3Max = 448.0f;
constexpr float kE4m3Least = 0.001953125f;                    // 2^-9, the smallest value above zero
constexpr float kScaleLeast = 7.888609052210118e-31f;         // 2^-100: 448 / most stays finite

// A group's scale and the factor that takes a value to units of it. `bits`: the largest |x| of the group as an
// unsigned integer (the bits of non-negative floats order as the floats do, a NaN above everything, so that
// an integer maximum passes a NaN on where a float maximum would drop it).
struct E4m3Scale {
    float scale, inv;
};
__device__ __forceinline__ E4m3Scale e4m3_scale(uint32_t bits)
{
    const uint32_t least = __float_as_uint(kScaleLeast);
    const float most = __uint_as_float(bits > least ? bits : least);
    return {most * (1.0f / kE4m3Max), __frcp_rn(most) * kE4m3Max};
}

__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// The four codes of four values in units of their scale, the first in the lowest byte (to nearest even,
// saturating at 448; a NaN gives the NaN code).
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d)
{
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
    return lo | (hi << 16);
}
__device__ __forceinline__ uint8_t e4m3x1(float a)
{
    return (uint8_t)__nv_cvt_float_to_fp8(a, __NV_SATFINITE, __NV_E4M3);
}

// The values of four codes (exact in half precision)
__device__ __forceinline__ float4 from_e4m3x4(uint32_t u)
{
    const __half2 lo(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(u & 0xFFFFu), __NV_E4M3));
    const __half2 hi(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(u >> 16), __NV_E4M3));
    const float2 a = __half22float2(lo), b = __half22float2(hi);
    return make_float4(a.x, a.y, b.x, b.y);
}
__device__ __forceinline__ float from_e4m3(uint8_t u)
{
    return __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)u, __NV_E4M3)));
}

}  // namespace resbm
