// Caches held in 8 bits: an element stands for e4m3 times the scale of its (page, kv head).  e4m3 (the OCP form) keeps 4
// significant bits between 2^-6 and 448, fewer down to 2^-9, has no infinity and a NaN with all seven bits set.
//
// Scales that the library writes are powers of two.  They cost an e4m3 nothing (its exponent is what a finer scale would move;
// only values below 2^-6 of the scaled range lose bits), and they make a page cheap to keep: when a louder token arrives, the
// kept ones are rounded again by a power of two, which changes none of them but those that become subnormal.
#pragma once
#include "device_utils.h"

namespace adaspec {

constexpr int kPageTokens = 16;
constexpr int kLeastScaleLog2 = -100, kMostScaleLog2 = 120;     // 448 * 2^120 is about the largest float

// bytes 0, 1 (kHigh: 2, 3) of a word
template <bool kHigh>
__device__ __forceinline__ void e4m3_to_float2(uint32_t w, float &a, float &b)
{
    typedef float f2 __attribute__((ext_vector_type(2)));
    const f2 v = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, kHigh);
    a = v[0];
    b = v[1];
}
// x, of magnitude up to 448 (by at most a rounding more) or not finite, to e4m3, nearest even; what is not finite becomes NaN
__device__ __forceinline__ float e4m3_input(float x) { return fabsf(x) <= 3.4028235e38f ? x : __uint_as_float(0x7fc00000u); }
__device__ __forceinline__ uint32_t float4_to_e4m3(float a, float b, float c, float d)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_input(a), e4m3_input(b), 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_input(c), e4m3_input(d), w, true);
    return (uint32_t)w;
}
__device__ __forceinline__ uint32_t float2_to_e4m3(float a, float b)
{
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(e4m3_input(a), e4m3_input(b), 0, false) & 0xffffu;
}

// elements times `ratio` (at most 1: nothing overflows), rounded again
__device__ __forceinline__ uint32_t e4m3_rescale4(uint32_t w, float ratio)
{
    float f[4];
    e4m3_to_float2<false>(w, f[0], f[1]);
    e4m3_to_float2<true>(w, f[2], f[3]);
    return float4_to_e4m3(f[0] * ratio, f[1] * ratio, f[2] * ratio, f[3] * ratio);
}
__device__ __forceinline__ void e4m3_rescale8(const uint8_t *from, uint8_t *to, float ratio)
{
    const uint2 w = *reinterpret_cast<const uint2 *>(from);
    *reinterpret_cast<uint2 *>(to) = make_uint2(e4m3_rescale4(w.x, ratio), e4m3_rescale4(w.y, ratio));
}

// log2 of the least power of two s with most <= (448 s)^2: 448^2 = 1.53125 * 2^17.  In squares of 64 bits, so that it does not
// depend on any rounding (products of two floats are exact there).
__device__ __forceinline__ int scale_log2_for(double most)
{
    const unsigned long long bits = __double_as_longlong(most);
    const int over = (int)((bits >> 52) & 0x7ff) - 1023 - 17;       // most = f 2^17 2^over, 1 <= f < 2
    const bool above = (bits & 0xfffffffffffffull) > 0x8800000000000ull;
    const int e = (over >> 1) + ((over & 1) || above ? 1 : 0);
    return most > 0.0 ? min(max(e, kLeastScaleLog2), kMostScaleLog2) : kLeastScaleLog2;
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

}  // namespace adaspec
