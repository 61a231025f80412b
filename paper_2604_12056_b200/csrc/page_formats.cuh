// Codes of the quantised K/V pages: E4M3 with a scale per page and KV head, and four bits with a scale per run of 32
// elements of a token's row.
#pragma once
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "common.cuh"

namespace losa {

// eight codes -> values, eight values -> codes (round to nearest even, saturate at +-448)
__device__ __forceinline__ void fp8_decode8(uint2 w, float (&v)[8]) {
  const uint32_t x[2] = {w.x, w.y};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(x[i >> 1] >> (16 * (i & 1))), __NV_E4M3);
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
    v[2 * i] = f.x;
    v[2 * i + 1] = f.y;
  }
}
__device__ __forceinline__ uint2 fp8_encode8(const float (&v)[8], float inv_scale) {
  uint32_t x[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    x[i] = __nv_cvt_float2_to_fp8x2(make_float2(v[2 * i] * inv_scale, v[2 * i + 1] * inv_scale), __NV_SATFINITE, __NV_E4M3);
  return make_uint2(x[0] | (x[1] << 16), x[2] | (x[3] << 16));
}
__device__ __forceinline__ float pow2f(int e) { return __int_as_float((127 + e) << 23); }   // -126 <= e <= 127
// e = the smallest integer in [-6, 7] with amax <= 448 * 2^e = 1.75 * 2^(e + 8)
__device__ __forceinline__ int fp8_scale_exp(float amax) {
  const uint32_t b = __float_as_uint(amax);
  const int e = static_cast<int>(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
  return min(7, max(-6, e));
}

// ---- 4-bit codes ------------------------------------------------------------------------------
constexpr int kInt4Run = 32;                       // elements under one scale
constexpr float kInt4MinScale = 0.000244140625f, kInt4MaxScale = 960.f;
// Scale of a run: the smallest number of four significant bits >= amax / 7, within the limits.  The quotient
// is rounded to fp32 first.  amax is a bf16 number: its quotient by 7 either has at most four significant bits, and is exact, or
// is further than fp32's rounding from any number that has (7 s has seven bits, amax eight).
__device__ __forceinline__ float int4_scale(float amax) {
  const uint32_t up = (__float_as_uint(__fdiv_rn(amax, 7.f)) + 0xfffffu) & ~0xfffffu;
  return fminf(fmaxf(__uint_as_float(up), kInt4MinScale), kInt4MaxScale);
}
// ... and as the cache holds it: a run with a NaN in it is NaN
__device__ __forceinline__ float int4_held_scale(float scale, float amax) { return amax != amax ? amax : scale; }
// the largest of three, NaN if one of them is
__device__ __forceinline__ float max_nan(float a, float b, float c) {
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// ... its byte: exponent and mantissa of the fp16 number (NaN: 255)
__device__ __forceinline__ uint32_t int4_scale_byte(float s) { return __half_as_ushort(__float2half_rn(s)) >> 7; }
__device__ __forceinline__ float int4_scale_value(uint32_t byte) { return __half2float(__ushort_as_half(static_cast<unsigned short>(byte << 7))); }
// x / s to the nearest integer, halves away from zero, as the float kInt4Magic + c, whose low four bits are the stored c + 8.
// The multiplier is a little more than 1 / s: a half, (k + 1/2) s, is a number of at most eight significant bits, so
// it is a bf16 number, and lies above the tie by 2^-16 of itself; the next bf16 number towards zero, 2^-9 of itself below, stays below it.
constexpr float kInt4Magic = 12582912.f + 8.f;     // 1.5 * 2^23 + 8: one unit is one unit in the last place
__device__ __forceinline__ float int4_multiplier(float s) { return __fdiv_rn(1.0000152587890625f, s); }
__device__ __forceinline__ float int4_round(float x, float mul) { return fmaf(x, mul, kInt4Magic); }
__device__ __forceinline__ uint32_t int4_bits(float m) { return __float_as_uint(m) & 15u; }
// eight codes of a word -> values
__device__ __forceinline__ void int4_decode8(uint32_t w, float s, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (__uint_as_float(0x4b400000u | ((w >> (4 * i)) & 15u)) - kInt4Magic) * s;
}

}  // namespace losa
