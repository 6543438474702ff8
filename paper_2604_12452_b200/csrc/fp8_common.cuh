// Conversions between fp32 / bf16 and 8-bit floating-point codes, four at a time in one 32-bit word (lowest byte first).
#pragma once

#include <cuda_fp16.h>
#include <stdint.h>

namespace lca {

// Smallest exponent of a block's scale: blocks of zeros, or of values below 2^-92.  Keeps 1 / scale and the sums of
// softmax weights over scales (at most 2^100 per row) inside fp32.
static constexpr int PAGED8_MIN_EXP = -100;

__device__ __forceinline__ float exp2_int(int e) { return __int_as_float((e + 127) << 23); }   // -126 <= e <= 127

// round to nearest even, saturating at +-448 (infinities too); NaN stays NaN
__device__ __forceinline__ uint32_t e4m3x4_from_float(float a, float b, float c, float d) {
  uint32_t r;
  asm("{\n\t.reg .b16 lo, hi;\n\tcvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n\t"
      "mov.b32 %0, {lo, hi};\n\t}" : "=r"(r) : "f"(a), "f"(b), "f"(c), "f"(d));
  return r;
}
__device__ __forceinline__ uint32_t e5m2x4_from_float(float a, float b, float c, float d) {
  uint32_t r;
  asm("{\n\t.reg .b16 lo, hi;\n\tcvt.rn.satfinite.e5m2x2.f32 lo, %2, %1;\n\tcvt.rn.satfinite.e5m2x2.f32 hi, %4, %3;\n\t"
      "mov.b32 %0, {lo, hi};\n\t}" : "=r"(r) : "f"(a), "f"(b), "f"(c), "f"(d));
  return r;
}
// e5m2 is the upper half of f16
__device__ __forceinline__ void e5m2x4_to_float(uint32_t v, float (&f)[4]) {
  const uint32_t lo = __byte_perm(v, 0u, 0x1404), hi = __byte_perm(v, 0u, 0x3424);
  const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&lo)), y = __half22float2(*reinterpret_cast<const __half2*>(&hi));
  f[0] = x.x; f[1] = x.y; f[2] = y.x; f[3] = y.y;
}
__device__ __forceinline__ float4 e4m3x4_to_float4(uint32_t v) {
  uint32_t lo, hi;
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
      : "=r"(lo), "=r"(hi) : "r"(v));
  const float2 x = __half22float2(*reinterpret_cast<__half2*>(&lo)), y = __half22float2(*reinterpret_cast<__half2*>(&hi));
  return make_float4(x.x, x.y, y.x, y.y);
}
// two f16 values <-> two codes in the low half of a word
__device__ __forceinline__ uint32_t e4m3x2_from_half2(__half2 v) {
  unsigned short r;
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(r) : "r"(*reinterpret_cast<uint32_t*>(&v)));
  return r;
}
__device__ __forceinline__ __half2 half2_from_e4m3x2(uint32_t c) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((unsigned short)c));
  return *reinterpret_cast<__half2*>(&r);
}
// codes * f, rounded again
__device__ __forceinline__ uint32_t e4m3x4_scale(uint32_t v, float f) {
  const float4 x = e4m3x4_to_float4(v);
  return e4m3x4_from_float(x.x * f, x.y * f, x.z * f, x.w * f);
}
// four bf16 values (two words) * f
__device__ __forceinline__ uint32_t e4m3x4_from_bf16(uint32_t lo, uint32_t hi, float f) {
  return e4m3x4_from_float(__uint_as_float(lo << 16) * f, __uint_as_float(lo & 0xffff0000u) * f,
                           __uint_as_float(hi << 16) * f, __uint_as_float(hi & 0xffff0000u) * f);
}

}  // namespace lca
