// fp8.cuh -- e4m3 codes of the 8-bit paged cache.
#pragma once

#include "common.cuh"

namespace hpd {

constexpr float kCodeMax = 448.f;                     // the largest e4m3 value
constexpr float kLeastScale = 7.888609052210118e-31f;  // 2^-100, of a page of zeros
constexpr float kMostScale = 2.658455991569832e+36f;   // 2^121, above twice the largest float / 448

// Four codes (the low byte first) as two pairs of f16, which holds every code.  (A half of
// a register is an operand as it is: masks and shifts would be as many instructions again,
// and had 11 % of the attention's time.)
__device__ __forceinline__ void f16_of_codes(uint32_t four, uint32_t &lo, uint32_t &hi) {
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\t"
      "cvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
      : "=r"(lo), "=r"(hi)
      : "r"(four));
}
__device__ __forceinline__ float2 floats_of_f16(uint32_t h) {
  float2 r;
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}"
      : "=f"(r.x), "=f"(r.y)
      : "r"(h));
  return r;
}
// Two f16 values that bf16 holds too.
__device__ __forceinline__ uint32_t bf16_of_f16(uint32_t h) {
  const float2 x = floats_of_f16(h);
  return pack_bf16x2(x.x, x.y);
}
// Two values as f16 (to nearest, beyond its range to infinity).
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// Four values as codes, to nearest, ties to even; beyond 448 to 448; NaN stays NaN.
__device__ __forceinline__ uint32_t to_codes4(float a, float b, float c, float d) {
  uint32_t r;
  asm("{\n\t.reg .b16 x, y;\n\tcvt.rn.satfinite.e4m3x2.f32 x, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 y, %4, %3;\n\t"
      "mov.b32 %0, {x, y};\n\t}"
      : "=r"(r)
      : "f"(a), "f"(b), "f"(c), "f"(d));
  return r;
}
// Four codes as values.
__device__ __forceinline__ void of_codes4(uint32_t four, float2 &lo, float2 &hi) {
  uint32_t a, b;
  f16_of_codes(four, a, b);
  lo = floats_of_f16(a);
  hi = floats_of_f16(b);
}

}  // namespace hpd
