// fp8.cuh -- e4m3 codes of the 8-bit paged cache.
#pragma once

#include "common.cuh"

namespace hpd {

constexpr float kCodeMax = 448.f;                     // the largest e4m3 value
constexpr float kLeastScale = 7.888609052210118e-31f;  // 2^-100, of a page of zeros
constexpr float kMostScale = 1.329227995784916e+36f;   // 2^120, above the largest float / 448

// Two codes (the low byte first) as values, and back (to nearest, ties to even, beyond
// 448 to 448; NaN stays NaN).
__device__ __forceinline__ uint32_t f16_of_codes(uint32_t two) {
  uint32_t h;
  asm("{\n\t.reg .b16 c;\n\tcvt.u16.u32 c, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, c;\n\t}" : "=r"(h) : "r"(two));
  return h;
}
// Two f16 values that bf16 holds too.
__device__ __forceinline__ uint32_t bf16_of_f16(uint32_t h) {
  float x, y;
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(x), "=f"(y) : "r"(h));
  return pack_bf16x2(x, y);
}
__device__ __forceinline__ float2 of_codes(uint32_t two) {
  const uint32_t h = f16_of_codes(two);
  float2 r;
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}"
      : "=f"(r.x), "=f"(r.y)
      : "r"(h));
  return r;
}
__device__ __forceinline__ uint32_t to_codes(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
// Two values as f16 (to nearest, beyond its range to infinity).
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t to_codes4(float a, float b, float c, float d) {
  return to_codes(a, b) | to_codes(c, d) << 16;
}

}  // namespace hpd
