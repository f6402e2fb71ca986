// The warp-wide product of the kernels for few rows: 16 rows by 8 columns by 16, bf16 or f16 operands, sums in 32 bits; and codes as its
// operands.
#pragma once

#include "common.cuh"

namespace lv {

template <bool kHalfFloat>
__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (kHalfFloat) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  } else {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  }
}
// Two codes (the low or the high half of a word) to two f16 numbers, exactly.
__device__ __forceinline__ uint32_t widen_low(uint32_t w) {
  uint32_t r;
  asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\t}" : "=r"(r) : "r"(w));
  return r;
}
__device__ __forceinline__ uint32_t widen_high(uint32_t w) {
  uint32_t r;
  asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, hi;\n\t}" : "=r"(r) : "r"(w));
  return r;
}
// The four bytes of a word, two E2M1 codes each, to pairs of f16 numbers, exactly; the low half's code to the low number.
__device__ __forceinline__ void widen_codes4(uint32_t w, uint32_t (&out)[4]) {
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "mov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
      "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
      "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(out[0]), "=r"(out[1]), "=r"(out[2]), "=r"(out[3])
      : "r"(w));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// Powers of two of exponent bytes side by side; infinity for 255.
__device__ __forceinline__ void power_word(uint32_t v, float (&p)[4]) {
  p[0] = __uint_as_float(v << 23 & 0x7f800000u);
  p[1] = __uint_as_float(v << 15 & 0x7f800000u);
  p[2] = __uint_as_float(v << 7 & 0x7f800000u);
  p[3] = __uint_as_float(v >> 1 & 0x7f800000u);
}

// The factor that brings a row's largest element, of the bf16 bits `top`, to [2^13, 2^14) in f16, and its inverse: rows of zeros or under
// 2^-113, and those that are not finite, as near as it goes.
__device__ __forceinline__ float2 f16_factor(uint32_t top) {
  if (top >= 0x7f80u) return make_float2(1.0f, 1.0f);
  const int up = min(max(13 - ((int)(top >> 7) - 127), -126), 126);
  return make_float2(__int_as_float((up + 127) << 23), __int_as_float((127 - up) << 23));
}

}  // namespace lv
