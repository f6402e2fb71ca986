// Powers of two for the attention kernels, on the special-function unit and on the FMA pipes.
#pragma once

#include "common.cuh"

namespace lv {

__device__ __forceinline__ float fast_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// 2^(x - m) for a pair of arguments on the FMA pipes, `magic` = 1.5 * 2^23 - m with m a whole number.
// Adding it rounds x to the nearest integer and leaves n = that integer - m in the low mantissa
// bits; the fraction's power comes from a polynomial fitted on [-1/2, 1/2] and n is added to the exponent
// field; of a NaN that makes a number beyond the largest bf16, so its row still ends up not finite.
// Valid for x - m in [-126, 120].  The cubic is good to 7.5e-5 relative.  With kFull the degree is 6 and
// the result, rounding included, within 6.6e-8 of 2^(x - m): closer than the special-function unit,
// whose ex2.approx was measured at up to 1.45e-7 (5.4e-8 against 2.6e-8 in the mean square).
template <bool kFull>
__device__ __forceinline__ float2 poly_exp2_pair(float2 x, float2 magic, float2 neg_magic) {
  const float2 t = __fadd2_rn(x, magic);
  const float2 n = __fadd2_rn(t, neg_magic);
  const float2 f = __ffma2_rn(n, make_float2(-1.0f, -1.0f), x);
  auto horner = [&](float2 p, float c) { return __ffma2_rn(p, f, make_float2(c, c)); };
  float2 p;
  if constexpr (kFull) {
    p = horner(make_float2(1.5820509e-4f, 1.5820509e-4f), 1.341820345e-3f);
    p = horner(p, 9.617063217e-3f);
    p = horner(p, 5.55027239e-2f);
    p = horner(p, 0.2402265519f);
    p = horner(p, 0.6931472421f);
    p = horner(p, 1.0f);
  } else {
    p = horner(make_float2(0.0551716648f, 0.0551716648f), 0.2426111251f);
    p = horner(p, 0.6932609677f);
    p = horner(p, 0.9999280572f);
  }
  float2 r;
  r.x = __uint_as_float(__float_as_uint(p.x) + (__float_as_uint(t.x) << 23));
  r.y = __uint_as_float(__float_as_uint(p.y) + (__float_as_uint(t.y) << 23));
  return r;
}
__device__ __forceinline__ float2 poly_exp2_pair(float2 x) {
  return poly_exp2_pair<false>(x, make_float2(12582912.0f, 12582912.0f), make_float2(-12582912.0f, -12582912.0f));
}

}  // namespace lv
