// The 8-bit form of a cached row: E4M3 codes x and one power of two 2^e, the value of an element being x 2^e.
//   e = the least whole number >= -118 with max |row| <= 448 * 2^e, stored as the byte e + 127
//   x = the element times 2^-e, rounded to E4M3 (nearest even); every x 2^e is a bf16 number
//   a row with an element that is not finite is held as byte 255, and reads as NaN
// A power of two costs a floating-point code no precision, and it makes reading exact: a code is widened by moving its bits
// into a bf16 and one multiplication, with no rounding behind which the attention or a reader would have to look.
#pragma once

#include "common.cuh"

namespace lv {

constexpr uint32_t kKvNanByte = 255u;

// The exponent byte of a row whose largest magnitude has the bf16 bits `top` (0x7f80 and more: not finite).
__device__ __forceinline__ uint32_t kv_exponent_byte(uint32_t top) {
  if (top >= 0x7f80u) return kKvNanByte;
  // top = m 2^x, 1 <= m < 2: 448 = 1.75 * 2^8, so e = x - 8, or one more where m > 1.75 (mantissa bits over 0x60)
  const int byte = (int)(top >> 7) - 8 + ((top & 0x7fu) > 0x60u ? 1 : 0);
  return (uint32_t)max(byte, 9);
}
// 2^-e
__device__ __forceinline__ float kv_inverse_scale(uint32_t byte) { return __uint_as_float((254u - min(byte, 253u)) << 23); }

// Two multiplications widen a code: its bits moved into a bf16 stand for x 2^-120, so the first factor is 2^(120 + e) where
// that is a bf16 number, the second what is missing beyond 2^127 (rows whose largest magnitude is over 57,344).
struct KvFactor {
  uint32_t first, second;  // bf16
};
__device__ __forceinline__ KvFactor kv_factor(uint32_t byte) {
  KvFactor f;
  f.first = byte == kKvNanByte ? 0x7fc0u : min(byte + 120u, 254u) << 7;
  f.second = byte == kKvNanByte ? 0x3f80u : max((int)byte - 7, 127) << 7;
  return f;
}
__device__ __forceinline__ bool kv_needs_second(uint32_t byte) { return byte > 134u; }

// Bytes 1 and 3 of `t` as a pair of bf16 numbers 2^-120 times their E4M3 values (bytes 0 and 2 may hold anything).
__device__ __forceinline__ uint32_t kv_code_bits(uint32_t t) { return ((t >> 4) & 0x07f007f0u) | (t & 0x80008000u); }

__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

}  // namespace lv
