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

// The 4-bit form: E2M1 codes x (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) under one power of two 2^e for every 32 channels,
//   e = the least whole number >= -126 with max |block| <= 6 * 2^e, stored as the byte e + 127 (255: not finite, codes of zero)
// the code of an even channel in the low half of its byte.  Again every x 2^e is a bf16 number, so that reading is exact; blocks of 32
// because a code has one bit of mantissa and a range of twelve: what shares a power of two with an element twelve times as large is
// lost, and in a whole row that is common.  Under 2^126 codes end at 3: 4 * 2^126 would be no number.
constexpr uint32_t kKv4LastByte = 253u;
__device__ __forceinline__ uint32_t kv4_exponent_byte(uint32_t top) {
  if (top >= 0x7f80u) return kKvNanByte;
  // top = m 2^x, 1 <= m < 2: 6 = 1.5 * 2^2, so e = x - 2, or one more where m > 1.5
  const int byte = (int)(top >> 7) - 2 + ((top & 0x7fu) > 0x40u ? 1 : 0);
  return (uint32_t)max(byte, 1);
}
// As kv_factor: the bits of a code moved into a bf16 stand for x 2^-126.
__device__ __forceinline__ KvFactor kv4_factor(uint32_t byte) {
  KvFactor f;
  f.first = byte == kKvNanByte ? 0x7fc0u : min(byte + 126u, 254u) << 7;
  f.second = byte == kKvNanByte ? 0x3f80u : max((int)byte - 1, 127) << 7;
  return f;
}
__device__ __forceinline__ bool kv4_needs_second(uint32_t byte) { return byte > 128u; }  // (blocks whose largest magnitude is over 12)
// The codes in the low and in the high halves of four bytes, a byte each.
__device__ __forceinline__ uint32_t kv4_low(uint32_t w) { return w & 0x0f0f0f0fu; }
__device__ __forceinline__ uint32_t kv4_high(uint32_t w) { return w >> 4 & 0x0f0f0f0fu; }
// Codes that are bytes of `low` and of `high` to four pairs of bf16, times a pair of factors.  A code's bits times 2^6 + 2^12 are its
// magnitude's where they belong, and its sign's, and others that a mask takes out: a multiplication, which the FMA pipes have time
// for, in place of the shifts that the logic unit, which bounds all this, has not.
__device__ __forceinline__ void kv4_widen_by(uint32_t low, uint32_t high, uint32_t factors, uint32_t (&out)[4]) {
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) {
    uint32_t t;  // (8: the sign of a byte that has none, a byte of zeros; __byte_perm does not know it)
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(t) : "r"(low), "r"(high), "r"(0x8480u + 0x101u * i));
    out[i] = mul_bf16x2(t * 0x1040u & 0x81c081c0u, factors);
  }
}
// Eight codes of a block to eight bf16.
__device__ __forceinline__ void kv4_widen(uint32_t w, uint32_t byte, uint32_t (&out)[4]) {
  const KvFactor f = kv4_factor(byte);
  kv4_widen_by(kv4_low(w), kv4_high(w), f.first * 0x10001u, out);
  if (kv4_needs_second(byte)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = mul_bf16x2(out[i], f.second * 0x10001u);
  }
}
// Eight floats, at most 6 in magnitude, to eight codes.
__device__ __forceinline__ uint32_t pack_e2m1x8(const float (&x)[8]) {
  uint32_t r;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(r)
      : "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]));
  return r;
}

// What a pool holds of a row of a head: bytes of values or codes, and of exponents.
template <int kHd, int kKind>
struct KvRow {
  static constexpr int kBytes = kKind == LITEVGGT_KV_BF16 ? 2 * kHd : kKind == LITEVGGT_KV_E4M3 ? kHd : kHd / 2;
  static constexpr int kExps = kKind == LITEVGGT_KV_BF16 ? 0 : kKind == LITEVGGT_KV_E4M3 ? 1 : kHd / 32;
};

}  // namespace lv
