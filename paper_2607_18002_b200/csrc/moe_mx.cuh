// Microscaled 4-bit rows (OCP MX: e2m1 values, a power-of-two scale per 32 neighbours): the arithmetic that the quantiser and the
// products share.
//
// The scale byte of a block is floor(log2(amax)) - 2 + 127, at least 0 (2 is the exponent of 6, the largest e2m1 value), so scaled values
// lie below 8 and those above 6 saturate.  Scaling by a power of two is exact, so the only rounding is the one to e2m1, to nearest, ties to
// the even code.  A block that holds a NaN or an infinity gets scale byte 255, which makes all of its values NaN.
#pragma once
#include <stdint.h>

namespace moe {

constexpr int kMxBlock = 32;

// of a block whose largest magnitude has these bits (NaN and infinities are above every number)
__device__ __forceinline__ unsigned mx_scale_byte(unsigned amax_bits) {
  const int exponent = (int)(amax_bits >> 23);
  return exponent == 255 ? 255u : (unsigned)max(exponent - 2, 0);
}
// 2^(127 - byte): the exponent field of the product is never out of range for bytes up to 253
__device__ __forceinline__ float mx_inverse(unsigned byte) { return __uint_as_float(byte == 255u ? 0u : (254u - byte) << 23); }
// 2^(byte - 127); 2^-127 is a subnormal number
__device__ __forceinline__ float mx_scale(unsigned byte) {
  return __uint_as_float(byte == 255u ? 0x7fffffffu : byte == 0u ? 0x00400000u : byte << 23);
}
// two codes in a byte's worth of bits, `even` in the low half
__device__ __forceinline__ unsigned mx_codes2(float even, float odd) {
  unsigned r;
  asm("{\n\t.reg .b8 c;\n\tcvt.rn.satfinite.e2m1x2.f32 c, %2, %1;\n\tcvt.u32.u8 %0, c;\n\t}" : "=r"(r) : "f"(even), "f"(odd));
  return r;
}

}  // namespace moe
