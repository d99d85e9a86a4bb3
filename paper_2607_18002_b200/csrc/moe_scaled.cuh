// Rows in e4m3 with an fp32 scale per 128 neighbours: the arithmetic that the quantisers and the products share.
//
// The scale of a block is amax times the fp32 number nearest to 1/448 (448: the largest e4m3 value), rounded once, 1 for a block of zeros, 2^-126 at least (a
// normal number, so that its reciprocal is one too).  That it is this product, and not the nearest number to amax / 448, counts: of 16-bit values one in some hundred is as far
// from two codes for a scale of amax / 448, and the last bit of the scale says which it gets.  (The re-quantisation inside moe_run divides: there the code is a product with 448 / amax.)  A block that holds a NaN or an infinity has a NaN scale, which makes all of its values NaN.
#pragma once
#include <stdint.h>

namespace moe {

constexpr int kScaledBlock = 128;

// of a block whose largest magnitude has these bits (NaN and infinities are above every number)
__device__ __forceinline__ float scaled_scale(unsigned amax_bits) {
  if (amax_bits >= 0x7f800000u) return __uint_as_float(0x7fffffffu);
  return amax_bits == 0u ? 1.f : fmaxf(__uint_as_float(amax_bits) * (1.f / 448.f), 0x1p-126f);
}
// two e4m3 codes, `first` in the low byte; rounded to nearest, ties to even, magnitudes above 448 to 448
__device__ __forceinline__ unsigned e4m3_codes2(float first, float second) {
  unsigned short r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %2, %1;" : "=h"(r) : "f"(first), "f"(second));
  return r;
}
__device__ __forceinline__ unsigned e4m3_codes4(const float* v) { return e4m3_codes2(v[0], v[1]) | e4m3_codes2(v[2], v[3]) << 16; }

}  // namespace moe
