// Rows in 4 bits.  A row of D values is D / 32 blocks of 32 neighbouring channels; a block is a scale byte s, which stands for
// 2^(s - 127), and 32 codes of four bits, the lower channel in the lower nibble: sign, two bits of exponent, one of mantissa,
// i.e. 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives, times the scale.  s = 255: every value of the block is a NaN.
#pragma once

#include "kvs_device.h"

namespace kvs {
namespace fp4 {

constexpr int kBlock = 32;
constexpr uint32_t kNanScale = 255;
// Scales are 2^-125 to 2^125: what they make of the codes is neither subnormal nor beyond the largest number.
constexpr int kLeastScale = 127 - 125, kMostScale = 127 + 125;

// What two_of takes for a block with scale byte s: the conversion looks at the float's exponent alone, as a scale byte, so that
// 255 (an infinity) makes NaNs of all codes.
__device__ __forceinline__ float scale_of(uint32_t s) { return __uint_as_float(s << 23); }

// The two values of byte B of `codes`, as packed bf16 (exact).
template <int B>
__device__ __forceinline__ uint32_t two_of(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, B));
}

// The scale byte of a block whose largest magnitude has these bits: the smallest power of two with which no value rounds
// beyond 6, i.e. with which the largest is below 7 (from 7 on the nearest number of the next binade is 8).
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax_bits) {
  if (amax_bits >= 0x7f800000u) return kNanScale;
  const int s = (int)(amax_bits >> 23) - 2 + ((amax_bits & 0x7fffffu) >= 0x600000u ? 1 : 0);
  return min(max(s, kLeastScale), kMostScale);
}

}  // namespace fp4
}  // namespace kvs
