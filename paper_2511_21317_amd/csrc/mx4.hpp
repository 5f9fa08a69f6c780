// Rows of 64 channels in 4 bits: e2m1 codes (a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6), two channels a byte, the even one in
// the low half, with a power of two per block of 32 channels, held as its exponent + 127 in a byte (255: the block is NaN).  A
// cache's row of a key head has 32 bytes of key codes, 32 of value codes and four exponents: key and value of the first
// block, key and value of the second, so that a lane's block has both of its exponents in two bytes.
//
// The matrix cores would take such codes as they are, but only next to a B operand of at most 8 bits: queries as two e4m3 terms in
// one 16x16x128 product came out 7e-5 of sum |q k| off, the sums of it are not kept in 32 bits.  The conversions to bf16 are exact
// and take one instruction for two channels.
#pragma once
#include "dev_common.hpp"

namespace httm {

constexpr int kMxRowBytes = kDHead / 2;
constexpr int kMxScaleBytes = 4;

// The exponent byte of a block from the bits of its largest |x|: that of x rounded to two bits of significand, less two, so that
// x, held as 4 or 6 units, lies at 3.5 to 7 of them, and nothing in the block is more than half a step off.  The smallest unit is 2^-126, below which codes lose
// bits; the largest 2^125, at which the last quarter below 2^128 is held as 6 units: 2^126 would make it infinite.
// Infinities and NaN make the block NaN.
__device__ __forceinline__ uint32_t mx4_exponent(uint32_t top) {
  const int e = (int)((top + 0x200000u) >> 23) - 2;
  return top >= 0x7F800000u ? 255u : (uint32_t)(e < 1 ? 1 : e > 252 ? 252 : e);
}
// 8 channels to codes, nearest, ties to the even code
__device__ __forceinline__ uint32_t mx4_codes(const float (&x)[8], uint32_t exponent) {
  const float unit = __uint_as_float(exponent << 23);
  uint32_t r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[0], x[1], unit, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], unit, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], unit, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], unit, 3);
}
// 8 codes to bf16 (exact); `unit` has the exponent byte in its bits 23 .. 30 (0 stands for 2^-127 as it should)
__device__ __forceinline__ u32x4 mx4_values(uint32_t codes, float unit) {
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 0)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 1)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 2)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 3))};
}
// A block's two exponents (key low, value high) as units
__device__ __forceinline__ float mx4_key_unit(uint32_t pair) { return __uint_as_float((pair & 0xFFu) << 23); }
__device__ __forceinline__ float mx4_value_unit(uint32_t pair) { return __uint_as_float((pair >> 8 & 0xFFu) << 23); }

}  // namespace httm
