// Microscaled 4-bit values on the device: the conversions of gfx950, whose scale
// operand is a float of which only the exponent counts (a scale of exponent 255
// gives NaN, exponent 0 counts as 2^-127; all bf16 patterns at all exponents
// agree with the rounding by hand).
#pragma once

#include "dev.hpp"

namespace vsk {

typedef __bf16 mx_bf16x2 __attribute__((ext_vector_type(2)));

// The exponent byte for a block whose largest magnitude has these float bits
// (sign clear): floor(log2) - 2, biased; 255 where it is not finite.
__device__ __forceinline__ uint32_t mx4_exponent(uint32_t top) {
  const uint32_t e = top >> 23;
  return e == 255u ? 255u : e > 2u ? e - 2u : 0u;
}
__device__ __forceinline__ float mx4_scale(uint32_t e) { return __uint_as_float(e << 23); }

// Two bf16 values (a pair as it lies in memory) as the byte SEL of `old`.
template <int SEL>
__device__ __forceinline__ uint32_t mx4_encode_bf16(uint32_t old, uint32_t pair, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(old, __builtin_bit_cast(mx_bf16x2, pair), scale, SEL);
}
template <int SEL>
__device__ __forceinline__ uint32_t mx4_encode_f32(uint32_t old, float lo, float hi, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(old, lo, hi, scale, SEL);
}
// The byte SEL of `codes` as two bf16 values.
template <int SEL>
__device__ __forceinline__ uint32_t mx4_decode(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, SEL));
}
// The same as two fp16 values.
template <int SEL>
__device__ __forceinline__ uint32_t mx4_decode_half(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, SEL));
}
// Eight codes as eight bf16 values.
__device__ __forceinline__ u32x4 mx4_decode8(uint32_t codes, float scale) {
  return u32x4{mx4_decode<0>(codes, scale), mx4_decode<1>(codes, scale), mx4_decode<2>(codes, scale),
               mx4_decode<3>(codes, scale)};
}

// The larger magnitudes of two pairs of bf16 values (signs clear).
__device__ __forceinline__ uint32_t mx4_top2(uint32_t a, uint32_t b) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
// The larger of a pair's magnitudes as float bits.
__device__ __forceinline__ uint32_t mx4_top(uint32_t pair) {
  return max(pair << 16, pair & 0xffff0000u);
}

}  // namespace vsk
