// Rows of a cache held in four bits.  A row of d elements is d / 32 groups of 32; a group is 32 codes (e2m1: a sign and one of
// 0, .5, 1, 1.5, 2, 3, 4, 6) and the exponent byte e of its unit 2^(e - 127).  The unit is the largest power of two u with 3.5 u <=
// max |x|, so that the largest element is 3.5 to 7 units and its code 4 or 6.  255 marks a group that holds a NaN or an infinity, which four bits cannot tell apart: it reads as NaN.
// Units stay within 2^-125 and 2^125, where every value a code stands for is a normal bf16 and fp32 number: values are exact in
// either type, and a group whose largest element is below 2^-126 reads as zeros (or half a unit).  A group of zeros has the unit one.
// Codes and units are what gfx950's conversions take, so a pair of elements costs one instruction either way.
#pragma once

#include "star_internal.h"

namespace star {

typedef __attribute__((ext_vector_type(2))) __bf16 q4_bf16x2;
typedef __attribute__((ext_vector_type(2))) float q4_f32x2;

// The exponent byte of a group whose largest element has the bits `most` (sign off; as integers they are in the order of the
// values, NaN above infinity above all).
__device__ __forceinline__ uint32_t q4_unit(uint32_t most) {
  if (most >= 0x7f800000u) return 255u;
  if (most == 0u) return 127u;
  const int e = (int)((most + 0x200000u) >> 23) - 2;         // (a mantissa of 1.75 and more: the next power of two)
  return (uint32_t)(e < 2 ? 2 : e > 252 ? 252 : e);
}
__device__ __forceinline__ float q4_unit_value(uint32_t e) { return __uint_as_float(e << 23); }

// Eight elements to eight codes, the first in the low bits.
__device__ __forceinline__ uint32_t q4_codes(const float (&x)[8], float unit) {
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], unit, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], unit, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], unit, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], unit, 3);
}

__device__ __forceinline__ uint32_t magnitude_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// N neighbouring elements (4 or 8) of row `row`, from column c on, filed by the lane that has them; the 32 / N lanes of a group
// are neighbours and call this together.
template <int N, int d, typename Vec>
__device__ __forceinline__ void q4_file(void* codes, void* scales, size_t row, int c, const Vec& v) {
  uint32_t most = 0;
  float x[8] = {};
#pragma unroll
  for (int e = 0; e < N; ++e) {
    x[e] = (float)v[e];
    const uint32_t b = magnitude_bits(x[e]);
    most = b > most ? b : most;
  }
#pragma unroll
  for (int s = 1; s < 32 / N; s <<= 1) {
    const uint32_t b = (uint32_t)__shfl_xor((int)most, s);
    most = b > most ? b : most;
  }
  const uint32_t e = q4_unit(most);
  const uint32_t code = e == 255 ? 0u : q4_codes(x, q4_unit_value(e));
  unsigned char* at = (unsigned char*)codes + row * (d / 2) + c / 2;
  if (N == 8) *(uint32_t*)at = code;
  else *(uint16_t*)at = (uint16_t)code;
  if (c % 32 == 0) ((unsigned char*)scales)[row * (d / 32) + c / 32] = (unsigned char)e;
}

}  // namespace star
