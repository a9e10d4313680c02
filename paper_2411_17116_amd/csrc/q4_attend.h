// What the kernels that attend to a cache in four bits share.
#pragma once

#include "q4.h"

namespace star {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(2))) int i32x2;

#define LDS_AS __attribute__((address_space(3)))
#define INLINE __attribute__((always_inline))

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

// Eight elements of a plain row.
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    const bf16x8 v = *(const bf16x8*)p;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)v[e];
  } else {
    const f32x4 v = *(const f32x4*)p, w = *(const f32x4*)(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) { x[e] = v[e]; x[4 + e] = w[e]; }
  }
}

// Four elements of an output row in the storage type.
__device__ __forceinline__ void store4(float* p, const f32x4& x) { *(f32x4*)p = x; }
__device__ __forceinline__ void store4(__bf16* p, const f32x4& x) {
  *(bf16x4*)p = bf16x4{(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
}

// Eight codes times their unit.
__device__ __forceinline__ bf16x8 values(uint32_t c, float unit) {
  const q4_bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, unit, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, unit, 1);
  const q4_bf16x2 x = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, unit, 2), y = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, unit, 3);
  return bf16x8{a[0], a[1], b[0], b[1], x[0], x[1], y[0], y[1]};
}

// x = p[0] + p[1] + p[2] in bf16 parts, which hold 24 bits; cut off, so that none overflows.  An infinity or NaN is the first's alone.
__device__ __forceinline__ void split(float x, __bf16 (&p)[3]) {
  const bool finite = magnitude_bits(x) < 0x7f800000u;
  float r = x;
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const float y = __uint_as_float(__float_as_uint(r) & 0xffff0000u);
    p[i] = i == 0 && !finite ? (__bf16)x : (__bf16)y;
    r = finite ? r - y : 0.f;
  }
}
__device__ __forceinline__ void split(float x, __bf16 (&p)[1]) { p[0] = (__bf16)x; }

// The products of weights and values are taken in fp16: it has three bits more than bf16 where a weight is rounded once (outputs in bf16), and two parts of it
// hold 22 bits, where three of bf16 would be needed.  Weights are some powers of two large (TOP), so that small ones keep their bits as well; values have to have units
// from 2^-23 to 2^13, which fp16 holds exactly.  A workgroup that meets a unit outside them does its rows again in bf16 (WIDE), weights in one part or three; where some are
// larger, with values 2^-48 as large, so that no sum overflows.
constexpr uint32_t UNIT_LEAST = 104, UNIT_MOST = 140;
constexpr int DOWN = 48;
constexpr float TOP = 14.f;             // exponent of the largest weight
struct Wide {                           // lanes that met such units, and such that are too large
  uint64_t any, large;
  __device__ __forceinline__ void note(uint32_t e) {
    any |= __builtin_amdgcn_ballot_w64(e - UNIT_LEAST > UNIT_MOST - UNIT_LEAST);
    large |= __builtin_amdgcn_ballot_w64(e > UNIT_MOST);
  }
  __device__ __forceinline__ int flags() const { return (any != 0) | (large != 0) << 1; }
};
__device__ __forceinline__ float unit_down(uint32_t e, int down) { return q4_unit_value(e == 255u || (int)e > down ? e - (e == 255u ? 0 : down) : 0u); }
template <bool WIDE> struct Product;
template <> struct Product<false> {
  typedef f16x8 Vec;
  static __device__ __forceinline__ Vec values(uint32_t c, float unit) {
    const f16x2 a = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, unit, 0));
    const f16x2 b = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, unit, 1));
    const f16x2 x = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, unit, 2));
    const f16x2 y = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, unit, 3));
    return Vec{a[0], a[1], b[0], b[1], x[0], x[1], y[0], y[1]};
  }
  static __device__ __forceinline__ f32x4 multiply(Vec a, Vec b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
  // Weights x and y, slots e and e + 1 of the operands.
  template <int P>
  static __device__ __forceinline__ void split(float x, float y, Vec (&p)[P], int e) {
    static_assert(P <= 2, "");
    f16x2 z = {(_Float16)x, (_Float16)y};
    p[0][e] = z[0];
    p[0][e + 1] = z[1];
    if constexpr (P == 2) {
      // (a multiplier that the compiler cannot see, so that it takes the difference to a half in one instruction)
      float minus = -1.f;
      asm("" : "+s"(minus));
      uint32_t u = __builtin_bit_cast(uint32_t, z);
      asm("" : "+v"(u));
      z = __builtin_bit_cast(f16x2, u);
      p[1][e] = (_Float16)__builtin_fmaf((float)z[0], minus, x);
      p[1][e + 1] = (_Float16)__builtin_fmaf((float)z[1], minus, y);
    }
  }
};
template <> struct Product<true> {
  typedef bf16x8 Vec;
  static __device__ __forceinline__ Vec values(uint32_t c, float unit) { return star::values(c, unit); }
  static __device__ __forceinline__ f32x4 multiply(Vec a, Vec b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
  template <int P>
  static __device__ __forceinline__ void split(float x, float y, Vec (&p)[P], int e) {
    static_assert(P == 1 || P == 3, "");
    if constexpr (P == 1) {
      const bf16x2 z = {(__bf16)x, (__bf16)y};
      p[0][e] = z[0];
      p[0][e + 1] = z[1];
      return;
    }
    float a = x, b = y;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const uint32_t u = __float_as_uint(a) & 0xffff0000u, v = __float_as_uint(b) & 0xffff0000u;
      const bf16x2 z = __builtin_bit_cast(bf16x2, (u >> 16) | v);
      p[i][e] = z[0];
      p[i][e + 1] = z[1];
      a -= __uint_as_float(u);
      b -= __uint_as_float(v);
    }
  }
};

// Exponents of eight weights (as powers of two) against a reference, and the largest of them; NaN are passed over.
struct Exponents {
  float x[8];
};
__device__ __forceinline__ Exponents exponents(const f32x4 (&s)[2], float c, float neg) {
  Exponents t;
#pragma unroll
  for (int i = 0; i < 8; ++i) t.x[i] = __builtin_fmaf(s[i >> 2][i & 3], c, neg);
  return t;
}
__device__ __forceinline__ float largest(const Exponents& t) {
  return fmaxf(fmaxf(fmaxf(fmaxf(t.x[0], t.x[1]), t.x[2]), fmaxf(fmaxf(t.x[3], t.x[4]), t.x[5])), fmaxf(t.x[6], t.x[7]));
}

// Chunk c (16 bytes) of row r in LDS sits in slot c ^ swz(r).  What a wavefront reads or writes at once is chunk c + D / 32 (lane / 16) of row lane % 16 or, transposing, two
// chunks of each row; with the row's bits rotated (of 128-byte rows, two to a line, without the lowest) neither meets itself in a bank.
template <int D>
__device__ __forceinline__ int swz(int r) {
  return D == 128 ? ((r << 1) & 15) | ((r >> 3) & 1) : ((r & 6) | ((r >> 3) & 1));
}

// The four lanes l, l ^ 16, l ^ 32, l ^ 48 hold the keys of one row.
__device__ __forceinline__ float xor16(float x) { return __int_as_float(__builtin_amdgcn_ds_swizzle(__float_as_int(x), 0x401F)); }
__device__ __forceinline__ float quad_max(float x) {
  x = fmaxf(x, xor16(x));
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float quad_sum(float x) {
  x += xor16(x);
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

}  // namespace
}  // namespace star
