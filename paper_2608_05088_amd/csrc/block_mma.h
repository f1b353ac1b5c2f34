// Device side of the 8-bit operands: conversion with a power-of-two scale, and the
// two ways the matrix cores take them (block_matmul.hip).
#pragma once

#include "block_fp8.h"
#include "ns_common.h"
#include "ops_common.h"

namespace malt {

typedef int i32x8 __attribute__((ext_vector_type(8)));

// --------------------------------------------------------------- conversion
// Largest magnitude as a bit pattern: an infinity or a NaN is larger than any number.
__device__ __forceinline__ uint32_t mag(float v) { return __float_as_uint(v) & 0x7fffffffu; }
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }

// Exponent byte of the scale for a largest magnitude: 448 = 1.75 * 2^8; 255 (not
// a number) where the block holds an infinity or a NaN.
__device__ __forceinline__ uint32_t scale_byte(uint32_t b) {
  if (b >= 0x7f800000u) return 255u;
  if (b == 0) return 127u;
  const int e = (int)(b >> 23) - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
  return e < 0 ? 0u : (uint32_t)e;
}
// 1 / s, exact; NaN for a block that holds an infinity or a NaN.
__device__ __forceinline__ float scale_inverse(uint32_t byte) {
  return __uint_as_float(byte < 254u ? (254u - byte) << 23 : 0x7fc00000u);
}
__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
  return (uint32_t)r;
}

// Columns c .. c + 7 of a row, zero past its end.
__device__ __forceinline__ void load8(const float* row, int c, int cols, float (&v)[8]) {
  const op_f32x4 a = row_load4(row, c, cols), b = row_load4(row, c + 4, cols);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[j] = a[j];
    v[4 + j] = b[j];
  }
}
__device__ __forceinline__ void load8(const bf16_t* row, int c, int cols, float (&v)[8]) {
  if (c + 8 <= cols) {
    const op_u32x4 r = *reinterpret_cast<const MALT_GLOBAL op_u32x4_any*>(gptr(row) + c);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[2 * j] = bf16_lo(r[j]);
      v[2 * j + 1] = bf16_hi(r[j]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = c + j < cols ? to_f32(gptr(row)[c + j]) : 0.f;
  }
}

// ------------------------------------------------------------------- product
// c += (2^sb B) (2^sa A)^T of one block; byte OB / OA of the scale registers counts.
template <int OB, int OA>
__device__ __forceinline__ ns::f32x4 mma(i32x8 b, i32x8 a, ns::f32x4 c, int sb, int sa) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, c, 0, 0, OB, sb, OA, sa);
}
__device__ __forceinline__ ns::f32x4 mma_sel(i32x8 b, i32x8 a, ns::f32x4 c, int sb, int ob, int sa, int oa) {
  // ob, oa are constants after unrolling
  switch (ob * 4 + oa) {
#define MALT_SEL(x, y) case x * 4 + y: return mma<x, y>(b, a, c, sb, sa);
    MALT_SEL(0, 0) MALT_SEL(0, 1) MALT_SEL(0, 2) MALT_SEL(0, 3)
    MALT_SEL(1, 0) MALT_SEL(1, 1) MALT_SEL(1, 2) MALT_SEL(1, 3)
    MALT_SEL(2, 0) MALT_SEL(2, 1) MALT_SEL(2, 2) MALT_SEL(2, 3)
    MALT_SEL(3, 0) MALT_SEL(3, 1) MALT_SEL(3, 2) default: return mma<3, 3>(b, a, c, sb, sa);
#undef MALT_SEL
  }
}

// Eight 8-bit values (two dwords) times 2^e as bf16, exactly where they are multiples
// of 2^-133, bf16's smallest number; `scale` is 2^e, of which the exponent byte counts.
__device__ __forceinline__ ns::bf16x8 widen(int lo, int hi, float scale) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)lo, scale, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)lo, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)hi, scale, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)hi, scale, true);
  return ns::bf16x8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}
// The power of two of exponent byte i of a scale register, for `widen`: byte 0, a float32
// zero, is taken as 2^-127 there, and byte 255 as no number.
__device__ __forceinline__ float scale_of(int bytes, int i) {
  return __uint_as_float((((uint32_t)bytes >> (8 * i)) & 0xffu) << 23);
}


}  // namespace malt
