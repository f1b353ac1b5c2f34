// What the operators around the optimizer step (embedding, distillation loss,
// 8-bit linear layers) share: element types, loads and stores of four columns,
// sums over a wave.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "errors.h"
#include "malt_internal.h"

namespace malt {

typedef float op_f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t op_u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t op_u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(bf16_t v) { return __uint_as_float((uint32_t)v << 16); }
template <class T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ bf16_t from_f32<bf16_t>(float v) { return (bf16_t)(pack_bf16x2(v, 0.f) & 0xffffu); }

// Four consecutive elements at p (16-byte aligned floats, 8-byte aligned bf16).
__device__ __forceinline__ op_f32x4 load4(const float* p) {
  return *reinterpret_cast<const MALT_GLOBAL op_f32x4*>(gptr(p));
}
__device__ __forceinline__ op_f32x4 load4(const bf16_t* p) {
  const op_u32x2 r = *reinterpret_cast<const MALT_GLOBAL op_u32x2*>(gptr(p));
  return op_f32x4{bf16_lo(r.x), bf16_hi(r.x), bf16_lo(r.y), bf16_hi(r.y)};
}
__device__ __forceinline__ void store4(float* p, op_f32x4 v) { *reinterpret_cast<MALT_GLOBAL op_f32x4*>(gptr(p)) = v; }
__device__ __forceinline__ void store4(bf16_t* p, op_f32x4 v) {
  *reinterpret_cast<MALT_GLOBAL op_u32x2*>(gptr(p)) = op_u32x2{pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w)};
}

// The four columns of one lane in a strip of 256 columns starting at c0.  VEC:
// columns c0 + 4 lane .. + 3 (rows aligned for load4, width a multiple of 4);
// otherwise c0 + lane + 64 j, so that a wave's accesses stay contiguous.
constexpr int STRIP = 256;
template <bool VEC>
__device__ __forceinline__ int strip_col(int c0, int lane, int j) {
  return VEC ? c0 + 4 * lane + j : c0 + lane + 64 * j;
}
template <bool VEC, class T>
__device__ __forceinline__ op_f32x4 strip_load(const T* row, int c0, int lane, int width) {
  op_f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if constexpr (VEC) {
    if (c0 + 4 * lane < width) v = load4(row + c0 + 4 * lane);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (c0 + lane + 64 * j < width) v[j] = to_f32(gptr(row)[c0 + lane + 64 * j]);
  }
  return v;
}
template <bool VEC, class T>
__device__ __forceinline__ void strip_store(T* row, int c0, int lane, int width, op_f32x4 v) {
  if constexpr (VEC) {
    if (c0 + 4 * lane < width) store4(row + c0 + 4 * lane, v);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (c0 + lane + 64 * j < width) gptr(row)[c0 + lane + 64 * j] = from_f32<T>(v[j]);
  }
}

__device__ __forceinline__ int64_t load_id(const void* ids, bool wide, int64_t t) {
  return wide ? gptr(static_cast<const int64_t*>(ids))[t] : (int64_t)gptr(static_cast<const int32_t*>(ids))[t];
}

// --------------------------------------------------------------- host checks
inline bool op_dtype_ok(int t) { return t == MALT_FLOAT32 || t == MALT_BFLOAT16; }
inline size_t op_dtype_bytes(int t) { return t == MALT_FLOAT32 ? 4 : 2; }
inline bool op_aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
// Rows of `ld` elements at p can be read four columns at a time.
inline bool op_rows_by_four(const void* p, int type, int64_t ld, int64_t width) {
  return width % 4 == 0 && ld % 4 == 0 && op_aligned(p, 4 * op_dtype_bytes(type));
}
inline bool op_overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return na && nb && x < y + nb && y < x + na;
}

}  // namespace malt
