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

// Four consecutive elements at p, aligned to one element only: gfx950 takes wide
// loads and stores at any address, and aligned ones cost the same instruction.
typedef op_f32x4 op_f32x4_any __attribute__((aligned(4)));
typedef op_u32x2 op_u32x2_any __attribute__((aligned(2)));
typedef op_u32x4 op_u32x4_any __attribute__((aligned(2)));
__device__ __forceinline__ op_f32x4 load4(const float* p) {
  return *reinterpret_cast<const MALT_GLOBAL op_f32x4_any*>(gptr(p));
}
__device__ __forceinline__ op_f32x4 load4(const bf16_t* p) {
  const op_u32x2 r = *reinterpret_cast<const MALT_GLOBAL op_u32x2_any*>(gptr(p));
  return op_f32x4{bf16_lo(r.x), bf16_hi(r.x), bf16_lo(r.y), bf16_hi(r.y)};
}
__device__ __forceinline__ void store4(float* p, op_f32x4 v) { *reinterpret_cast<MALT_GLOBAL op_f32x4_any*>(gptr(p)) = v; }
__device__ __forceinline__ void store4(bf16_t* p, op_f32x4 v) {
  *reinterpret_cast<MALT_GLOBAL op_u32x2_any*>(gptr(p)) = op_u32x2{pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w)};
}

// Columns c .. c + 3 of a row of `width`; what lies past its end is zero and is not stored.
template <class T>
__device__ __forceinline__ op_f32x4 row_load4(const T* row, int64_t c, int64_t width) {
  if (c + 4 <= width) return load4(row + c);
  op_f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < 3; ++j)
    if (c + j < width) v[j] = to_f32(gptr(row)[c + j]);
  return v;
}
template <class T>
__device__ __forceinline__ void row_store4(T* row, int64_t c, int64_t width, op_f32x4 v) {
  if (c + 4 <= width) {
    store4(row + c, v);
    return;
  }
#pragma unroll
  for (int j = 0; j < 3; ++j)
    if (c + j < width) gptr(row)[c + j] = from_f32<T>(v[j]);
}

__device__ __forceinline__ int64_t load_id(const void* ids, bool wide, int64_t t) {
  return wide ? gptr(static_cast<const int64_t*>(ids))[t] : (int64_t)gptr(static_cast<const int32_t*>(ids))[t];
}

// --------------------------------------------------------------- host checks
inline bool op_dtype_ok(int t) { return t == MALT_FLOAT32 || t == MALT_BFLOAT16; }
inline size_t op_dtype_bytes(int t) { return t == MALT_FLOAT32 ? 4 : 2; }
inline bool op_aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
inline bool op_overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return na && nb && x < y + nb && y < x + na;
}

}  // namespace malt
