// AdamW over many tensors at once: the layout of a tensor's moments, arguments and
// launchers (adamw.hip).
//
// 32 bits: float32 m[numel], then v[numel].
// 8 bits, blocks of 256 places: m's codes [blocks][256], v's codes [blocks][256],
//   m's scales float32 [blocks], v's scales float32 [blocks].
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace malt {

constexpr int ADAM_BLOCK = 256;    // places that share a scale
constexpr int ADAM_CHUNK = 4096;   // places a workgroup takes
constexpr int64_t ADAM_MAX_NUMEL = int64_t(1) << 35;

__host__ __device__ constexpr int64_t adam_blocks(int64_t n) { return (n + ADAM_BLOCK - 1) / ADAM_BLOCK; }
__host__ __device__ constexpr int64_t adam_state_bytes(int64_t n, int bits) {
  return bits == 32 ? 8 * n : adam_blocks(n) * (2 * ADAM_BLOCK + 8);
}

// Types of a tensor, above its size.
constexpr int64_t ADAM_P_F32 = int64_t(1) << 40, ADAM_G_F32 = int64_t(1) << 41, ADAM_8BIT = int64_t(1) << 42;

struct AdamTensor {
  void* param;         // moments' reader: the float32 output
  const void* grad;
  void* state;
  int64_t numel;       // and the types
};

// A launch's tensors travel in its arguments (4 KB of them at most): nothing has to be
// copied to the device first, and a captured launch keeps them.
constexpr int ADAM_TENSORS = 108;

struct AdamArgs {
  float b1, c1, b2, c2;        // beta1, 1 - beta1, ...
  float shrink;                // 1 - lr decay
  float rate;                  // lr / (1 - beta1^t)
  float root;                  // 1 / sqrt(1 - beta2^t)
  float eps;
  float grad_scale;
  uint32_t seed_lo, seed_hi;
  int32_t count;               // tensors
  int32_t first;               // the first tensor's number in the call
  const float* grad_scale_at;  // or null
  uint32_t chunk[ADAM_TENSORS];   // a tensor's first chunk in the launch
  AdamTensor t[ADAM_TENSORS];
};
static_assert(sizeof(AdamArgs) <= 4096, "kernel arguments");

hipError_t launch_adamw(const AdamArgs& a, uint32_t chunks, hipStream_t s);
hipError_t launch_adamw_moments(const AdamArgs& a, uint32_t chunks, hipStream_t s);

}  // namespace malt
