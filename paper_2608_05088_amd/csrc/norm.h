// Root-mean-square norm of rows, with a residual's addition before it: arguments and
// launchers (norm.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace malt {

constexpr int64_t NORM_MAX_WIDTH = 16384;
constexpr int NORM_PARTS = 1024;   // partial sums of a weight's gradient, at most

struct NormArgs {
  const void* x;         // rows x width, type T
  const void* residual;  // or null
  const void* weight;    // width
  void* sum;             // x + residual, type T; or null
  void* y;               // or null
  uint8_t* values;       // an 8-bit operand (block_fp8.h) in y's place, or null
  uint8_t* scales;
  float* rstd;           // rows, or null
  int64_t rows, ldx, ldr, lds, ldy;
  int32_t width;
  bool w_f32, y_f32;
  double eps;
};

struct NormGradArgs {
  const void* h;        // what was normed, type T
  const void* weight;
  const float* rstd;
  const void* dy;
  const void* dsum;     // gradient of h itself, type T, or null
  void* dx;             // type T, or null
  float* partial;       // [parts][width], or null
  void* dweight;
  int64_t rows, ldh, ldy, lds, ldx;
  int32_t width, parts;
  bool w_f32, dy_f32;
};

int norm_grad_parts(int64_t rows, int64_t width);
hipError_t launch_norm(const NormArgs& a, bool f32, hipStream_t s);
hipError_t launch_norm_grad(const NormGradArgs& a, bool f32, hipStream_t s);

}  // namespace malt
