// Arguments and launcher of the distillation loss (distill.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace malt {

constexpr int DISTILL_MAX_TOP = 1024;   // teacher's entries a row may have

struct DistillArgs {
  const void* logits;
  const void* top;         // null: no teacher
  const void* top_ids;
  const void* labels;      // null: no labels
  const float* weight;     // null: weight_value for every row
  float* losses;           // null: not wanted
  void* dlogits;           // null: not wanted
  int64_t rows, vocab, ld, top_ld, id_ld, weight_stride, label_stride, dld;
  int32_t n_top;
  bool top_f32, wide_ids, wide_labels;
  float tau, alpha, weight_value;
};

hipError_t launch_distill(const DistillArgs& a, bool f32, hipStream_t s);

}  // namespace malt
