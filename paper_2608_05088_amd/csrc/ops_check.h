// What the C entries of the operators check on the host, before anything is enqueued.
#pragma once

#include "ops_common.h"

namespace malt {

constexpr int64_t kMaxPitch = (int64_t(1) << 31) - 1;
constexpr int64_t kMaxMatrix = int64_t(1) << 35;   // elements of a table, or of one matrix of a layer

// A strided matrix as the checks see it.
struct Mat {
  const char* name;
  const void* p;
  int type;               // malt_dtype_t
  int64_t rows, cols, ld;
  size_t elem() const { return op_dtype_bytes(type); }
  size_t bytes() const { return rows > 0 && cols > 0 ? (size_t(rows - 1) * ld + cols) * elem() : 0; }
};

inline malt_status_t check_mat(const Mat& m) {
  if (!op_dtype_ok(m.type)) return fail(MALT_ERR_INVALID_ARG, "%s: unknown element type %d", m.name, m.type);
  if (m.rows > 0 && m.cols > 0 && !m.p) return fail(MALT_ERR_INVALID_ARG, "%s is NULL", m.name);
  if (m.ld < m.cols || m.ld > kMaxPitch)
    return fail(MALT_ERR_SHAPE, "%s: row pitch %lld of %lld columns", m.name, (long long)m.ld, (long long)m.cols);
  if (!op_aligned(m.p, m.elem())) return fail(MALT_ERR_ALIGNMENT, "%s is not aligned to its elements", m.name);
  return MALT_OK;
}

inline malt_status_t check_ids(const char* name, const void* p, int type, int64_t n) {
  if (type != MALT_INT32 && type != MALT_INT64) return fail(MALT_ERR_INVALID_ARG, "%s: unknown index type %d", name, type);
  if (n > 0 && !p) return fail(MALT_ERR_INVALID_ARG, "%s is NULL", name);
  if (!op_aligned(p, type == MALT_INT64 ? 8 : 4)) return fail(MALT_ERR_ALIGNMENT, "%s is not aligned to its elements", name);
  return MALT_OK;
}

inline malt_status_t launched(hipError_t e, const char* what) { return e == hipSuccess ? MALT_OK : hip_fail(e, what); }

inline malt_status_t check_workspace(const void* p, size_t bytes, size_t need) {
  if (need > 0 && !p) return fail(MALT_ERR_INVALID_ARG, "workspace is NULL");
  if (!op_aligned(p, 256)) return fail(MALT_ERR_ALIGNMENT, "workspace must be 256-byte aligned");
  if (bytes < need) return fail(MALT_ERR_INVALID_ARG, "a workspace of %zu bytes where %zu are needed", bytes, need);
  return MALT_OK;
}

inline size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

#define MALT_TRY(expr)                          \
  do {                                          \
    const malt_status_t st_ = (expr);           \
    if (st_ != MALT_OK) return st_;             \
  } while (0)

}  // namespace malt
