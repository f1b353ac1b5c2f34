// 8-bit operands with a power-of-two scale for each block of 128 values: layout,
// arguments and launchers (block_quant.hip, block_matmul.hip, block_linear.hip).
//
// An operand of `rows` rows over a contraction of `cols` values is
//   values  [rows][pad128(cols)] bytes (4 exponent, 3 mantissa bits), zeros past cols;
//   scales  one exponent byte e + 127 for each row and 128 values, by blocks of the
//           contraction: [cols / 128][pad256(rows)], where within 128 rows row r lies
//           at 8 (r % 16) + (r / 16) % 8: the bytes a lane of a 16-row matrix
//           instruction needs for eight row groups are neighbours.
// A weight has a scale for each 128 x 128 block instead, [row block][column block].
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace malt {

constexpr int QB = 128;   // block edge

__host__ __device__ constexpr int64_t q_pad(int64_t n) { return (n + QB - 1) / QB * QB; }
__host__ __device__ constexpr int64_t q_scale_rows(int64_t rows) { return (rows + 255) / 256 * 256; }
__host__ __device__ constexpr int q_scale_pos(int r) { return 8 * (r & 15) + ((r >> 4) & 7); }   // within 128 rows

struct QuantArgs {
  const void* x;
  int64_t rows, cols, ld;
  uint8_t* values;        // rows x pad128(cols), or null
  uint8_t* scales;        // for `values`, one scale a row; null for a weight
  uint8_t* t_values;      // cols x pad128(rows): the transpose, blocks along the rows; or null
  uint8_t* t_scales;
  uint8_t* block_scales;  // weight: one scale a 128 x 128 block, both for values and t_values
};

struct BlockMatmulArgs {
  int64_t m, n, k;
  const uint8_t* a;
  const uint8_t* a_scales;
  const uint8_t* b;
  const uint8_t* b_scales;
  int64_t b_row_stride, b_col_stride;   // weight scales: between blocks of rows, of the contraction
  void* out;
  int64_t ldo;
  bool accumulate;
  float* partial;   // parts > 1: [part][tile][rows][columns]
  int32_t parts;    // set by the launcher: parts the contraction is cut into
};

// A linear layer on kept weights, x (m x k) W^T, for m <= BLOCK_FEW rows.  us this way and by
// conversion and tiles: 1 row, 4096 -> 4096 10 and 17, 32 rows 15 and 18; 4096 -> 16384 18 and
// 24, 25 and 26 (17 rows), 29 and 26 (32 rows).
constexpr int BLOCK_FEW = 32;
struct BlockLinearArgs {
  const void* x;
  int64_t m, n, k, ldx;
  const uint8_t* w;         // n x pad128(k)
  const uint8_t* w_scales;  // [n / 128][k / 128]
  void* out;
  int64_t ldo;
};
hipError_t launch_block_linear(const BlockLinearArgs& g, bool x_f32, bool out_f32, hipStream_t s);

// How a product is tiled, by its sizes and the type of its result.
struct BlockMatmulPlan {
  bool big;       // 256 x 256 tiles; otherwise 128 x 128
  int32_t parts;  // of the contraction
  size_t bytes;   // of the partial sums
};
BlockMatmulPlan block_matmul_plan(int64_t m, int64_t n, int64_t k, bool out_f32);

hipError_t launch_block_quant(const QuantArgs& a, bool f32, hipStream_t s);
hipError_t launch_block_quant_pair(const QuantArgs& x, bool x_f32, const QuantArgs& w, bool w_f32, hipStream_t s);
hipError_t launch_block_matmul(BlockMatmulArgs a, bool b_blocks, bool out_f32, hipStream_t s);

}  // namespace malt
