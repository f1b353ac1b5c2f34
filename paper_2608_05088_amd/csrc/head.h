// Cross entropy of a linear head over a large vocabulary, and its gradients, without
// the logits: arguments, layout of the workspace and launchers (head.hip,
// head_rows.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "malt_internal.h"

namespace malt {

// A matrix in the gradients' products as bf16 planes whose sum it is: one where it is bf16, three
// (high, middle, low bits: exact) where it is float32.  In the logits' products, where one of both is
// float32: float16 planes, rows scaled to 2^15, one of bf16 and two of float32 (22 bits).
constexpr int HEAD_PLANES = 3, HEAD_HALVES = 2;
constexpr int HEAD_TILE = 256;   // output tile edge, and what rows are padded to
constexpr int HEAD_BK = 64;      // contraction per stage, and what columns are padded to

// A row's softmax after the first pass, in log2: probabilities are 2^(z log2 e - top) * inverse.
struct HeadRow {
  float top;       // log2 e times the row's largest logit
  float inverse;   // 1 / sum over the vocabulary of 2^(z log2 e - top)
  float others;    // 1 - the label's probability, from the others' sum
  int32_t label;   // for the second pass, where `inverse` and `others` hold the row's weight; -1: no gradient
};

// What decides about a row.
struct HeadLabels {
  const void* labels;
  bool wide;
  int64_t stride;
  const float* weights;    // or null
  int64_t weight_stride;
};

// One side of a product: planes of bf16, rows with the contraction along them.  As they lie (a
// weight): tile = 256 ld, step = 64.  Packed: blocks of 256 rows by 64 values, what a stage reads
// of a tile, each 32 KB in a piece: [row / 256][value / 64][row % 256][value % 64].
constexpr int HEAD_BLOCK = HEAD_TILE * HEAD_BK;
struct HeadSide {
  const uint16_t* p;
  int64_t plane;   // elements from one plane to the next
  int64_t tile;    // from 256 rows to the next
  int64_t step;    // from a stage to the next
  int32_t ld;      // from a row to the next
  int64_t rows;    // rows there are: further ones are not read
};

// C = sum over pairs of planes of A B^T, over `k` values.
struct HeadProduct {
  HeadSide a, b;
  int32_t m, n;              // output rows and columns there are
  int64_t k;
  int32_t pairs;
  uint32_t pair_a, pair_b;   // a pair's planes, four bits each, the first in the lowest
  int32_t tiles_m, tiles_n;
};

struct HeadLogits {
  HeadProduct g;         // m rows, n vocabulary columns from `col0`
  HeadLabels rows;
  int64_t vocab, col0;
  // first pass
  malt_f32x2* partial;       // [m][tiles]: a tile's largest (log2) and sum without the label's column
  float* at_label;       // [m]: log2 e times the label's logit
  int32_t parts;         // tiles
  // second pass
  const HeadRow* records;   // of the padded rows
  // float32 operands: float16 planes, rows scaled by powers of two (both null: bf16)
  const float* x_scales;    // of the padded rows
  const float* w_scales;    // of the padded vocabulary, from `col0`
  uint16_t* dz;          // packed planes, rows m by n, or null
  uint16_t* dz_t;        // packed planes, rows n by m, or null
  int64_t dz_plane, dz_tile, dz_t_tile;
  int32_t dz_planes;
};

struct HeadOut {
  HeadProduct g;
  void* out;
  int64_t ldo;
  float* partial;        // float32 sums, [splits][m][n], where `out` is not written at once
  int32_t splits;        // parts of the contraction, each a workgroup's
  bool f32, add_partial, write_partial, accumulate;
  bool mask_rows;        // rows without gradient are zero (dx)
};
struct HeadGrads {
  HeadOut part[2];       // one launch: dx's tiles, then dW's
  int32_t parts;
  const HeadRow* records;
  float scale;
  const float* scale_at; // or null
};

// Few rows, weights as they lie.
constexpr int HEAD_FEW = 32;
struct HeadFew {
  const void* x;
  const void* w;
  int64_t ldx, ldw, vocab;
  int32_t m, k, parts;
  HeadLabels rows;
  malt_f32x2* partial;
  float* at_label;
};
int head_few_parts(int64_t vocab, int64_t inner);

struct HeadPack {
  const void* x;
  int64_t rows, cols, ld;
  uint16_t* out;           // packed planes, rows by cols, or cols by rows for the transpose
  int64_t plane;
  int64_t out_rows, out_cols;   // as the output lies: rows to write, padded columns (the contraction)
  int32_t planes;
  bool finite;             // infinities become the largest numbers
  HeadLabels labels;       // rows without label (or weight) become zeros; labels null: every row stays
  int64_t vocab;
};

// Everything that is packed, in one launch.
struct HeadPrepare {
  HeadPack part[4];        // x, x^T, weight, weight^T
  int32_t blocks[4];       // each part's, 0: not wanted; set by the launcher
  float* scales[2];        // of x and weight: planes of float16, each row under a power of two, and what it was divided by
  bool halves;
};
hipError_t launch_head_prepare(HeadPrepare a, bool x_f32, bool w_f32, hipStream_t s);
hipError_t launch_head_records(const HeadLabels& l, int64_t rows, int64_t rows_pad, int64_t vocab, const HeadRow* stats,
                               HeadRow* records, hipStream_t s);
hipError_t launch_head_few(const HeadFew& a, bool x_f32, bool w_f32, hipStream_t s);
// A row's parts joined: its loss, its statistics and, for the gradients, its record (of the padded rows).
struct HeadJoin {
  HeadLabels rows;
  int64_t m, rows_pad, vocab;
  const malt_f32x2* partial;
  int32_t parts;
  const float* at_label;
  HeadRow* stats;      // or null
  HeadRow* records;    // or null
  float* losses;       // or null
};
hipError_t launch_head_join(const HeadJoin& a, hipStream_t s);
hipError_t launch_head_logits(const HeadLogits& a, int edge, bool second, hipStream_t s);   // of the tiles, as below
hipError_t launch_head_grads(const HeadGrads& a, int edge, hipStream_t s);
hipError_t launch_head_sum(const HeadGrads& a, bool first, bool second, hipStream_t s);
hipError_t head_setup();

}  // namespace malt
