// Cross entropy of a linear head: everything but its tiled products (head.hip).
//
//   z = x W^T, loss = log sum_v exp z_v - z_y
//
// Statistics are kept without the label's column: with o = sum over v != y of exp z_v, 1 - q_y =
// o / (o + exp z_y) has all its bits where the model is sure of the label and 1 - q_y by
// subtraction would have none, and so has loss = log(1 + o / exp z_y).
#include "head.h"
#include "ns_common.h"
#include "ops_common.h"

namespace malt {

namespace {

using ns::bf16x8;
using ns::f32x4;

constexpr float FAR = 0x1p100f;   // a logit (log2) that counts as infinite
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

// A row's label, or -1: outside the vocabulary.
__device__ __forceinline__ int64_t label_of(const HeadLabels& l, int64_t r, int64_t vocab) {
  const int64_t y = load_id(l.labels, l.wide, r * l.stride);
  return (uint64_t)y < (uint64_t)vocab ? y : -1;
}

// ---------------------------------------------------------------------- packing
// Rows that stay: those with a label and a weight, or all.
__device__ __forceinline__ bool stays(const HeadLabels& l, int64_t r, int64_t vocab) {
  return !l.labels || (label_of(l, r, vocab) >= 0 && (!l.weights || gptr(l.weights)[r * l.weight_stride] != 0.f));
}

// Four values as planes.  What a plane leaves is exact: its bits are those of v past the plane's.
// finite: the largest values, infinities among them, stay so, since an infinity times another value's empty
// plane would be no number.  Logits past FAR count as infinite.
constexpr float BF16_MAX = 0x1.fep127f;
__device__ __forceinline__ void store_planes(uint16_t* out, int64_t plane, int planes, bool finite, op_f32x4 v) {
  if (finite)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (fabsf(v[j]) == __builtin_inff()) v[j] = copysignf(BF16_MAX, v[j]);
  for (int p = 0; p < planes; ++p) {
    uint32_t lo = pack_bf16x2(v.x, v.y), hi = pack_bf16x2(v.z, v.w);
    if (finite) {
      // Rounded past bf16's largest.
      if ((lo & 0x7fffu) == 0x7f80u) lo -= 1;
      if ((lo & 0x7fff0000u) == 0x7f800000u) lo -= 0x10000u;
      if ((hi & 0x7fffu) == 0x7f80u) hi -= 1;
      if ((hi & 0x7fff0000u) == 0x7f800000u) hi -= 0x10000u;
    }
    *reinterpret_cast<MALT_GLOBAL op_u32x2*>(gptr(out) + p * plane) = op_u32x2{lo, hi};
    const float h[4] = {bf16_lo(lo), bf16_hi(lo), bf16_lo(hi), bf16_hi(hi)};
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] -= h[j];
  }
}
// Where value c of row r lies in a plane whose rows hold `cols`.
__device__ __forceinline__ int64_t packed_at(int64_t r, int64_t c, int64_t cols) {
  return (r / HEAD_TILE * (cols / HEAD_BK) + c / HEAD_BK) * HEAD_BLOCK + r % HEAD_TILE * HEAD_BK + c % HEAD_BK;
}

// Four columns a thread.
template <class T>
__device__ __forceinline__ void pack_rows(const HeadPack& a, int block) {
  const int64_t per = a.out_cols / 4, i = (int64_t)block * 256 + threadIdx.x;
  if (i >= a.out_rows * per) return;
  const int64_t r = i / per, c = i % per * 4;
  op_f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (r < a.rows && stays(a.labels, r, a.vocab)) v = row_load4(static_cast<const T*>(a.x) + r * a.ld, c, a.cols);
  store_planes(a.out + packed_at(r, c, a.out_cols), a.plane, a.planes, a.finite, v);
}

// A wave a row: its largest magnitude, then its values times the power of two that brings it to
// [2^14, 2^15), as float16 numbers: 11 bits, and 11 of what they leave, to 2^-39 of the largest.  A row with an
// infinity keeps its infinities alone, as 1 under a scale past every logit.
template <class T>
__device__ __forceinline__ void pack_halves(const HeadPack& a, float* scales, int block) {
  const int64_t r = (int64_t)block * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (r >= a.out_rows) return;
  const bool there = r < a.rows && stays(a.labels, r, a.vocab);
  const T* const row = static_cast<const T*>(a.x) + (there ? r : 0) * a.ld;
  uint32_t top = 0;
  if (there)
    for (int64_t c = 4 * lane; c < a.cols; c += 256) {
      const op_f32x4 v = row_load4(row, c, a.cols);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t b = __float_as_uint(v[j]) & 0x7fffffffu;
        top = top > b ? top : b;
      }
    }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t o = (uint32_t)__shfl_xor((int)top, d, 64);
    top = top > o ? top : o;
  }
  const bool far = top >= 0x7f800000u;
  int e = (int)(top >> 23) - 127 - 14;   // the scale's exponent
  e = top == 0 ? 0 : e < -126 ? -126 : e;
  const float scale = far ? 0x1p120f : __uint_as_float((uint32_t)(e + 127) << 23), inverse = __uint_as_float((uint32_t)(127 - e) << 23);
  if (lane == 0) gptr(scales)[r] = scale;
  for (int64_t c = 4 * lane; c < a.out_cols; c += 256) {
    op_f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (there) v = row_load4(row, c, a.cols);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (!far) v[j] *= inverse;
      else if (v[j] == v[j]) v[j] = fabsf(v[j]) == __builtin_inff() ? copysignf(1.f, v[j]) : 0.f;
    }
    uint16_t* out = a.out + packed_at(r, c, a.out_cols);
    for (int p = 0; p < a.planes; ++p) {
      _Float16 h[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        h[j] = (_Float16)v[j];
        v[j] -= (float)h[j];
      }
      typedef _Float16 half4 __attribute__((ext_vector_type(4)));
      *reinterpret_cast<MALT_GLOBAL op_u32x2*>(gptr(out) + p * a.plane) = __builtin_bit_cast(op_u32x2, half4{h[0], h[1], h[2], h[3]});
    }
  }
}

// The transpose of a 64 x 64 tile through LDS; rows past the end are zeros.
// Everything that a step of 8192 x 50257 x 1280 in bf16 packs (320 MB in and out): 77 us, 4.2 TB/s.
template <class T>
__device__ __forceinline__ void pack_turned(const HeadPack& a, float (&tile)[64][65], int block) {
  const int tiles_r = (int)(a.out_cols / 64);
  const int64_t r0 = (int64_t)(block % tiles_r) * 64, c0 = (int64_t)(block / tiles_r) * 64;
  const int lo = threadIdx.x & 15, hi = threadIdx.x >> 4;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int64_t r = r0 + hi + 16 * k;
    op_f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (r < a.rows && stays(a.labels, r, a.vocab)) v = row_load4(static_cast<const T*>(a.x) + r * a.ld, c0 + 4 * lo, a.cols);
#pragma unroll
    for (int j = 0; j < 4; ++j) tile[hi + 16 * k][4 * lo + j] = v[j];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int c = hi + 16 * k;
    if (c0 + c >= a.out_rows) continue;
    const op_f32x4 v = {tile[4 * lo][c], tile[4 * lo + 1][c], tile[4 * lo + 2][c], tile[4 * lo + 3][c]};
    store_planes(a.out + packed_at(c0 + c, r0 + 4 * lo, a.out_cols), a.plane, a.planes, a.finite, v);
  }
}

template <class X, class W>
__global__ __launch_bounds__(256) void head_prepare_kernel(HeadPrepare a) {
  __shared__ float tile[64][65];
  int block = blockIdx.x, part = 0;
  while (block >= a.blocks[part]) block -= a.blocks[part++];   // the grid is their sum
  if (part == 0) {
    if (a.halves) pack_halves<X>(a.part[0], a.scales[0], block);
    else pack_rows<X>(a.part[0], block);
  } else if (part == 1) {
    pack_turned<X>(a.part[1], tile, block);
  } else if (part == 2) {
    if (a.halves) pack_halves<W>(a.part[2], a.scales[1], block);
    else pack_rows<W>(a.part[2], block);
  } else {
    pack_turned<W>(a.part[3], tile, block);
  }
}

// What the second pass asks about a row.
__device__ __forceinline__ void write_record(const HeadLabels& l, int64_t r, bool there, int64_t y, f32x4 v, HeadRow* records) {
  if (there && l.weights) {
    const float w = gptr(l.weights)[r * l.weight_stride];
    v.y *= w;
    v.z *= w;
    if (w == 0.f) y = -1;
  }
  v.w = __int_as_float(there ? (int)y : -1);
  *reinterpret_cast<MALT_GLOBAL f32x4*>(gptr(reinterpret_cast<float*>(records + r))) = v;
}
__global__ __launch_bounds__(256) void head_records_kernel(HeadLabels l, int64_t rows, int64_t rows_pad, int64_t vocab,
                                                           const HeadRow* stats, HeadRow* records) {
  const int64_t r = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (r >= rows_pad) return;
  const bool there = r < rows;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (there) v = *reinterpret_cast<const MALT_GLOBAL f32x4*>(gptr(reinterpret_cast<const float*>(stats + r)));
  write_record(l, r, there, there ? label_of(l, r, vocab) : -1, v, records);
}

// --------------------------------------------------------------------- few rows
// Up to 32 rows of x: bound by reading the weights, once, as they lie.  A wave takes 16 rows of
// the weight at a time over the whole contraction: a lane holds 32 values (bf16) or 16 of one
// of them, neighbours, so that its loads are wide; the products' order of k is the same for both sides.
// One row of 50257 x 1280 in bf16: 24 us, 5.4 TB/s, and 4 for the join.
template <class T>
struct Few;
template <>
struct Few<bf16_t> {
  static constexpr int PER = 32, K = 4 * PER;   // values a lane holds, contraction of a step
  bf16x8 v[4];
  __device__ __forceinline__ void load(const bf16_t* row, int k, int cols) {
    if (k + PER <= cols) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        v[i] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const MALT_GLOBAL op_u32x4_any*>(gptr(row) + k + 8 * i));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        op_u32x4 q;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int c = k + 8 * i + 2 * j;
          const uint32_t lo = c < cols ? gptr(row)[c] : 0, hi = c + 1 < cols ? gptr(row)[c + 1] : 0;
          q[j] = lo | hi << 16;
        }
        v[i] = __builtin_bit_cast(bf16x8, q);
      }
    }
  }
  __device__ static __forceinline__ f32x4 mma(const Few& w, const Few& x, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.v[i], x.v[i], c, 0, 0, 0);
    return c;
  }
};
// float32, or bf16 widened to it beside a float32 weight.
template <>
struct Few<float> {
  static constexpr int PER = 16, K = 4 * PER;
  op_f32x4 v[4];
  template <class S>
  __device__ __forceinline__ void load(const S* row, int k, int cols) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = row_load4(row, k + 4 * i, cols);
  }
  __device__ static __forceinline__ f32x4 mma(const Few& w, const Few& x, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(w.v[i][j], x.v[i][j], c, 0, 0, 0);
    return c;
  }
};

constexpr int FEW_WAVES = 4;
// SPLIT: a workgroup's waves share 16 rows of the weight and cut the contraction; else they take 16 each.
// us a call, split | whole, one row of bf16: 3000 x 4096 15 | 31 (the host), 12000 x 4096 25 | 40, 50257 x 1280
// 32 | 34, 50257 x 4096 79 | 101, 50257 x 768 24 | 24; 32 rows of float32: 3000 x 4096 37 | 121, 18000 x 768 32 | 40.
// Whole where there are many rows or short ones: 131072 x 2048 120 | 104, 32 rows of 50257 x 128 21 | 15.
bool few_split(int64_t vocab, int64_t inner) { return vocab <= 65536 && inner >= (vocab <= 20480 ? 512 : 1024); }

template <class C, class X, class W, int MB, bool SPLIT>
__global__ __launch_bounds__(64 * FEW_WAVES) void head_few_kernel(HeadFew a) {
  constexpr int COLS = SPLIT ? 16 : 16 * FEW_WAVES, JOIN = SPLIT ? 1 : FEW_WAVES, CUT = SPLIT ? FEW_WAVES : 1;
  __shared__ malt_f32x2 join[JOIN][MB * 16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * COLS + (SPLIT ? 0 : 16 * wave);
  const int64_t n = n0 + r < a.vocab ? n0 + r : a.vocab - 1;   // past the end: not counted below
  const W* const w = static_cast<const W*>(a.w) + n * a.ldw;
  const X* x[MB];
#pragma unroll
  for (int b = 0; b < MB; ++b) {
    const int m = 16 * b + r;
    x[b] = static_cast<const X*>(a.x) + (m < a.m ? m : a.m - 1) * a.ldx;
  }
  f32x4 acc[MB];
#pragma unroll
  for (int b = 0; b < MB; ++b) acc[b] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int k0 = SPLIT ? wave * C::K : 0; k0 < a.k; k0 += CUT * C::K) {
    const int k = k0 + C::PER * g;
    C fw, fx;
    fw.load(w, k, a.k);
#pragma unroll
    for (int b = 0; b < MB; ++b) {
      fx.load(x[b], k, a.k);
      acc[b] = C::mma(fw, fx, acc[b]);
    }
  }
  if constexpr (SPLIT) {
    __shared__ f32x4 parts[FEW_WAVES][MB][64];
#pragma unroll
    for (int b = 0; b < MB; ++b) parts[wave][b][lane] = acc[b];
    __syncthreads();
#pragma unroll
    for (int b = 0; b < MB; ++b) acc[b] = (parts[0][b][lane] + parts[1][b][lane]) + (parts[2][b][lane] + parts[3][b][lane]);
  }
  const int slot = SPLIT ? 0 : wave;   // of SPLIT all waves hold the same sums, the first writes
  // acc[b][e]: row 16 b + lane % 16, column n0 + 4 (lane / 16) + e.
#pragma unroll
  for (int b = 0; b < MB; ++b) {
    const int m = 16 * b + r;
    const int64_t y = m < a.m ? label_of(a.rows, m, a.vocab) : -1, c = n0 + 4 * g;
    float top = -__builtin_inff(), sum = 0.f, z[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      z[e] = acc[b][e] * LOG2E;
      if (c + e == y && (!SPLIT || wave == 0)) gptr(a.at_label)[m] = z[e];
      if (c + e == y || c + e >= a.vocab) z[e] = -__builtin_inff();
      top = fmaxf(top, z[e]);
    }
    top = fmaxf(top, __shfl_xor(top, 16, 64));
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    const float ref = top == -__builtin_inff() ? 0.f : top;
#pragma unroll
    for (int e = 0; e < 4; ++e) sum += exp2f(z[e] - ref);
    sum += __shfl_xor(sum, 16, 64);
    sum += __shfl_xor(sum, 32, 64);
    if (g == 0 && (!SPLIT || wave == 0)) join[slot][m] = malt_f32x2{top, sum};
  }
  __syncthreads();
  if (threadIdx.x < a.m) {
    float top = -__builtin_inff(), sum = 0.f;
#pragma unroll
    for (int i = 0; i < JOIN; ++i) top = fmaxf(top, join[i][threadIdx.x].x);
    const float ref = top == -__builtin_inff() ? 0.f : top;
#pragma unroll
    for (int i = 0; i < JOIN; ++i) sum += join[i][threadIdx.x].y * exp2f(join[i][threadIdx.x].x - ref);
    gptr(a.partial)[(int64_t)threadIdx.x * a.parts + blockIdx.x] = malt_f32x2{top, sum};
  }
}

// ------------------------------------------------------------------------- join
// A row's parts, one workgroup of T threads a row.
template <int T>
__global__ __launch_bounds__(T) void head_join_kernel(HeadJoin a) {
  __shared__ float red[2][T / 64];
  const int64_t r = blockIdx.x;
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  if (r >= a.m) {
    if (threadIdx.x == 0) write_record(a.rows, r, false, -1, zero, a.records);
    return;
  }
  const int parts = a.parts;
  const malt_f32x2* const p = a.partial + r * parts;
  float top = -__builtin_inff(), sum = 0.f;
#pragma unroll 4
  for (int i = threadIdx.x; i < parts; i += T) {
    const malt_f32x2 v = gptr(p)[i];
    const float t = fmaxf(top, v.x), ref = t == -__builtin_inff() ? 0.f : t;
    sum = sum * exp2f(top - ref) + v.y * exp2f(v.x - ref);
    top = t;
  }
  float all = top;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) all = fmaxf(all, __shfl_xor(all, d, 64));
  if constexpr (T > 64) {
    if ((threadIdx.x & 63) == 0) red[0][threadIdx.x >> 6] = all;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < T / 64; ++i) all = fmaxf(all, red[0][i]);
  }
  if (all <= -FAR) all = -__builtin_inff();
  const float ref = all == -__builtin_inff() ? 0.f : all;
  sum = all == -__builtin_inff() && sum == sum ? 0.f : sum * exp2f(top - ref);
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d, 64);
  if constexpr (T > 64) {
    if ((threadIdx.x & 63) == 0) red[1][threadIdx.x >> 6] = sum;
    __syncthreads();
    sum = red[1][0];
#pragma unroll
    for (int i = 1; i < T / 64; ++i) sum += red[1][i];
  }
  if (threadIdx.x != 0) return;
  const int64_t label = label_of(a.rows, r, a.vocab);
  if (label < 0) {
    if (a.losses) gptr(a.losses)[r] = 0.f;
    if (a.stats) *reinterpret_cast<MALT_GLOBAL f32x4*>(gptr(reinterpret_cast<float*>(a.stats + r))) = zero;
    if (a.records) write_record(a.rows, r, true, -1, zero, a.records);
    return;
  }
  float y = gptr(a.at_label)[r];   // log2
  if (y <= -FAR) y = -__builtin_inff();
  if (y >= FAR || all >= FAR) sum = __builtin_nanf("");
  if (a.losses) {
    // log(1 + o / e^y) where the label leads, log(o) - y + log(1 + e^y / o) where it does not; log1p keeps
    // what a sum of nearly 1 would lose.
    const float d = y - ref;   // log2 of e^y over the others' largest
    float loss;
    if (d > log2f(sum)) loss = log1pf(sum * exp2f(-d));
    else loss = (log2f(sum) - d) * LN2 + log1pf(exp2f(d) / sum);
    if (sum == 0.f && y > -__builtin_inff()) loss = 0.f;   // no other column has mass
    if (sum != sum) loss = sum;
    gptr(a.losses)[r] = loss;
  }
  if (a.stats || a.records) {
    // The reference is the larger of both: no power of two above 1 is formed.  Where no other column has mass it is the
    // label's logit itself, however small: 2^(y - 0) would underflow below -149, and the total with it.
    const bool alone = all == -__builtin_inff();
    const float t = alone ? y : fmaxf(all, y), o = alone ? sum : sum * exp2f(all - t), total = o + exp2f(y - t);
    const f32x4 v = {t, 1.f / total, o / total, 0.f};
    if (a.stats) *reinterpret_cast<MALT_GLOBAL f32x4*>(gptr(reinterpret_cast<float*>(a.stats + r))) = v;
    if (a.records) write_record(a.rows, r, true, label, v, a.records);
  }
}

template <class C, class X, class W, bool SPLIT>
void few_of(const HeadFew& a, hipStream_t s) {
  const dim3 grid((unsigned)a.parts), block(64 * FEW_WAVES);
  if (a.m <= 16) hipLaunchKernelGGL((head_few_kernel<C, X, W, 1, SPLIT>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((head_few_kernel<C, X, W, 2, SPLIT>), grid, block, 0, s, a);
}
template <class C, class X, class W>
void few(const HeadFew& a, hipStream_t s) {
  if (few_split(a.vocab, a.k)) few_of<C, X, W, true>(a, s);
  else few_of<C, X, W, false>(a, s);
}

}  // namespace

int head_few_parts(int64_t vocab, int64_t inner) {
  const int cols = few_split(vocab, inner) ? 16 : 16 * FEW_WAVES;
  return (int)((vocab + cols - 1) / cols);
}

hipError_t launch_head_few(const HeadFew& a, bool x_f32, bool w_f32, hipStream_t s) {
  if (x_f32 && w_f32) few<Few<float>, float, float>(a, s);
  else if (x_f32) few<Few<float>, float, bf16_t>(a, s);
  else if (w_f32) few<Few<float>, bf16_t, float>(a, s);
  else few<Few<bf16_t>, bf16_t, bf16_t>(a, s);
  return hipGetLastError();
}

hipError_t launch_head_join(const HeadJoin& a, hipStream_t s) {
  // A wave a row where there are enough rows to fill the card.
  const dim3 grid((unsigned)(a.records ? a.rows_pad : a.m));
  if (a.m <= HEAD_FEW) hipLaunchKernelGGL((head_join_kernel<1024>), grid, dim3(1024), 0, s, a);
  else hipLaunchKernelGGL((head_join_kernel<64>), grid, dim3(64), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_head_prepare(HeadPrepare a, bool x_f32, bool w_f32, hipStream_t s) {
  int64_t all = 0;
  for (int i = 0; i < 4; ++i) {
    const HeadPack& p = a.part[i];
    int64_t n = 0;
    if (p.out && i % 2) n = p.out_cols / 64 * ((p.out_rows + 63) / 64);
    else if (p.out && a.halves) n = (p.out_rows + 3) / 4;
    else if (p.out) n = (p.out_rows * (p.out_cols / 4) + 255) / 256;
    a.blocks[i] = (int32_t)n;
    all += n;
  }
  if (all == 0) return hipSuccess;
  const dim3 grid((unsigned)all);
  if (x_f32 && w_f32) hipLaunchKernelGGL((head_prepare_kernel<float, float>), grid, dim3(256), 0, s, a);
  else if (x_f32) hipLaunchKernelGGL((head_prepare_kernel<float, bf16_t>), grid, dim3(256), 0, s, a);
  else if (w_f32) hipLaunchKernelGGL((head_prepare_kernel<bf16_t, float>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((head_prepare_kernel<bf16_t, bf16_t>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_head_records(const HeadLabels& l, int64_t rows, int64_t rows_pad, int64_t vocab, const HeadRow* stats,
                               HeadRow* records, hipStream_t s) {
  hipLaunchKernelGGL(head_records_kernel, dim3((unsigned)((rows_pad + 255) / 256)), dim3(256), 0, s, l, rows, rows_pad, vocab, stats, records);
  return hipGetLastError();
}

}  // namespace malt
