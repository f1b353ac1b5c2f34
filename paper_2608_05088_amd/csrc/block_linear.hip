// A linear layer on kept 8-bit weights for a few rows (generated tokens), in one
// launch: out (M x N) = Q(x) (M x K) W (N x K)^T with M <= 32.
//
// Bound by reading the weights.  A workgroup takes 16 NB columns; its eight waves
// take every eighth block of 128 k and join their sums through LDS in a fixed
// order.  Each wave brings the rows of x it needs to 8 bits in registers, as the
// matrix instruction takes them: a lane holds 32 of a row's 128 values, so the
// block's maximum is two exchanges away.  A separate conversion would cost a
// launch and a round trip through memory, longer than the product itself.
//
// Measured: one token, 1280 -> 5120 (6.6 MB of weights) 5.9 us: of ten blocks two waves
// take two, and a block is a chain of loads, exchanges and products with nothing
// loaded ahead, then the join; 4096 -> 16384 (67 MB) 18 us, 3.7 TB/s; 32 tokens 29.
#include <type_traits>

#include "block_mma.h"

namespace malt {

namespace {

using ns::bf16x8;
using ns::f32x4;
using ns::i32x4;

constexpr int FEW_WAVES = 8;

template <class T, int MB, int NB, class TO>
__global__ __launch_bounds__(64 * FEW_WAVES) void block_linear_kernel(BlockLinearArgs g) {
  constexpr bool WIDE = std::is_same<TO, float>::value;
  __shared__ f32x4 sums[FEW_WAVES][MB * NB][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int KT = (int)((g.k + QB - 1) / QB);
  const int64_t kp = (int64_t)KT * QB, n0 = (int64_t)blockIdx.x * (16 * NB);
  const int r = lane & 15, k_lane = 32 * (lane >> 4);
  const uint8_t* w[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int64_t n = n0 + 16 * b + r;   // rows past the end repeat the last one and are not stored
    w[b] = g.w + (n < g.n ? n : g.n - 1) * kp + k_lane;
  }
  const T* x[MB];
#pragma unroll
  for (int a = 0; a < MB; ++a) {
    const int m = 16 * a + r;
    x[a] = static_cast<const T*>(g.x) + (m < g.m ? m : g.m - 1) * g.ldx;
  }
  const uint8_t* const ws = g.w_scales + n0 / QB * KT;

  f32x4 acc[MB][NB];
#pragma unroll
  for (int a = 0; a < MB; ++a)
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[a][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int kt = wave; kt < KT; kt += FEW_WAVES) {
    i32x8 fw[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const MALT_GLOBAL i32x4* p = reinterpret_cast<const MALT_GLOBAL i32x4*>(gptr(w[b]) + (int64_t)kt * QB);
      const i32x4 lo = p[0], hi = p[1];
      fw[b] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    const int sw = gptr(ws)[kt];   // 16 NB <= 64 columns lie in one block of the weight
#pragma unroll
    for (int a = 0; a < MB; ++a) {
      float v[4][8];
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        load8(x[a], kt * QB + k_lane + 8 * i, (int)g.k, v[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) top = umax(top, mag(v[i][j]));
      }
      top = umax(top, (uint32_t)__shfl_xor((int)top, 16, 64));
      top = umax(top, (uint32_t)__shfl_xor((int)top, 32, 64));
      const int sx = (int)scale_byte(top);
      const float inv = scale_inverse((uint32_t)sx);
      i32x8 fx;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        fx[2 * i] = (int)pack4(v[i][0] * inv, v[i][1] * inv, v[i][2] * inv, v[i][3] * inv);
        fx[2 * i + 1] = (int)pack4(v[i][4] * inv, v[i][5] * inv, v[i][6] * inv, v[i][7] * inv);
      }
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        if constexpr (WIDE) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            acc[a][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(fw[b][2 * i], fw[b][2 * i + 1], scale_of(sw, 0)),
                                                                widen(fx[2 * i], fx[2 * i + 1], scale_of(sx, 0)),
                                                                acc[a][b], 0, 0, 0);
        } else {
          acc[a][b] = mma<0, 0>(fw[b], fx, acc[a][b], sw, sx);
        }
      }
    }
  }
#pragma unroll
  for (int a = 0; a < MB; ++a)
#pragma unroll
    for (int b = 0; b < NB; ++b) sums[wave][a * NB + b][lane] = acc[a][b];
  __syncthreads();
  // Block q of the tile, lane l: row l % 16 of row block q / NB, columns 4 (l / 16) .. + 3.
  for (int i = threadIdx.x; i < MB * NB * 64; i += 64 * FEW_WAVES) {
    const int q = i >> 6, l = i & 63;
    f32x4 v = sums[0][q][l];
#pragma unroll
    for (int u = 1; u < FEW_WAVES; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += sums[u][q][l][e];
    const int m = 16 * (q / NB) + (l & 15);
    const int64_t n = n0 + 16 * (q % NB) + 4 * (l >> 4);
    if (m >= g.m) continue;
    row_store4(static_cast<TO*>(g.out) + m * g.ldo, n, g.n, op_f32x4{v[0], v[1], v[2], v[3]});
  }
}

template <class T, int MB, class TO>
void few_rows(const BlockLinearArgs& g, hipStream_t s) {
  // Two column blocks a workgroup where that still leaves more than one a CU.  us with one and
  // two: 1 token, 5120 -> 1280 (80 blocks) 10.4 and 11.0, 16 tokens 10.4 and 12.6, 17 tokens,
  // 4096 -> 4096 (256) 13.0 and 14.5; 16 tokens, 2048 -> 16384 (1024) 14.1 and 10.3.
  const int64_t blocks = (g.n + 15) / 16;
  if (blocks <= 384) hipLaunchKernelGGL((block_linear_kernel<T, MB, 1, TO>), dim3((unsigned)blocks), dim3(64 * FEW_WAVES), 0, s, g);
  else hipLaunchKernelGGL((block_linear_kernel<T, MB, 2, TO>), dim3((unsigned)((blocks + 1) / 2)), dim3(64 * FEW_WAVES), 0, s, g);
}
template <class T, class TO>
void few_typed(const BlockLinearArgs& g, hipStream_t s) {
  if (g.m <= 16) few_rows<T, 1, TO>(g, s);
  else few_rows<T, 2, TO>(g, s);
}

}  // namespace

hipError_t launch_block_linear(const BlockLinearArgs& g, bool x_f32, bool out_f32, hipStream_t s) {
  if (x_f32 && out_f32) few_typed<float, float>(g, s);
  else if (x_f32) few_typed<float, bf16_t>(g, s);
  else if (out_f32) few_typed<bf16_t, float>(g, s);
  else few_typed<bf16_t, bf16_t>(g, s);
  return hipGetLastError();
}

}  // namespace malt
