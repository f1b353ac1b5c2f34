// Bringing a matrix to 8 bits with a power-of-two scale for each block of 128:
// s = 2^e with the least e >= -127 for which max|x| <= 448 s, q = x / s rounded
// to the nearest 8-bit float.  A power of two makes the division exact and lets
// the matrix instruction apply the scale by itself.
//
// Bound by memory: one workgroup reads a 128 x 128 tile once, into registers,
// and writes what is wanted of it: the rows' form (blocks along a row), the
// transpose's (blocks along a column), or both under one scale (a weight).
//
// Measured (a large copy reaches 5.17 TB/s on the same card): 8192 x 5120 bf16, both
// forms, 37 us, 4.5 TB/s; 8192 x 1280 bf16, rows only, 8.3 us, 3.8 TB/s; that matrix in
// both forms and a 5120 x 1280 float32 weight in one launch 24 us, 3.4 TB/s.
#include "block_mma.h"
#include "ops_common.h"

namespace malt {

namespace {

// Maximum over the 16 lanes of a row of lanes, in every one of them.
__device__ __forceinline__ uint32_t max16(uint32_t v) {
  v = umax(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xf, 0xf, true));   // rotate by 8, 4, 2, 1
  v = umax(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x124, 0xf, 0xf, true));
  v = umax(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x122, 0xf, 0xf, true));
  v = umax(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x121, 0xf, 0xf, true));
  return v;
}

struct QuantShared {
  __attribute__((aligned(16))) uint8_t tile[QB * QB];   // the transpose's bytes
  uint32_t col_max[8][QB];
};

// Tile (bx, by) of one matrix.  Thread (rg, cg) of 512 holds rows 4 rg .. + 3,
// columns 8 cg .. + 7 of the tile.  WEIGHT: one scale for the whole tile.
template <class T, bool WEIGHT>
__device__ __forceinline__ void quantize_tile(const QuantArgs& a, int bx, int by, QuantShared& sh) {
  uint8_t* const tile = sh.tile;
  uint32_t(*const col_max)[QB] = sh.col_max;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int cg = tid & 15, rg = tid >> 4;
  const int64_t r0 = (int64_t)by * QB, c0 = (int64_t)bx * QB;
  const int rows = (int)(a.rows - r0 < QB ? a.rows - r0 : QB), cols = (int)(a.cols - c0 < QB ? a.cols - c0 : QB);
  const T* x = static_cast<const T*>(a.x) + r0 * a.ld + c0;
  const int64_t pitch = q_pad(a.cols), t_pitch = q_pad(a.rows);

  float v[4][8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = 4 * rg + i;
    if (r < rows) load8(x + (int64_t)r * a.ld, 8 * cg, cols, v[i]);
    else
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
  }

  uint32_t one = 127;   // the tile's scale
  if constexpr (WEIGHT) {
    uint32_t b = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) b = umax(b, mag(v[i][j]));
    b = max16(b);
    b = umax(b, (uint32_t)__shfl_xor((int)b, 16, 64));
    b = umax(b, (uint32_t)__shfl_xor((int)b, 32, 64));
    if (lane == 0) col_max[wave][0] = b;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 8; ++w) b = umax(b, col_max[w][0]);
    one = scale_byte(b);
    if (tid == 0) gptr(a.block_scales)[by * (pitch / QB) + bx] = (uint8_t)one;
  }

  if (a.values) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 4 * rg + i;
      uint32_t byte = one;
      if constexpr (!WEIGHT) {
        uint32_t b = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) b = umax(b, mag(v[i][j]));
        byte = scale_byte(max16(b));
      }
      if (r < rows) {
        const float s = scale_inverse(byte);
        const op_u32x2 q = {pack4(v[i][0] * s, v[i][1] * s, v[i][2] * s, v[i][3] * s),
                            pack4(v[i][4] * s, v[i][5] * s, v[i][6] * s, v[i][7] * s)};
        *reinterpret_cast<MALT_GLOBAL op_u32x2*>(gptr(a.values) + (r0 + r) * pitch + c0 + 8 * cg) = q;
        if (!WEIGHT && cg == 0)
          gptr(a.scales)[bx * q_scale_rows(a.rows) + r0 + q_scale_pos(r)] = (uint8_t)byte;
      }
    }
  }

  if (a.t_values) {
    uint32_t byte[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) byte[j] = one;
    if constexpr (!WEIGHT) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        uint32_t b = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) b = umax(b, mag(v[i][j]));
        b = umax(b, (uint32_t)__shfl_xor((int)b, 16, 64));
        b = umax(b, (uint32_t)__shfl_xor((int)b, 32, 64));
        if (lane < 16) col_max[wave][8 * cg + j] = b;
      }
      __syncthreads();
      if (tid < QB) {   // thread c: column c's scale
        uint32_t b = 0;
#pragma unroll
        for (int w = 0; w < 8; ++w) b = umax(b, col_max[w][tid]);
        b = scale_byte(b);
        col_max[0][tid] = b;
        if (tid < cols) gptr(a.t_scales)[by * q_scale_rows(a.cols) + c0 + q_scale_pos(tid)] = (uint8_t)b;
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 8; ++j) byte[j] = col_max[0][8 * cg + j];
    }
    // Column c's 128 bytes lie in 4-byte pieces, piece rg at rg ^ 2 (c / 8) (its
    // lowest bit kept): the 16 lanes that write one rg and column spread over the banks.
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float s = scale_inverse(byte[j]);
      *reinterpret_cast<uint32_t*>(tile + (8 * cg + j) * QB + ((rg ^ (2 * cg)) << 2)) =
          pack4(v[0][j] * s, v[1][j] * s, v[2][j] * s, v[3][j] * s);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int c = (tid >> 3) + 64 * i, p = tid & 7;   // column, 16-byte piece of its 128 bytes
      const int g = c >> 3;
      // Pieces 4 p .. 4 p + 3 lie in one 16-byte run, its halves swapped where bit 1 of 2 g is set.
      op_u32x4 q = *reinterpret_cast<const op_u32x4*>(tile + c * QB + ((p ^ (g >> 1)) << 4));
      if (g & 1) q = op_u32x4{q.z, q.w, q.x, q.y};
      if (c < cols) *reinterpret_cast<MALT_GLOBAL op_u32x4*>(gptr(a.t_values) + (c0 + c) * t_pitch + r0 + 16 * p) = q;
    }
  }
}

template <class T, bool WEIGHT>
__global__ __launch_bounds__(512) void block_quant_kernel(QuantArgs a) {
  __shared__ QuantShared sh;
  quantize_tile<T, WEIGHT>(a, blockIdx.x, blockIdx.y, sh);
}

// A layer's input and weight in one launch: x's tiles, then w's.
template <class TX, class TW>
__global__ __launch_bounds__(512) void block_quant_pair_kernel(QuantArgs x, QuantArgs w, int x_tiles, int x_cols, int w_cols) {
  __shared__ QuantShared sh;
  const int b = blockIdx.x;
  if (b < x_tiles) quantize_tile<TX, false>(x, b % x_cols, b / x_cols, sh);
  else quantize_tile<TW, true>(w, (b - x_tiles) % w_cols, (b - x_tiles) / w_cols, sh);
}

template <class T>
void quant_typed(const QuantArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(q_pad(a.cols) / QB), (unsigned)(q_pad(a.rows) / QB));
  if (a.block_scales) hipLaunchKernelGGL((block_quant_kernel<T, true>), grid, dim3(512), 0, s, a);
  else hipLaunchKernelGGL((block_quant_kernel<T, false>), grid, dim3(512), 0, s, a);
}

template <class TX, class TW>
void pair_typed(const QuantArgs& x, const QuantArgs& w, hipStream_t s) {
  const int xc = int(q_pad(x.cols) / QB), wc = int(q_pad(w.cols) / QB);
  const int64_t xt = xc * (q_pad(x.rows) / QB), wt = wc * (q_pad(w.rows) / QB);
  hipLaunchKernelGGL((block_quant_pair_kernel<TX, TW>), dim3((unsigned)(xt + wt)), dim3(512), 0, s, x, w, int(xt), xc, wc);
}

}  // namespace

hipError_t launch_block_quant(const QuantArgs& a, bool f32, hipStream_t s) {
  if (f32) quant_typed<float>(a, s);
  else quant_typed<bf16_t>(a, s);
  return hipGetLastError();
}

hipError_t launch_block_quant_pair(const QuantArgs& x, bool x_f32, const QuantArgs& w, bool w_f32, hipStream_t s) {
  if (x_f32 && w_f32) pair_typed<float, float>(x, w, s);
  else if (x_f32) pair_typed<float, bf16_t>(x, w, s);
  else if (w_f32) pair_typed<bf16_t, float>(x, w, s);
  else pair_typed<bf16_t, bf16_t>(x, w, s);
  return hipGetLastError();
}

}  // namespace malt
