// Root-mean-square norm of rows h = x + residual (rounded to their type: what is kept is
// what is normed), and its gradient:
//
//   r = 1 / sqrt(mean(h^2) + eps),  y = (h r) w
//   dh = r (dy w - n mean(dy w n)) + dsum,  n = h r;   dw = sum over rows of dy n
//
// Bound by memory: a row is read once, held in registers for its sum and its output, and
// x, residual, sum and y (h, dy, dsum and dx) pass through memory once each.
//
// The sum of squares is in 64 bits: squares of float32 numbers are exact there, and the order
// of summation changes r's last of 24 bits in one row of 10^8.  The 8-bit output has borders
// beside which that bit decides, so with float32 sums another order would be another result.
//
// y may leave as an operand of the 8-bit products (block_fp8.h): 32 lanes hold a block of 128
// columns, so that its largest magnitude is five exchanges away, and the float32 y is
// rounded once.
#include "block_mma.h"
#include "norm.h"
#include "ops_common.h"

namespace malt {

namespace {

__device__ __forceinline__ op_f32x4 weight4(const void* w, bool f32, int c, int width) {
  return f32 ? row_load4(static_cast<const float*>(w), c, width) : row_load4(static_cast<const bf16_t*>(w), c, width);
}

template <class V>
__device__ __forceinline__ V wave_sum(V v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
  return v;
}

// Sum over the TPR threads of a row, in each of them; `red` has a place for each wave.
// Calls in a row take turns with two places, so that one barrier each is enough.
template <int TPR, class V>
__device__ __forceinline__ V row_sum(V v, V* red) {
  v = wave_sum(v);
  if constexpr (TPR > 64) {
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) red[wave] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int i = 1; i < TPR / 64; ++i) v += red[i];
  }
  return v;
}

constexpr int threads_of(int tpr) { return tpr > 256 ? tpr : 256; }

// TPR threads a row, G groups of four columns each.
template <class T, int TPR, int G>
__global__ __launch_bounds__(threads_of(TPR)) void norm_kernel(NormArgs a) {
  constexpr int THREADS = threads_of(TPR), RPW = THREADS / TPR;
  __shared__ double red[THREADS / 64];
  const int tid = threadIdx.x % TPR;
  const int64_t r = (int64_t)blockIdx.x * RPW + threadIdx.x / TPR;
  if (r >= a.rows) return;   // whole waves; with more than one wave a row, whole workgroups
  const T* const x = static_cast<const T*>(a.x) + r * a.ldx;
  op_f32x4 h[G];
#pragma unroll
  for (int g = 0; g < G; ++g) h[g] = row_load4(x, 4 * (tid + TPR * g), a.width);
  if (a.residual) {
    const T* const res = static_cast<const T*>(a.residual) + r * a.ldr;
    T* const sum = static_cast<T*>(a.sum) + r * a.lds;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int c = 4 * (tid + TPR * g);
      const op_f32x4 v = row_load4(res, c, a.width);
#pragma unroll
      for (int j = 0; j < 4; ++j) h[g][j] = to_f32(from_f32<T>(h[g][j] + v[j]));
      row_store4(sum, c, a.width, h[g]);
    }
  }
  double s = 0.0;
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int j = 0; j < 4; ++j) s += (double)h[g][j] * (double)h[g][j];
  s = row_sum<TPR>(s, red);
  const float rstd = (float)(1.0 / sqrt(s / a.width + a.eps));
  if (a.rstd && tid == 0) gptr(a.rstd)[r] = rstd;
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const int c = 4 * (tid + TPR * g);
    const op_f32x4 w = weight4(a.weight, a.w_f32, c, a.width);
    op_f32x4 y;
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = (h[g][j] * rstd) * w[j];
    if (a.values) {
      const int64_t pitch = q_pad(a.width);
      uint32_t top = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) top = umax(top, mag(y[j]));
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) top = umax(top, (uint32_t)__shfl_xor((int)top, d, 64));
      const uint32_t byte = scale_byte(top);
      const float inv = scale_inverse(byte);
      if (c < pitch) {
        *reinterpret_cast<MALT_GLOBAL uint32_t*>(gptr(a.values) + r * pitch + c) =
            pack4(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
        if ((tid & 31) == 0)
          gptr(a.scales)[c / QB * q_scale_rows(a.rows) + r / QB * QB + q_scale_pos((int)(r % QB))] = (uint8_t)byte;
      }
    } else if (a.y_f32) {
      row_store4(static_cast<float*>(a.y) + r * a.ldy, c, a.width, y);
    } else {
      row_store4(static_cast<bf16_t*>(a.y) + r * a.ldy, c, a.width, y);
    }
  }
}

// A workgroup takes every gridDim.x-th group of rows and holds its columns' share of the
// weight's gradient in registers.  HOLD: the row's values stay in registers between the sum and
// the output; otherwise they are read again, from the cache.
template <class T, class D, int TPR, int G, bool HOLD>
__global__ __launch_bounds__(threads_of(TPR)) void norm_grad_kernel(NormGradArgs a) {
  constexpr int THREADS = threads_of(TPR), RPW = THREADS / TPR;
  __shared__ float red[2][THREADS / 64];
  __shared__ op_f32x4 join[RPW > 1 ? RPW : 1][RPW > 1 ? TPR * G : 1];
  const int tid = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  op_f32x4 acc[G];
#pragma unroll
  for (int g = 0; g < G; ++g) acc[g] = op_f32x4{0.f, 0.f, 0.f, 0.f};
  const T* const dsum = static_cast<const T*>(a.dsum);
  int turn = 0;
  for (int64_t r = (int64_t)blockIdx.x * RPW + sub; r < a.rows; r += (int64_t)gridDim.x * RPW) {
    const T* const h = static_cast<const T*>(a.h) + r * a.ldh;
    const D* const dy = static_cast<const D*>(a.dy) + r * a.ldy;
    const float rstd = gptr(a.rstd)[r];
    op_f32x4 n[HOLD ? G : 1], d[HOLD ? G : 1];
    float s = 0.f;
    if constexpr (HOLD) {
#pragma unroll
      for (int g = 0; g < G; ++g) {
        n[g] = row_load4(h, 4 * (tid + TPR * g), a.width);
        d[g] = row_load4(dy, 4 * (tid + TPR * g), a.width);
      }
    }
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int c = 4 * (tid + TPR * g), k = HOLD ? g : 0;
      if constexpr (!HOLD) {
        n[0] = row_load4(h, c, a.width);
        d[0] = row_load4(dy, c, a.width);
      }
      const op_f32x4 w = weight4(a.weight, a.w_f32, c, a.width);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        n[k][j] *= rstd;
        acc[g][j] += d[k][j] * n[k][j];
        d[k][j] *= w[j];
        s += d[k][j] * n[k][j];
      }
    }
    if (!a.dx) continue;   // the same for all threads
    s = row_sum<TPR>(s, red[turn]) / (float)a.width;
    turn ^= 1;
    T* const dx = static_cast<T*>(a.dx) + r * a.ldx;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int c = 4 * (tid + TPR * g), k = HOLD ? g : 0;
      if constexpr (!HOLD) {
        const op_f32x4 w = weight4(a.weight, a.w_f32, c, a.width);
        n[0] = row_load4(h, c, a.width);
        d[0] = row_load4(dy, c, a.width);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          n[0][j] *= rstd;
          d[0][j] *= w[j];
        }
      }
      op_f32x4 out;
#pragma unroll
      for (int j = 0; j < 4; ++j) out[j] = rstd * (d[k][j] - n[k][j] * s);
      if (dsum) {
        const op_f32x4 e = row_load4(dsum + r * a.lds, c, a.width);
#pragma unroll
        for (int j = 0; j < 4; ++j) out[j] += e[j];
      }
      row_store4(dx, c, a.width, out);
    }
  }
  if (!a.partial) return;
  if constexpr (RPW > 1) {
#pragma unroll
    for (int g = 0; g < G; ++g) join[sub][tid + TPR * g] = acc[g];
    __syncthreads();
    for (int i = threadIdx.x; i < TPR * G; i += THREADS) {
      op_f32x4 v = join[0][i];
#pragma unroll
      for (int k = 1; k < RPW; ++k) {
        const op_f32x4 u = join[k][i];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] += u[j];
      }
      row_store4(a.partial + (int64_t)blockIdx.x * a.width, 4 * i, a.width, v);
    }
  } else {
#pragma unroll
    for (int g = 0; g < G; ++g)
      row_store4(a.partial + (int64_t)blockIdx.x * a.width, 4 * (tid + TPR * g), a.width, acc[g]);
  }
}

// Sums of the parts, 16 columns a workgroup: thread (p, c) of 16 x 16 adds every 16th part.
template <class W>
__global__ __launch_bounds__(256) void norm_join_kernel(const float* partial, W* dweight, int parts, int width) {
  __shared__ float sums[16][17];
  const int c = blockIdx.x * 16 + (threadIdx.x & 15), p0 = threadIdx.x >> 4;
  float s = 0.f;
  if (c < width) {
#pragma unroll 8
    for (int p = p0; p < parts; p += 16) s += gptr(partial)[(int64_t)p * width + c];
  }
  sums[p0][threadIdx.x & 15] = s;
  __syncthreads();
  if (p0 == 0 && c < width) {
#pragma unroll
    for (int i = 1; i < 16; ++i) s += sums[i][threadIdx.x];
    gptr(dweight)[c] = from_f32<W>(s);
  }
}

template <class T, int TPR, int G>
void norm_shape(const NormArgs& a, hipStream_t s) {
  constexpr int THREADS = threads_of(TPR), RPW = THREADS / TPR;
  hipLaunchKernelGGL((norm_kernel<T, TPR, G>), dim3((unsigned)((a.rows + RPW - 1) / RPW)), dim3(THREADS), 0, s, a);
}
template <class T>
void norm_typed(const NormArgs& a, hipStream_t s) {
  const int64_t w = a.values ? q_pad(a.width) : a.width;
  if (w <= 512 && a.rows > 512) norm_shape<T, 64, 2>(a, s);
  else if (w <= 2048 && a.rows > 512) norm_shape<T, 64, 8>(a, s);
  else if (w <= 2048) norm_shape<T, 256, 2>(a, s);
  else if (w <= 8192) norm_shape<T, 256, 8>(a, s);
  else norm_shape<T, 1024, 4>(a, s);
}

// Rows that a workgroup of the gradient takes at a time.
int grad_rows(int64_t width) { return width <= 2048 ? 4 : 1; }

template <class T, class D, int TPR, int G, bool HOLD>
void grad_shape(const NormGradArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((norm_grad_kernel<T, D, TPR, G, HOLD>), dim3((unsigned)a.parts), dim3(threads_of(TPR)), 0, s, a);
}
template <class T, class D>
void grad_typed(const NormGradArgs& a, hipStream_t s) {
  if (a.width <= 512) grad_shape<T, D, 64, 2, true>(a, s);
  else if (a.width <= 2048) grad_shape<T, D, 64, 8, true>(a, s);
  else if (a.width <= 8192) grad_shape<T, D, 256, 8, true>(a, s);
  else grad_shape<T, D, 1024, 4, false>(a, s);
}

}  // namespace

int norm_grad_parts(int64_t rows, int64_t width) {
  const int64_t groups = (rows + grad_rows(width) - 1) / grad_rows(width);
  return (int)(groups < NORM_PARTS ? groups : NORM_PARTS);
}

hipError_t launch_norm(const NormArgs& a, bool f32, hipStream_t s) {
  if (f32) norm_typed<float>(a, s);
  else norm_typed<bf16_t>(a, s);
  return hipGetLastError();
}

hipError_t launch_norm_grad(const NormGradArgs& a, bool f32, hipStream_t s) {
  if (a.parts > 0) {
    if (f32 && a.dy_f32) grad_typed<float, float>(a, s);
    else if (f32) grad_typed<float, bf16_t>(a, s);
    else if (a.dy_f32) grad_typed<bf16_t, float>(a, s);
    else grad_typed<bf16_t, bf16_t>(a, s);
  }
  if (a.dweight) {
    const dim3 grid((unsigned)((a.width + 15) / 16));
    if (a.w_f32) hipLaunchKernelGGL((norm_join_kernel<float>), grid, dim3(256), 0, s, a.partial, static_cast<float*>(a.dweight), a.parts, a.width);
    else hipLaunchKernelGGL((norm_join_kernel<bf16_t>), grid, dim3(256), 0, s, a.partial, static_cast<bf16_t*>(a.dweight), a.parts, a.width);
  }
  return hipGetLastError();
}

}  // namespace malt
