// Root-mean-square norm of rows h = x + residual (rounded to their type: what is kept is
// what is normed), and its gradient:
//
//   r = 1 / sqrt(mean(h^2) + eps),  y = (h r) w
//   dh = r (dy w - n mean(dy w n)) + dsum,  n = h r;   dw = sum over rows of dy n
//
// Bound by memory: a row is read once, held in registers for its sum and its output, and
// x, residual, sum and y (h, dy, dsum and dx) pass through memory once each.
// 8192 x 1280 in bf16, 84 MB each way: 18 us (4.7 TB/s), the gradient 27 (3.1 TB/s) and 4 for the join
// of the weight's.  The gradient waits for a row's sum before it can write and holds the weight's columns besides; the
// next row's loads ahead of that took 27 to 29.  One row: 3.5 us; 1024 rows of 1280 into 8 bits 5.8.
//
// The sum of squares is in 64 bits: squares of float32 numbers are exact there, and the order
// of summation changes r's last of 24 bits in one row of 10^8.  The 8-bit output has borders
// beside which that bit decides, so with float32 sums another order would be another result.
//
// y may leave as an operand of the 8-bit products (block_fp8.h): 16 lanes hold a block of 128
// columns, so that its largest magnitude is four exchanges away, and the float32 y is
// rounded once.
#include "block_mma.h"
#include "norm.h"
#include "ops_common.h"

namespace malt {

namespace {

// Eight neighbouring columns c .. c + 7 of a row; what lies past its end is zero and is not stored.
struct Eight {
  float v[8];
};
template <class T>
__device__ __forceinline__ Eight get8(const T* row, int c, int width) {
  Eight r;
  load8(row, c, width, r.v);
  return r;
}
__device__ __forceinline__ void put8(float* row, int c, int width, const Eight& r) {
  row_store4(row, c, width, op_f32x4{r.v[0], r.v[1], r.v[2], r.v[3]});
  row_store4(row, c + 4, width, op_f32x4{r.v[4], r.v[5], r.v[6], r.v[7]});
}
__device__ __forceinline__ void put8(bf16_t* row, int c, int width, const Eight& r) {
  if (c + 8 <= width) {
    op_u32x4 q;
#pragma unroll
    for (int j = 0; j < 4; ++j) q[j] = pack_bf16x2(r.v[2 * j], r.v[2 * j + 1]);
    *reinterpret_cast<MALT_GLOBAL op_u32x4_any*>(gptr(row) + c) = q;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (c + j < width) gptr(row)[c + j] = from_f32<bf16_t>(r.v[j]);
  }
}
__device__ __forceinline__ Eight weight8(const void* w, bool f32, int c, int width) {
  return f32 ? get8(static_cast<const float*>(w), c, width) : get8(static_cast<const bf16_t*>(w), c, width);
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

// TPR threads a row, G groups of eight columns each.
template <class T, int TPR, int G>
__global__ __launch_bounds__(threads_of(TPR)) void norm_kernel(NormArgs a) {
  constexpr int THREADS = threads_of(TPR), RPW = THREADS / TPR;
  __shared__ double red[THREADS / 64];
  const int tid = threadIdx.x % TPR;
  const int64_t r = (int64_t)blockIdx.x * RPW + threadIdx.x / TPR;
  if (r >= a.rows) return;   // whole waves; with more than one wave a row, whole workgroups
  const T* const x = static_cast<const T*>(a.x) + r * a.ldx;
  Eight h[G];
#pragma unroll
  for (int g = 0; g < G; ++g) h[g] = get8(x, 8 * (tid + TPR * g), a.width);
  if (a.residual) {
    const T* const res = static_cast<const T*>(a.residual) + r * a.ldr;
    T* const sum = static_cast<T*>(a.sum) + r * a.lds;
    Eight v[G];
#pragma unroll
    for (int g = 0; g < G; ++g) v[g] = get8(res, 8 * (tid + TPR * g), a.width);
#pragma unroll
    for (int g = 0; g < G; ++g) {
#pragma unroll
      for (int j = 0; j < 8; ++j) h[g].v[j] = to_f32(from_f32<T>(h[g].v[j] + v[g].v[j]));
      put8(sum, 8 * (tid + TPR * g), a.width, h[g]);
    }
  }
  double s = 0.0;
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int j = 0; j < 8; ++j) s += (double)h[g].v[j] * (double)h[g].v[j];
  s = row_sum<TPR>(s, red);
  const float rstd = (float)(1.0 / sqrt(s / a.width + a.eps));
  if (a.rstd && tid == 0) gptr(a.rstd)[r] = rstd;
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const int c = 8 * (tid + TPR * g);
    const Eight w = weight8(a.weight, a.w_f32, c, a.width);
    Eight y;
#pragma unroll
    for (int j = 0; j < 8; ++j) y.v[j] = (h[g].v[j] * rstd) * w.v[j];
    if (a.values) {
      const int64_t pitch = q_pad(a.width);
      uint32_t top = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) top = umax(top, mag(y.v[j]));
#pragma unroll
      for (int d = 1; d < 16; d <<= 1) top = umax(top, (uint32_t)__shfl_xor((int)top, d, 64));
      const uint32_t byte = scale_byte(top);
      const float inv = scale_inverse(byte);
      if (c < pitch) {
        *reinterpret_cast<MALT_GLOBAL op_u32x2*>(gptr(a.values) + r * pitch + c) =
            op_u32x2{pack4(y.v[0] * inv, y.v[1] * inv, y.v[2] * inv, y.v[3] * inv),
                     pack4(y.v[4] * inv, y.v[5] * inv, y.v[6] * inv, y.v[7] * inv)};
        if ((tid & 15) == 0)
          gptr(a.scales)[c / QB * q_scale_rows(a.rows) + r / QB * QB + q_scale_pos((int)(r % QB))] = (uint8_t)byte;
      }
    } else if (a.y_f32) {
      put8(static_cast<float*>(a.y) + r * a.ldy, c, a.width, y);
    } else {
      put8(static_cast<bf16_t*>(a.y) + r * a.ldy, c, a.width, y);
    }
  }
}

// A workgroup takes every gridDim.x-th group of rows and holds its columns' share of the
// weight's gradient in registers.
template <class T, class D, int TPR, int G>
__global__ __launch_bounds__(threads_of(TPR)) void norm_grad_kernel(NormGradArgs a) {
  constexpr int THREADS = threads_of(TPR), RPW = THREADS / TPR;
  __shared__ float red[2][THREADS / 64];
  __shared__ float join[RPW > 1 ? RPW : 1][RPW > 1 ? 8 * TPR * G : 1];
  const int tid = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  Eight acc[G];
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[g].v[j] = 0.f;
  const T* const dsum = static_cast<const T*>(a.dsum);
  int turn = 0;
  for (int64_t r = (int64_t)blockIdx.x * RPW + sub; r < a.rows; r += (int64_t)gridDim.x * RPW) {
    const T* const h = static_cast<const T*>(a.h) + r * a.ldh;
    const D* const dy = static_cast<const D*>(a.dy) + r * a.ldy;
    const float rstd = gptr(a.rstd)[r];
    Eight n[G], d[G];
    float s = 0.f;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      n[g] = get8(h, 8 * (tid + TPR * g), a.width);
      d[g] = get8(dy, 8 * (tid + TPR * g), a.width);
    }
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const Eight w = weight8(a.weight, a.w_f32, 8 * (tid + TPR * g), a.width);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        n[g].v[j] *= rstd;
        acc[g].v[j] += d[g].v[j] * n[g].v[j];
        d[g].v[j] *= w.v[j];
        s += d[g].v[j] * n[g].v[j];
      }
    }
    if (!a.dx) continue;   // the same for all threads
    s = row_sum<TPR>(s, red[turn]) / (float)a.width;
    turn ^= 1;
    T* const dx = static_cast<T*>(a.dx) + r * a.ldx;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int c = 8 * (tid + TPR * g);
#pragma unroll
      for (int j = 0; j < 8; ++j) d[g].v[j] = rstd * (d[g].v[j] - n[g].v[j] * s);
      if (dsum) {
        const Eight e = get8(dsum + r * a.lds, c, a.width);
#pragma unroll
        for (int j = 0; j < 8; ++j) d[g].v[j] += e.v[j];
      }
      put8(dx, c, a.width, d[g]);
    }
  }
  if (!a.partial) return;
  float* const out = a.partial + (int64_t)blockIdx.x * a.width;
  if constexpr (RPW > 1) {
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int j = 0; j < 8; ++j) join[sub][j * TPR * G + tid + TPR * g] = acc[g].v[j];   // column 8 i + j at j TPR G + i
    __syncthreads();
    for (int i = threadIdx.x; i < TPR * G; i += THREADS) {
      Eight v;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v.v[j] = join[0][j * TPR * G + i];
#pragma unroll
        for (int k = 1; k < RPW; ++k) v.v[j] += join[k][j * TPR * G + i];
      }
      put8(out, 8 * i, a.width, v);
    }
  } else {
#pragma unroll
    for (int g = 0; g < G; ++g) put8(out, 8 * (tid + TPR * g), a.width, acc[g]);
  }
}

// Sums of the parts, 16 columns a workgroup: thread (p, c) of 32 x 16 adds every 32nd part.
template <class W>
__global__ __launch_bounds__(512) void norm_join_kernel(const float* partial, W* dweight, int parts, int width) {
  __shared__ float sums[32][17];
  const int c = blockIdx.x * 16 + (threadIdx.x & 15), p0 = threadIdx.x >> 4;
  float s = 0.f;
  if (c < width) {
#pragma unroll 16
    for (int p = p0; p < parts; p += 32) s += gptr(partial)[(int64_t)p * width + c];
  }
  sums[p0][threadIdx.x & 15] = s;
  __syncthreads();
  if (p0 == 0 && c < width) {
#pragma unroll
    for (int i = 1; i < 32; ++i) s += sums[i][threadIdx.x];
    gptr(dweight)[c] = from_f32<W>(s);
  }
}

template <class T, int TPR, int G>
void norm_shape(const NormArgs& a, hipStream_t s) {
  constexpr int THREADS = threads_of(TPR), RPW = THREADS / TPR;
  hipLaunchKernelGGL((norm_kernel<T, TPR, G>), dim3((unsigned)((a.rows + RPW - 1) / RPW)), dim3(THREADS), 0, s, a);
}
// A wave a row up to 2048 columns, where there are rows enough for a wave each on every SIMD; a
// workgroup otherwise.
template <class T>
void norm_typed(const NormArgs& a, hipStream_t s) {
  const int64_t w = a.values ? q_pad(a.width) : a.width;
  const bool many = a.rows > 2048;
  if (w <= 512 && many) norm_shape<T, 64, 1>(a, s);
  else if (w <= 1024 && many) norm_shape<T, 64, 2>(a, s);
  else if (w <= 1536 && many) norm_shape<T, 64, 3>(a, s);
  else if (w <= 2048 && many) norm_shape<T, 64, 4>(a, s);
  else if (w <= 2048) norm_shape<T, 256, 1>(a, s);
  else if (w <= 4096) norm_shape<T, 256, 2>(a, s);
  else if (w <= 8192) norm_shape<T, 256, 4>(a, s);
  else norm_shape<T, 1024, 2>(a, s);
}

// Rows that a workgroup of the gradient takes at a time.
int grad_rows(int64_t width) { return width <= 2048 ? 4 : 1; }

template <class T, class D, int TPR, int G>
void grad_shape(const NormGradArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((norm_grad_kernel<T, D, TPR, G>), dim3((unsigned)a.parts), dim3(threads_of(TPR)), 0, s, a);
}
template <class T, class D>
void grad_typed(const NormGradArgs& a, hipStream_t s) {
  if (a.width <= 512) grad_shape<T, D, 64, 1>(a, s);
  else if (a.width <= 1024) grad_shape<T, D, 64, 2>(a, s);
  else if (a.width <= 1536) grad_shape<T, D, 64, 3>(a, s);
  else if (a.width <= 2048) grad_shape<T, D, 64, 4>(a, s);
  else if (a.width <= 4096) grad_shape<T, D, 256, 2>(a, s);
  else if (a.width <= 8192) grad_shape<T, D, 256, 4>(a, s);
  else grad_shape<T, D, 1024, 2>(a, s);
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
    if (a.w_f32) hipLaunchKernelGGL((norm_join_kernel<float>), grid, dim3(512), 0, s, a.partial, static_cast<float*>(a.dweight), a.parts, a.width);
    else hipLaunchKernelGGL((norm_join_kernel<bf16_t>), grid, dim3(512), 0, s, a.partial, static_cast<bf16_t*>(a.dweight), a.parts, a.width);
  }
  return hipGetLastError();
}

}  // namespace malt
