// One AdamW step over many tensors:
//
//   g <- c g,  m <- b1 m + (1 - b1) g,  v <- b2 v + (1 - b2) g^2
//   p <- p (1 - lr decay) - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
//
// Bound by memory: p, m, v in and out, g in; 28 bytes an element in 32 bits, 16 with the
// moments in 8.  One launch takes up to 108 tensors, whose addresses lie in its arguments, so that
// nothing is copied before it; a workgroup takes 4096 places of one of them, a wave 256 at a time: four
// neighbours a lane.  64.3M elements: 347 us (5.2 TB/s), with 8-bit moments 222 (4.6 TB/s, beside which the
// instructions, some 400 for four elements, take nearly as long); 98 tensors of a width of 768: 5.3 us.
//
// Moments in 8 bits: 256 places, a wave's work, share a float32 scale s and hold codes of
// 3 mantissa bits.  Rounding to nearest would stop a moment from moving once a step
// changes it by less than half a code's step (1 - b2 is less than that), so a place is
// rounded up with the probability of its position between its two neighbours:
// floor(x / step + u) step, u from a hash of seed, tensor, block and place.  Sums over many
// steps then stay right on average.
//   first moment: sign, 4 exponent bits, 3 mantissa bits up to 448, s = max|m| / 448: 2^-18
//     of the largest is kept;
//   second: no sign, 5 exponent bits, 3 mantissa bits up to 61440 (a float16's bits shifted by
//     7), s = max v / 61440: 2^-33 of the largest.  A second moment above zero becomes zero only
//     with its whole block, and then the first moments go with it: where m outlives v the update
//     would be m / eps.  What m can keep otherwise (2^-18 of the largest, over the root of
//     2^-33) is an update of ordinary size.
// The step itself takes the moments before they are rounded.  Moments and codes are computed
// one rounding at a time (no fused multiply-add): the same bits on every machine.
#include "adamw.h"
#include "ops_common.h"

namespace malt {

namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64;
constexpr float FIRST_MAX = 448.f, SECOND_MAX = 61440.f;
constexpr float LEAST = 0x1p-100f;   // moments of a block whose largest is below are zero: its reciprocal times 61440 has to be a number

__device__ __forceinline__ uint32_t mixed(uint32_t x) {
  // Shifts, and products with odd numbers from the digits of the golden ratio and of the root of 3.
  x ^= x >> 16;
  x *= 0x9E3779B1u;
  x ^= x >> 15;
  x *= 0xBB67AE85u;
  return x ^ (x >> 16);
}

// Exchanges between registers: pairs, quads, halves of 16 lanes and 16 lanes mirrored, then rows of 16 and halves.
template <int CTRL>
__device__ __forceinline__ uint32_t max_with(uint32_t v) {
  const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
  return v > o ? v : o;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  v = max_with<0x140>(max_with<0x141>(max_with<0x4E>(max_with<0xB1>(v))));
  auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = p[0] > p[1] ? p[0] : p[1];
  p = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return p[0] > p[1] ? p[0] : p[1];
}

// x in [0, the format's largest], in steps of its binade (exponents from LO): its multiple below or above.
template <int LO>
__device__ __forceinline__ float to_step(float x, float u, float* step) {
#pragma clang fp contract(off)
  uint32_t e = __float_as_uint(x) & 0x7f800000u;
  e = e < (uint32_t)(LO + 127) << 23 ? (uint32_t)(LO + 127) << 23 : e;
  *step = __uint_as_float(e - (3u << 23));
  return floorf(x * __uint_as_float((257u << 23) - e) + u) * *step;   // exact but for the sum
}

// Codes of four first moments under inv = 448 / max.
__device__ __forceinline__ uint32_t first_codes(const float (&m)[4], float inv, const float (&u)[4]) {
  float r[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float step;
    r[j] = copysignf(to_step<-6>(fminf(fabsf(m[j]) * inv, FIRST_MAX), u[j], &step), m[j]);
  }
  int c = __builtin_amdgcn_cvt_pk_fp8_f32(r[0], r[1], 0, false);   // exact
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(r[2], r[3], c, true);
}
__device__ __forceinline__ uint32_t second_codes(const float (&v)[4], float inv, const float (&u)[4]) {
  float r[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float step;
    r[j] = to_step<-14>(fminf(v[j] * inv, SECOND_MAX), u[j], &step);
    if (v[j] > 0.f) r[j] = fmaxf(r[j], step);
  }
  const uint32_t lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(r[0], r[1]));   // exact
  const uint32_t hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(r[2], r[3]));
  return __builtin_amdgcn_perm(hi >> 7, lo >> 7, 0x06040200u);   // each half's bits 7 to 14
}
__device__ __forceinline__ void first_values(uint32_t c, float s, float (&m)[4]) {
  m[0] = __builtin_amdgcn_cvt_f32_fp8((int)c, 0) * s;
  m[1] = __builtin_amdgcn_cvt_f32_fp8((int)c, 1) * s;
  m[2] = __builtin_amdgcn_cvt_f32_fp8((int)c, 2) * s;
  m[3] = __builtin_amdgcn_cvt_f32_fp8((int)c, 3) * s;
}
__device__ __forceinline__ void second_values(uint32_t c, float s, float (&v)[4]) {
  typedef _Float16 half2 __attribute__((ext_vector_type(2)));
  const half2 lo = __builtin_bit_cast(half2, __builtin_amdgcn_perm(0u, c, 0x0c010c00u) << 7);   // a byte in each half
  const half2 hi = __builtin_bit_cast(half2, __builtin_amdgcn_perm(0u, c, 0x0c030c02u) << 7);
  v[0] = (float)lo.x * s;
  v[1] = (float)lo.y * s;
  v[2] = (float)hi.x * s;
  v[3] = (float)hi.y * s;
}

// The scale of a block and what its values are multiplied by; not a number where one of them is none.
__device__ __forceinline__ float block_scale(uint32_t top, float most, float* inv) {
#pragma clang fp contract(off)
  const float a = __uint_as_float(top);
  if (top >= 0x7f800000u) {
    *inv = 0.f;
    return __uint_as_float(0x7fc00000u);
  }
  if (a < LEAST) {
    *inv = 0.f;
    return 0.f;
  }
  *inv = (1.f / a) * most;
  return a * (1.f / most);
}

struct Where {
  int t;          // tensor of the launch
  int64_t at;     // first place of the chunk
};
__device__ __forceinline__ Where locate(const AdamArgs& a) {
  int lo = 0, hi = a.count - 1;   // the last tensor whose first chunk is not past this one
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.chunk[mid] <= blockIdx.x) lo = mid;
    else hi = mid - 1;
  }
  return {lo, (int64_t)(blockIdx.x - a.chunk[lo]) * ADAM_CHUNK};
}

// The moments that follow, in place.
__device__ __forceinline__ void moments(const AdamArgs& a, const float (&g)[4], float (&m)[4], float (&v)[4]) {
#pragma clang fp contract(off)
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    m[j] = m[j] * a.b1 + g[j] * a.c1;
    v[j] = v[j] * a.b2 + (g[j] * a.c2) * g[j];
  }
}
// The hardware's root and reciprocal, off by 2^-23 of their values: an update by less than 12 x 2^-24 of
// itself.  Correctly rounded ones made half of the 8-bit step's instructions, and that step wait for them.
__device__ __forceinline__ float fast_root(float v) {
  const bool small = v < 0x1p-96f;   // a subnormal number's root is taken of a normal one
  return __builtin_amdgcn_sqrtf(small ? v * 0x1p64f : v) * (small ? 0x1p-32f : 1.f);
}
__device__ __forceinline__ void weights(const AdamArgs& a, const float (&m)[4], const float (&v)[4], float (&p)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float down = __builtin_amdgcn_rcpf(__builtin_fmaf(fast_root(v[j]), a.root, a.eps));   // eps is no subnormal number
    p[j] = __builtin_fmaf(-(m[j] * a.rate), down, p[j] * a.shrink);
  }
}

__device__ __forceinline__ void spread(op_f32x4 x, float (&f)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) f[j] = x[j];
}
__device__ __forceinline__ op_f32x4 packed(const float (&f)[4]) { return op_f32x4{f[0], f[1], f[2], f[3]}; }

template <class P, class G>
__device__ __forceinline__ void step32(const AdamArgs& a, const AdamTensor& t, int64_t n, int64_t at, float gs) {
  P* const p = static_cast<P*>(t.param);
  const G* const g = static_cast<const G*>(t.grad);
  float *const ms = static_cast<float*>(t.state), *const vs = ms + n;
#pragma unroll 2
  for (int i = 0; i < ADAM_CHUNK / (4 * THREADS); ++i) {
    const int64_t c = at + 4 * (threadIdx.x + i * THREADS);
    if (c >= n) break;
    float pf[4], gf[4], m[4], v[4];
    spread(row_load4(g, c, n), gf);
    spread(row_load4(ms, c, n), m);
    spread(row_load4(vs, c, n), v);
    spread(row_load4(p, c, n), pf);
#pragma unroll
    for (int j = 0; j < 4; ++j) gf[j] *= gs;
    moments(a, gf, m, v);
    weights(a, m, v, pf);
    row_store4(p, c, n, packed(pf));
    row_store4(ms, c, n, packed(m));
    row_store4(vs, c, n, packed(v));
  }
}

template <class P, class G>
__device__ __forceinline__ void step8(const AdamArgs& a, const AdamTensor& t, int64_t n, int64_t at, float gs, uint32_t number) {
  P* const p = static_cast<P*>(t.param);
  const G* const g = static_cast<const G*>(t.grad);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t blocks = adam_blocks(n);
  uint8_t *const mc = static_cast<uint8_t*>(t.state), *const vc = mc + blocks * ADAM_BLOCK;
  float *const ms = reinterpret_cast<float*>(vc + blocks * ADAM_BLOCK), *const vs = ms + blocks;
  const uint32_t key = mixed(a.seed_lo ^ mixed(a.seed_hi + 0x9E3779B1u * (number + 1)));
  for (int i = wave; i < ADAM_CHUNK / ADAM_BLOCK; i += WAVES) {
    const int64_t b = at / ADAM_BLOCK + i, c = b * ADAM_BLOCK + 4 * lane;
    if (b >= blocks) break;
    float pf[4], gf[4], m[4], v[4];
    const uint32_t cm = *reinterpret_cast<const MALT_GLOBAL uint32_t*>(gptr(mc) + c);
    const uint32_t cv = *reinterpret_cast<const MALT_GLOBAL uint32_t*>(gptr(vc) + c);
    const float sm = gptr(ms)[b], sv = gptr(vs)[b];
    spread(row_load4(g, c, n), gf);   // zeros past the end, as the moments are there
    spread(row_load4(p, c, n), pf);
    first_values(cm, sm, m);
    second_values(cv, sv, v);
#pragma unroll
    for (int j = 0; j < 4; ++j) gf[j] *= gs;
    moments(a, gf, m, v);
    weights(a, m, v, pf);
    row_store4(p, c, n, packed(pf));
    uint32_t tm = 0, tv = 0;
    float um[4], uv[4];
    const uint32_t kb = mixed(key + (uint32_t)b * 0x9E3779B1u);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t bm = __float_as_uint(m[j]) & 0x7fffffffu, bv = __float_as_uint(v[j]) & 0x7fffffffu;
      tm = tm > bm ? tm : bm;
      tv = tv > bv ? tv : bv;
      const uint32_t r = mixed(kb ^ (uint32_t)(4 * lane + j));
      um[j] = __builtin_fmaf((float)(r & 0xffffu), 0x1p-16f, 0x1p-17f);   // exact
      uv[j] = __builtin_fmaf((float)(r >> 16), 0x1p-16f, 0x1p-17f);
    }
    float im, iv;
    const float nv = block_scale(wave_max(tv), SECOND_MAX, &iv);
    float nm = block_scale(wave_max(tm), FIRST_MAX, &im);
    if (nv == 0.f && nm > 0.f) nm = 0.f;
    *reinterpret_cast<MALT_GLOBAL uint32_t*>(gptr(mc) + c) = nm > 0.f ? first_codes(m, im, um) : 0u;
    *reinterpret_cast<MALT_GLOBAL uint32_t*>(gptr(vc) + c) = nv > 0.f ? second_codes(v, iv, uv) : 0u;
    if (lane == 0) {
      gptr(ms)[b] = nm;
      gptr(vs)[b] = nv;
    }
  }
}

__global__ __launch_bounds__(THREADS) void adamw_kernel(AdamArgs a) {
  const Where w = locate(a);
  const AdamTensor& t = a.t[w.t];
  const int64_t flags = t.numel, n = flags & (ADAM_P_F32 - 1);
  float gs = a.grad_scale;
  if (a.grad_scale_at) gs *= gptr(a.grad_scale_at)[0];
  const uint32_t number = (uint32_t)(a.first + w.t);
  const bool pf = flags & ADAM_P_F32, gf = flags & ADAM_G_F32;
  if (flags & ADAM_8BIT) {
    if (pf && gf) step8<float, float>(a, t, n, w.at, gs, number);
    else if (pf) step8<float, bf16_t>(a, t, n, w.at, gs, number);
    else if (gf) step8<bf16_t, float>(a, t, n, w.at, gs, number);
    else step8<bf16_t, bf16_t>(a, t, n, w.at, gs, number);
  } else {
    if (pf && gf) step32<float, float>(a, t, n, w.at, gs);
    else if (pf) step32<float, bf16_t>(a, t, n, w.at, gs);
    else if (gf) step32<bf16_t, float>(a, t, n, w.at, gs);
    else step32<bf16_t, bf16_t>(a, t, n, w.at, gs);
  }
}

// What 8-bit moments stand for: float32 m[numel], then v[numel].
__global__ __launch_bounds__(THREADS) void adamw_moments_kernel(AdamArgs a) {
  const Where w = locate(a);
  const AdamTensor& t = a.t[w.t];
  const int64_t n = t.numel & (ADAM_P_F32 - 1), blocks = adam_blocks(n);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint8_t *const mc = static_cast<const uint8_t*>(t.state), *const vc = mc + blocks * ADAM_BLOCK;
  const float *const ms = reinterpret_cast<const float*>(vc + blocks * ADAM_BLOCK), *const vs = ms + blocks;
  float* const out = static_cast<float*>(t.param);
  for (int i = wave; i < ADAM_CHUNK / ADAM_BLOCK; i += WAVES) {
    const int64_t b = w.at / ADAM_BLOCK + i, c = b * ADAM_BLOCK + 4 * lane;
    if (b >= blocks) break;
    float m[4], v[4];
    first_values(*reinterpret_cast<const MALT_GLOBAL uint32_t*>(gptr(mc) + c), gptr(ms)[b], m);
    second_values(*reinterpret_cast<const MALT_GLOBAL uint32_t*>(gptr(vc) + c), gptr(vs)[b], v);
    row_store4(out, c, n, packed(m));
    row_store4(out + n, c, n, packed(v));
  }
}

}  // namespace

hipError_t launch_adamw(const AdamArgs& a, uint32_t chunks, hipStream_t s) {
  hipLaunchKernelGGL(adamw_kernel, dim3(chunks), dim3(THREADS), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_adamw_moments(const AdamArgs& a, uint32_t chunks, hipStream_t s) {
  hipLaunchKernelGGL(adamw_moments_kernel, dim3(chunks), dim3(THREADS), 0, s, a);
  return hipGetLastError();
}

}  // namespace malt
