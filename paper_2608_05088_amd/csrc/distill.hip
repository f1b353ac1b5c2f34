// Distillation loss of one row of student logits z over the vocabulary against
// a teacher's top logits a_j at ids i_j, labels y mixed in, and its gradient:
//
//   p = softmax(a / tau) over the row's valid entries, q = softmax(z / tau), q1 = softmax(z)
//   loss = (1 - alpha) tau^2 sum_j p_j (log p_j - log q_{i_j}) - alpha log q1_y
//   dz   = w [ (1 - alpha) tau (q - p) + alpha (q1 - 1_y) ]
//
// Bound by memory: z in and dz out, 6 flops and one exponential a column.  A workgroup
// takes a row and holds it on the chip, in registers and, past them, in LDS: it is
// read once, for the maximum, the sums and the gradient, which is all the memory
// traffic there has to be.  Wave 0 also deals with the teacher's entries.  What does
// not fit is read again for each pass.  q and q1 are written to every column first;
// then the columns of the teacher's entries and of the label, whose logits were
// fetched at the start, are written again with p and 1_y taken off.
//
// Measured (a large copy reaches 5.17 TB/s on the same card): 8192 x 50257 bf16 with 64
// entries, tau = 2 and labels 360 us, 4.6 TB/s; losses alone with 32 entries 151 us, 5.5 TB/s
// of reads; 4096 x 128256 bf16 451 us, 4.7 TB/s; 1001 x 100277 float32 with 100 entries, tau
// = 1.5 and labels 214 us, 3.8 TB/s (four rounds of one row a CU, and the last 9% of it);
// 128 x 1000 float32 6 us, one load's latency and three barriers.
#include "distill.h"
#include "ns_common.h"
#include "ops_common.h"

namespace malt {

namespace {

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

template <class T>
struct Vec;
template <>
struct Vec<float> {
  static constexpr int N = 4;
  static constexpr uint32_t NEG_INF = 0xff800000u;
  __device__ static void open(op_u32x4 r, float (&f)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = __uint_as_float(r[e]);
  }
  __device__ static op_u32x4 close(const float (&f)[4]) {
    op_u32x4 r;
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = __float_as_uint(f[e]);
    return r;
  }
};
template <>
struct Vec<bf16_t> {
  static constexpr int N = 8;
  static constexpr uint32_t NEG_INF = 0xff80ff80u;
  __device__ static void open(op_u32x4 r, float (&f)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      f[2 * e] = bf16_lo(r[e]);
      f[2 * e + 1] = bf16_hi(r[e]);
    }
  }
  __device__ static op_u32x4 close(const float (&f)[8]) {
    op_u32x4 r;
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = pack_bf16x2(f[2 * e], f[2 * e + 1]);
    return r;
  }
};

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor(v, off, 64));
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
  return v;
}

// Which normalisers a call needs.
enum Mode {
  ONE,      // alpha = 0, alpha = 1 or tau = 1: a single one
  TWO,      // those of tau and of 1
  SQUARE    // tau = 2: exp(z) is the square of exp(z / 2), one exponential serves both
};

// NT threads hold H vectors of 16 bytes each in registers and L in LDS.  STEP: the
// gradient is written.
template <class T, int NT, int H, int L, int MODE, bool STEP, int WPE>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(WPE)))
void distill_kernel(DistillArgs a) {
  using V = Vec<T>;
  constexpr int N = V::N, NW = NT / 64;
  __shared__ float red_max[NW], red_tau[NW], red_one[NW];
  __shared__ float ent_off[DISTILL_MAX_TOP + 1], ent_z[DISTILL_MAX_TOP + 1];   // what a column is lowered by; its logit
  __shared__ int32_t ent_id[DISTILL_MAX_TOP + 1];                              // -1: no entry
  __shared__ op_u32x4 kept[L > 0 ? L * NT : 1];   // vector i of thread t at i NT + t
  __shared__ float flags[2];                                                   // the row has a teacher, a label

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t row = blockIdx.x;
  const T* z = static_cast<const T*>(a.logits) + row * a.ld;
  const int vocab = (int)a.vocab;
  // Columns before the first 16-byte boundary and after the last: one a thread.
  // (Vectors at whatever address are as right, but their stores, which then begin
  // and end within memory's lines, took the bf16 step from 380 to 470 us.)
  const int ahead = (int)((16 - (reinterpret_cast<uintptr_t>(z) & 15)) & 15) / (int)sizeof(T);
  const int head = ahead < vocab ? ahead : vocab;
  const int nvec = (vocab - head) / N;
  const int tail0 = head + nvec * N;
  const bool edge = tid < head + (vocab - tail0);
  const int edge_col = tid < head ? tid : tail0 + (tid - head);
  const MALT_GLOBAL op_u32x4* body = reinterpret_cast<const MALT_GLOBAL op_u32x4*>(gptr(z) + head);

  // Teacher and label are wave 0's.  Their first loads go out before the row's,
  // and the logits at their columns right behind it, so that nobody waits for
  // a chain of loads; the arithmetic comes after the row's sums.
  const char* const ids = static_cast<const char*>(a.top_ids) + row * a.id_ld * (a.wide_ids ? 8 : 4);
  auto entry = [&](int j, int32_t& id, float& v) {
    const int64_t i = load_id(ids, a.wide_ids, j);
    v = a.top_f32 ? gptr(static_cast<const float*>(a.top) + row * a.top_ld)[j]
                  : to_f32(gptr(static_cast<const bf16_t*>(a.top) + row * a.top_ld)[j]);
    id = i >= 0 && i < vocab ? (int32_t)i : -1;
  };
  int32_t id0 = -1, label = -1;
  float top0 = -INFINITY, z0 = 0.f, z_label = 0.f;
  if (wave == 0) {
    if (lane < a.n_top) entry(lane, id0, top0);
    if (a.labels) {
      const int64_t y = load_id(a.labels, a.wide_labels, row * a.label_stride);
      label = y >= 0 && y < vocab ? (int32_t)y : -1;
    }
  }

  op_u32x4 held[H];
#pragma unroll
  for (int i = 0; i < H; ++i) {
    held[i] = op_u32x4{V::NEG_INF, V::NEG_INF, V::NEG_INF, V::NEG_INF};
    if (tid + i * NT < nvec) held[i] = body[tid + i * NT];
  }
  // Vectors H NT + i NT + tid go straight to LDS, each wave's into its own part of it.
#pragma unroll
  for (int i = 0; i < L; ++i) {
    const int q0 = (H + i) * NT + wave * 64;
    if (q0 + lane < nvec) ns::dma16(ns::buf_rsrc(z + head + (int64_t)q0 * N), 16 * lane, 0, ns::lds_u32(kept + i * NT + wave * 64));
  }
  const float edge_z = edge ? to_f32(gptr(z)[edge_col]) : -INFINITY;
  // f(q, its values) for the vectors of this thread that LDS holds, and those read again.
  auto beyond = [&](auto&& each) {
#pragma unroll 1
    for (int i = 0; i < L; ++i) {
      const int q = (H + i) * NT + tid;
      if (q < nvec) {
        float f[N];
        V::open(kept[i * NT + tid], f);
        each(q, f);
      }
    }
    for (int q = (H + L) * NT + tid; q < nvec; q += NT) {
      float f[N];
      V::open(body[q], f);
      each(q, f);
    }
  };
  // The held bits are opened anew in each pass: kept open they would take twice the registers.
  auto close_held = [&]() {
#pragma unroll
    for (int i = 0; i < H; ++i) asm volatile("" : "+v"(held[i]));
  };

  if (wave == 0) {
    if (id0 >= 0) z0 = to_f32(gptr(z)[id0]);
    if (label >= 0) z_label = to_f32(gptr(z)[label]);
    // An entry without an id or with a logit of -inf has no mass.
    bool some = id0 >= 0 && top0 != -INFINITY;
    if (lane < a.n_top) {
      ent_id[lane] = id0;
      ent_off[lane] = id0 >= 0 ? top0 : -INFINITY;
    }
    for (int j = lane + 64; j < a.n_top; j += 64) {
      int32_t id;
      float v;
      entry(j, id, v);
      ent_id[j] = id;
      ent_off[j] = id >= 0 ? v : -INFINITY;
      ent_z[j] = id >= 0 ? to_f32(gptr(z)[id]) : 0.f;
      some |= id >= 0 && v != -INFINITY;
    }
    const bool teacher = __any(some);
    if (lane == 0) {
      flags[0] = teacher ? 1.f : 0.f;
      flags[1] = label >= 0 ? 1.f : 0.f;
      ent_id[a.n_top] = label;
    }
  }

  // ------------------------------------------------------------------ maximum
  float m = edge_z;
#pragma unroll
  for (int i = 0; i < H; ++i) {
    float f[N];
    V::open(held[i], f);
#pragma unroll
    for (int e = 0; e < N; ++e) m = fmaxf(m, f[e]);
  }
  if constexpr (L > 0) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // LDS holds this wave's vectors
  beyond([&](int, const float (&f)[N]) {
#pragma unroll
    for (int e = 0; e < N; ++e) m = fmaxf(m, f[e]);
  });
  m = wave_max(m);
  if (lane == 0) red_max[wave] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NW; ++w) m = fmaxf(m, red_max[w]);
  close_held();

  // --------------------------------------------------------------------- sums
  // exp((z - m) / t) = 2^(z c - m c), c = log2(e) / t; the same rounded m c goes
  // into the sums, the loss and the gradient, so it cancels.
  // The maximum's own exponent is then what m c was rounded by, below 2^5 while
  // |m c| <= 2^29.  Beyond that (logits of 10^8, a row of the type's lowest value) a
  // second distinct logit is at least 2^5 below the maximum in the exponent, 10^-10 of
  // it: there c is any power of two large enough that only maxima count, and m c exact.
  const float inv_tau = 1.f / a.tau;
  const float r_tau = MODE != ONE || a.alpha < 1.f ? LOG2E * inv_tau : LOG2E, r_one = MODE == ONE ? r_tau : LOG2E;
  auto usable = [&](float c) {
    if (!(fabsf(m) * c > 0x1p29f && fabsf(m) < INFINITY)) return c;
    return __uint_as_float(__float_as_uint(0x1p41f / fabsf(m)) & 0x7f800000u);
  };
  // Squares share the rounding of m c_tau, so c_one is twice c_tau whatever that is (r_one = 2 r_tau there).
  const float c_tau = usable(r_tau), c_one = MODE == SQUARE ? 2.f * c_tau : usable(r_one);
  const float mc_tau = m * c_tau, mc_one = MODE == SQUARE ? 2.f * mc_tau : m * c_one;
  float s_tau = 0.f, s_one = 0.f;
  auto add = [&](float f) {
    const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(f, c_tau, -mc_tau));
    s_tau += x;
    if constexpr (MODE == TWO) s_one += __builtin_amdgcn_exp2f(__builtin_fmaf(f, c_one, -mc_one));
    if constexpr (MODE == SQUARE) s_one = __builtin_fmaf(x, x, s_one);
  };
  add(edge_z);
#pragma unroll
  for (int i = 0; i < H; ++i) {
    float f[N];
    V::open(held[i], f);
#pragma unroll
    for (int e = 0; e < N; ++e) add(f[e]);
  }
  beyond([&](int, const float (&f)[N]) {
#pragma unroll
    for (int e = 0; e < N; ++e) add(f[e]);
  });
  s_tau = wave_sum(s_tau);
  if constexpr (MODE != ONE) s_one = wave_sum(s_one);
  if (lane == 0) {
    red_tau[wave] = s_tau;
    if constexpr (MODE != ONE) red_one[wave] = s_one;
  }
  // Past the barrier a gradient written in place replaces the logits.  Wave 0 may not have used its
  // entries' and its label's logits yet, which other waves' columns hold: its loads have to have arrived.
  if constexpr (STEP) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  s_tau = s_one = 0.f;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    s_tau += red_tau[w];
    if constexpr (MODE != ONE) s_one += red_one[w];
  }
  if constexpr (MODE == ONE) s_one = s_tau;
  close_held();
  const bool use_teacher = flags[0] != 0.f && a.alpha < 1.f, use_label = flags[1] != 0.f && a.alpha > 0.f;

  // ----------------------------------------------------------- loss (wave 0)
  if (wave == 0) {
    const float log_tau = log2f(s_tau), log_one = log2f(s_one);
    auto log2_of = [&](float f, float r, float c, float mc) { return r == c ? __builtin_fmaf(f, c, -mc) : (f - m) * r; };
    float top = -INFINITY, sum = 0.f, kl = 0.f;
    for (int j = lane; j < a.n_top; j += 64) top = fmaxf(top, ent_off[j]);
    top = wave_max(top);
    const float c_top = LOG2E * inv_tau;
    for (int j = lane; j < a.n_top; j += 64)
      if (ent_off[j] != -INFINITY) sum += exp2f((ent_off[j] - top) * c_top);
    const float log_sum = log2f(wave_sum(sum));
    if (lane < a.n_top) ent_z[lane] = z0;
    for (int j = lane; j < a.n_top; j += 64) {
      float p = 0.f;
      if (ent_off[j] != -INFINITY) {
        const float lp = (ent_off[j] - top) * c_top - log_sum;   // log2 p
        p = exp2f(lp);
        const float lq = log2_of(ent_z[j], r_tau, c_tau, mc_tau) - log_tau;
        if (p != 0.f) kl += p * (lp - lq);
      }
      ent_off[j] = (1.f - a.alpha) * a.tau * p;
    }
    kl = wave_sum(kl);
    if (lane == 0) {
      ent_off[a.n_top] = a.alpha;
      ent_z[a.n_top] = z_label;
      float loss = 0.f;
      if (use_teacher) loss += (1.f - a.alpha) * a.tau * a.tau * LN2 * kl;
      if (use_label) loss += a.alpha * LN2 * (log_one - log2_of(z_label, r_one, c_one, mc_one));
      if (a.losses) gptr(a.losses)[row] = loss;
    }
  }

  // ----------------------------------------------------------------- gradient
  if constexpr (STEP) {
    const float w = a.weight ? gptr(a.weight)[row * a.weight_stride] : a.weight_value;
    T* d = static_cast<T*>(a.dlogits) + row * a.dld;
    MALT_GLOBAL T* const dg = gptr(d);
    auto put = [&](int q, const float (&f)[N]) {
      *reinterpret_cast<MALT_GLOBAL op_u32x4_any*>(dg + head + (int64_t)q * N) = V::close(f);
    };
    // A row without weight, or without teacher and label, has no gradient, whatever its logits hold.
    if (w == 0.f || !(use_teacher || use_label)) {
      const float none[N] = {};
      for (int q = tid; q < nvec; q += NT) put(q, none);
      if (edge) dg[edge_col] = from_f32<T>(0.f);
      return;
    }
    // q = exp(..) / sum: the coefficient of each exponential.
    const float w_tau = use_teacher ? w * (1.f - a.alpha) * a.tau : 0.f, w_one = use_label ? w * a.alpha : 0.f;
    const float k_tau = MODE == ONE ? (w_tau + w_one) / s_tau : w_tau / s_tau, k_one = w_one / s_one;
    auto grad = [&](float f) {
      const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(f, c_tau, -mc_tau));
      if constexpr (MODE == TWO)
        return __builtin_fmaf(k_tau, x, k_one * __builtin_amdgcn_exp2f(__builtin_fmaf(f, c_one, -mc_one)));
      if constexpr (MODE == SQUARE) return x * __builtin_fmaf(k_one, x, k_tau);
      return k_tau * x;
    };
#pragma unroll
    for (int i = 0; i < H; ++i)
      if (tid + i * NT < nvec) {
        float f[N];
        V::open(held[i], f);
#pragma unroll
        for (int e = 0; e < N; ++e) f[e] = grad(f[e]);
        put(tid + i * NT, f);
      }
    beyond([&](int q, const float (&f)[N]) {
      float g[N];
#pragma unroll
      for (int e = 0; e < N; ++e) g[e] = grad(f[e]);
      put(q, g);
    });
    if (edge) dg[edge_col] = from_f32<T>(grad(edge_z));
    // Every store above has reached memory before a column is written again.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    const int n_ent = a.n_top + 1;
    for (int j = tid; j < n_ent; j += NT) {
      const int id = ent_id[j];
      if (id < 0) continue;
      float off = 0.f;   // an id named twice is lowered by both, and both write the same value
      for (int i = 0; i < n_ent; ++i)
        if (ent_id[i] == id && (i < a.n_top ? use_teacher : use_label)) off += ent_off[i];
      dg[id] = from_f32<T>(grad(ent_z[j]) - w * off);
    }
  }
}

template <class T, int NT, int H, int L, int WPE, int MODE>
void launch_mode(const DistillArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)a.rows), threads(NT);
  if (a.dlogits) hipLaunchKernelGGL((distill_kernel<T, NT, H, L, MODE, true, WPE>), grid, threads, 0, s, a);
  else hipLaunchKernelGGL((distill_kernel<T, NT, H, L, MODE, false, WPE>), grid, threads, 0, s, a);
}

template <class T, int NT, int H, int L, int WPE>
void launch_held(const DistillArgs& a, hipStream_t s) {
  if (a.alpha == 0.f || a.alpha == 1.f || a.tau == 1.f) launch_mode<T, NT, H, L, WPE, ONE>(a, s);
  else if (a.tau == 2.f) launch_mode<T, NT, H, L, WPE, SQUARE>(a, s);
  else launch_mode<T, NT, H, L, WPE, TWO>(a, s);
}

template <class T>
void launch_typed(const DistillArgs& a, hipStream_t s) {
  const int64_t nvec = a.vocab / Vec<T>::N;
  // Threads, vectors a thread holds in registers and in LDS, and the waves a SIMD (of
  // which four are a CU) that this leaves room for: as many rows a CU as fit, since one
  // row's loads go on during another's arithmetic and stores.
  // 8192 rows: 1000 float32 columns 26 us with one vector a thread, 27 with four; 4000 and
  // 8000 bf16 46 and 50 with four, 74 and 94 with 512 threads; 20001 bf16 146 with seven,
  // 149 four rows a CU.
  if (nvec <= 256) launch_held<T, 256, 1, 0, 8>(a, s);
  else if (nvec <= 256 * 4) launch_held<T, 256, 4, 0, 6>(a, s);
  else if (nvec <= 512 * 7) launch_held<T, 512, 7, 0, 6>(a, s);
  // Four rows a CU.  512 threads and three rows: step above 348 us, with tau = 1.5 373 (not
  // 367), losses alone 165 (not 151); registers alone, two rows: 369, 404 and 165.
  else if (nvec <= 256 * 25) launch_held<T, 256, 19, 6, 4>(a, s);
  // Two rows a CU.  Past what they hold (16384 vectors), reading the rest of a row again
  // costs less than one row a CU (1024 threads) while it is under a fifth: 4096 x 151936
  // bf16 566 and 608 us, 2048 x 88000 float32 351 and 313.  Without LDS 128256 columns of
  // bf16 took 523 us, not 451.
  else if (nvec <= 512 * 40) launch_held<T, 512, 24, 8, 4>(a, s);
  else launch_held<T, 1024, 24, 9, 4>(a, s);
}

}  // namespace

hipError_t launch_distill(const DistillArgs& a, bool f32, hipStream_t s) {
  if (f32) launch_typed<float>(a, s);
  else launch_typed<bf16_t>(a, s);
  return hipGetLastError();
}

}  // namespace malt
