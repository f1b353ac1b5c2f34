// Product of two 8-bit operands, out (M x N) (+)= A (M x K) B (N x K)^T, each with
// a power-of-two scale for every 128 values along K (see block_fp8.h), on
// the matrix cores, in one of two ways by the type of the result:
//
// bf16: v_mfma_scale_f32_16x16x128_f8f6f4 contracts a whole block and applies both
//   scales to it, so the scales cost no arithmetic.  It adds the products of 8
//   values with 14 bits below the largest of them, and these sums in 32 bits:
//   measured, results are 1e-5 to 6e-5 of their norm off, a thirtieth of what
//   rounding them to bf16 (1.7e-3) costs.
// float32: that is not enough for sums that are kept in 32 bits, so the values
//   are widened to bf16 on their way from LDS, scale included (both exact), and
//   v_mfma_f32_16x16x32_bf16, whose sums are off by 1e-8 to 1e-7, multiplies them
//   at half the rate.
//
// Tiled kernels: an output tile per workgroup; stages of one block (128 k, 128
// bytes a row) go straight from global memory into a two-slot LDS ring.  Which k
// a lane's 32 bytes are does not matter as long as both operands agree, since
// the block has one scale: a lane takes the 16-byte chunks g and g + 4 of its
// row (g = lane / 16), which hit 16 distinct groups of banks.  The instruction's
// first operand is B, so that a lane ends up with four consecutive columns.
#include <type_traits>

#include "block_fp8.h"
#include "ns_common.h"
#include "ops_common.h"

namespace malt {

namespace {

using ns::bf16x8;
using ns::buf_rsrc;
using ns::dma16;
using ns::f32x4;
using ns::i32x4;
using ns::lds_u32;
typedef int i32x8 __attribute__((ext_vector_type(8)));

// 4 bytes a lane into LDS, as dma16.
__device__ __forceinline__ void dma4(const i32x4& rsrc, uint32_t voff, uint32_t soff, uint32_t lds_addr) {
  asm volatile("s_nop 0\n\tbuffer_load_dword %0, %1, %2 offen lds"
               :
               : "v"(voff), "s"(rsrc), "s"(soff), "{m0}"(lds_addr)
               : "memory");
}

// c += (2^sb B) (2^sa A)^T of one block; byte OB / OA of the scale registers counts.
template <int OB, int OA>
__device__ __forceinline__ f32x4 mma(i32x8 b, i32x8 a, f32x4 c, int sb, int sa) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, c, 0, 0, OB, sb, OA, sa);
}
__device__ __forceinline__ f32x4 mma_sel(i32x8 b, i32x8 a, f32x4 c, int sb, int ob, int sa, int oa) {
  // ob, oa are constants after unrolling
  switch (ob * 4 + oa) {
#define MALT_SEL(x, y) case x * 4 + y: return mma<x, y>(b, a, c, sb, sa);
    MALT_SEL(0, 0) MALT_SEL(0, 1) MALT_SEL(0, 2) MALT_SEL(0, 3)
    MALT_SEL(1, 0) MALT_SEL(1, 1) MALT_SEL(1, 2) MALT_SEL(1, 3)
    MALT_SEL(2, 0) MALT_SEL(2, 1) MALT_SEL(2, 2) MALT_SEL(2, 3)
    MALT_SEL(3, 0) MALT_SEL(3, 1) MALT_SEL(3, 2) default: return mma<3, 3>(b, a, c, sb, sa);
#undef MALT_SEL
  }
}

// TM x TN tile, WM x WN waves of SM x SN each.
template <int TM_, int TN_, int WM_, int WN_, int WPE_>
struct MmGeom {
  static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_, WPE = WPE_;
  static constexpr int NW = WM * WN, NT = 64 * NW;
  static constexpr int SM = TM / WM, SN = TN / WN;
  static constexpr int MB = SM / 16, NB = SN / 16;           // 16-row blocks of a wave
  static constexpr int A_BYTES = TM * QB, B_BYTES = TN * QB; // one stage of each operand
  static constexpr int SLOT = A_BYTES + B_BYTES + TM + TN;   // and its scales
  static constexpr int A_LOADS = TM / 8, LOADS = (TM + TN) / 8 / NW;
  static_assert(LOADS * NW * 8 == TM + TN && A_LOADS % NW == 0, "loads split evenly over the waves");
  static_assert(SN <= 64 && 64 % SN == 0 && SM <= 128 && 128 % SM == 0, "a wave's scales lie in one group");
  static_assert(MB % 4 == 0, "row blocks are taken in pairs, an even number of times");
  static_assert(SLOT % 16 == 0, "slots are aligned");
};

__device__ __forceinline__ int swz(int row, int chunk) { return row * QB + ((chunk ^ ((row >> 1) & 7)) << 4); }

// Eight 8-bit values (two dwords) times 2^e as bf16, exactly; `scale` is 2^e.
__device__ __forceinline__ bf16x8 widen(int lo, int hi, float scale) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)lo, scale, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)lo, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)hi, scale, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)hi, scale, true);
  return bf16x8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}
// The power of two of exponent byte i of a scale register.
__device__ __forceinline__ float scale_of(int bytes, int i) {
  return __uint_as_float((((uint32_t)bytes >> (8 * i)) & 0xffu) << 23);
}

template <class G, bool BLOCKS, bool WIDE, class TO>
__global__ __launch_bounds__(G::NT) __attribute__((amdgpu_waves_per_eu(G::WPE, G::WPE)))
void block_matmul_kernel(BlockMatmulArgs g) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  constexpr int MB = G::MB, NB = G::NB;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / G::WN, wn = wave % G::WN;
  const int KT = (int)((g.k + QB - 1) / QB);
  const int64_t kp = (int64_t)KT * QB;
  const int64_t tn = (g.n + G::TN - 1) / G::TN, tm = (g.m + G::TM - 1) / G::TM;
  // Each XCD (block index mod 8) takes a run of consecutive tiles, column tiles of
  // a row tile first, so that the operands they share stay in its L2.
  const int64_t tiles = tm * tn, per = (tiles + 7) / 8;
  const int64_t tile = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if ((int64_t)(blockIdx.x >> 3) >= per || tile >= tiles) return;
  const int64_t m0 = tile / tn * G::TM, n0 = tile % tn * G::TN;

  const i32x4 rs_a = buf_rsrc(g.a + m0 * kp), rs_b = buf_rsrc(g.b + n0 * kp);
  const int64_t sa_pitch = q_scale_rows(g.m), sb_pitch = q_scale_rows(g.n);
  const i32x4 rs_sa = buf_rsrc(g.a_scales + m0), rs_sb = buf_rsrc(g.b_scales + n0);
  uint32_t voff[G::LOADS];
  int dst[G::LOADS];
#pragma unroll
  for (int q = 0; q < G::LOADS; ++q) {
    // Load l covers 8 rows of A (l < A_LOADS) or B; rows past the operand's end
    // repeat its last one, whose products are not stored.
    const int l = wave + q * G::NW;
    const bool is_a = q < G::A_LOADS / G::NW;
    const int row = 8 * (is_a ? l : l - G::A_LOADS) + (lane >> 3);
    const int64_t left = (is_a ? g.m - m0 : g.n - n0) - 1;
    const int src = row < left ? row : (int)left;
    voff[q] = (uint32_t)(src * kp) + (((lane & 7) ^ ((row >> 1) & 7)) << 4);
    dst[q] = l * 1024;
  }
  // Loads a wave has in flight for one stage: its share and, of two waves, the scales.
  const int in_flight = G::LOADS + (wave == 0 || (!BLOCKS && wave == 1) ? 1 : 0);
  const uint32_t lds0 = lds_u32(lds);
  auto issue = [&](int kt) {
    const uint32_t at = lds0 + (kt & 1) * G::SLOT, soff = (uint32_t)kt * QB;
#pragma unroll
    for (int q = 0; q < G::LOADS; ++q) dma16(q < G::A_LOADS / G::NW ? rs_a : rs_b, voff[q], soff, at + dst[q]);
    if (wave == 0 && lane < G::TM / 4) dma4(rs_sa, 4 * lane, (uint32_t)(kt * sa_pitch), at + G::A_BYTES + G::B_BYTES);
    if constexpr (!BLOCKS)
      if (wave == 1 && lane < G::TN / 4)
        dma4(rs_sb, 4 * lane, (uint32_t)(kt * sb_pitch), at + G::A_BYTES + G::B_BYTES + G::TM);
  };

  // Fragment offsets of a wave's first block; block b lies 16 rows (2 KB) further.
  int off_a[2], off_b[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    off_a[h] = swz(wm * G::SM + (lane & 15), (lane >> 4) + 4 * h);
    off_b[h] = G::A_BYTES + swz(wn * G::SN + (lane & 15), (lane >> 4) + 4 * h);
  }
  // Scales: 8 bytes a lane for each 128 rows; a wave's blocks start at byte (rows / 16) % 8.
  const int off_sa = G::A_BYTES + G::B_BYTES + (wm * G::SM) / 128 * 128 + 8 * (lane & 15) + (wm * G::SM) % 128 / 16;
  const int off_sb = G::A_BYTES + G::B_BYTES + G::TM + (wn * G::SN) / 128 * 128 + 8 * (lane & 15) + (wn * G::SN) % 128 / 16;
  // A weight's scales: lane l holds the one of block kt0 + l of the contraction.
  const uint8_t* const wscale = g.b_scales + (n0 + wn * G::SN) / QB * g.b_row_stride;

  f32x4 acc[NB][MB];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int a = 0; a < MB; ++a) acc[b][a] = f32x4{0.f, 0.f, 0.f, 0.f};

  // Fragments of one row block: the two chunks of a lane.
  auto frag = [&](const char* st, const int (&off)[2], int block) {
    const i32x4 lo = *reinterpret_cast<const i32x4*>(st + off[0] + block * 16 * QB);
    const i32x4 hi = *reinterpret_cast<const i32x4*>(st + off[1] + block * 16 * QB);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  constexpr int SAW = MB > 4 ? 2 : 1;   // registers of A's scales
  int wheld = 0;
  auto weight_scales = [&](int kt) {   // the next 64 blocks of the contraction
    if (n0 + wn * G::SN < g.n && kt + lane < KT) wheld = gptr(wscale)[(kt + lane) * g.b_col_stride];
  };
  auto read_scales = [&](const char* st, int kt, int (&sa)[SAW], int& sb) {
#pragma unroll
    for (int i = 0; i < SAW; ++i) sa[i] = *reinterpret_cast<const int*>(st + off_sa + 4 * i);
    if constexpr (BLOCKS) sb = __builtin_amdgcn_readlane(wheld, kt & 63);
    else sb = *reinterpret_cast<const int*>(st + off_sb);
  };

  // Two slots: at the barrier that closes stage kt, stage kt + 1 has landed and
  // every wave holds the rest of stage kt in registers, so its slot takes stage
  // kt + 2.
  if constexpr (BLOCKS) weight_scales(0);
  issue(0);
  if (KT > 1) issue(1);
  ns::wait_vm(KT > 1 ? in_flight : 0);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  int sa[SAW], sb;
  read_scales(lds, 0, sa, sb);
  auto next_stage = [&](int kt) {   // false: kt is the last one
    if (kt + 1 == KT) return false;
    if constexpr (BLOCKS)
      if (((kt + 1) & 63) == 0) weight_scales(kt + 1);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // this wave's reads of stage kt are done
    ns::wait_vm_c<0>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (kt + 2 < KT) issue(kt + 2);
    return true;
  };

  if constexpr (!WIDE) {
    constexpr int H = MB / 2;   // sub-steps of two row blocks of A against all of B
    i32x8 fa[2][2], fb[NB];
    fa[0][0] = frag(lds, off_a, 0);
    fa[0][1] = frag(lds, off_a, 1);
#pragma unroll
    for (int b = 0; b < NB; ++b) fb[b] = frag(lds, off_b, b);
    for (int kt = 0; kt < KT; ++kt) {
      const char* st = lds + (kt & 1) * G::SLOT;
      const char* nx = lds + (~kt & 1) * G::SLOT;
      int sa_next[SAW], sb_next = sb;
#pragma unroll
      for (int i = 0; i < SAW; ++i) sa_next[i] = sa[i];
#pragma unroll
      for (int h = 0; h < H; ++h) {
        bool more = true;
        if (h + 1 < H) {
          fa[(h + 1) & 1][0] = frag(st, off_a, 2 * h + 2);
          fa[(h + 1) & 1][1] = frag(st, off_a, 2 * h + 3);
        } else {
          more = next_stage(kt);
          if (more) {
            fa[0][0] = frag(nx, off_a, 0);
            fa[0][1] = frag(nx, off_a, 1);
            read_scales(nx, kt + 1, sa_next, sb_next);
          }
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int a = 2 * h + i;
            acc[b][a] = mma_sel(fb[b], fa[h & 1][i], acc[b][a], sb, BLOCKS ? 0 : b, sa[a / 4], a % 4);
          }
          if (h + 1 == H && more) fb[b] = frag(nx, off_b, b);   // its products of this stage are done
        }
        if (h + 1 < H) {
#pragma unroll
          for (int j = 0; j < 2 * NB; ++j) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      sb = sb_next;
#pragma unroll
      for (int i = 0; i < SAW; ++i) sa[i] = sa_next[i];
    }
  } else {
    for (int kt = 0; kt < KT; ++kt) {
      const char* st = lds + (kt & 1) * G::SLOT;
#pragma unroll
      for (int h = 0; h < 2; ++h) {   // the 16-byte chunks of a lane, 8 values a matrix instruction
        bf16x8 fb[NB][2];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          const i32x4 r = *reinterpret_cast<const i32x4*>(st + off_b[h] + b * 16 * QB);
          const float s = scale_of(sb, BLOCKS ? 0 : b);
          fb[b][0] = widen(r[0], r[1], s);
          fb[b][1] = widen(r[2], r[3], s);
        }
#pragma unroll
        for (int a = 0; a < MB; ++a) {
          const i32x4 r = *reinterpret_cast<const i32x4*>(st + off_a[h] + a * 16 * QB);
          const float s = scale_of(sa[a / 4], a % 4);
          const bf16x8 fa[2] = {widen(r[0], r[1], s), widen(r[2], r[3], s)};
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int b = 0; b < NB; ++b)
              acc[b][a] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[b][i], fa[i], acc[b][a], 0, 0, 0);
        }
      }
      if (next_stage(kt)) read_scales(lds + (~kt & 1) * G::SLOT, kt + 1, sa, sb);
    }
  }

  // acc[b][a][e] = out(m, n + e): m = block a, row lane % 16; n = block b, column 4 (lane / 16).
  const bool four = g.by_four;
#pragma unroll
  for (int a = 0; a < MB; ++a) {
    const int64_t m = m0 + wm * G::SM + 16 * a + (lane & 15);
    if (m >= g.m) continue;
    TO* row = static_cast<TO*>(g.out) + m * g.ldo;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int64_t n = n0 + wn * G::SN + 16 * b + 4 * (lane >> 4);
      if (four) {
        if (n < g.n) {
          op_f32x4 v = {acc[b][a][0], acc[b][a][1], acc[b][a][2], acc[b][a][3]};
          if (g.accumulate) {
            const op_f32x4 old = load4(row + n);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += old[e];
          }
          store4(row + n, v);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (n + e < g.n) {
            float v = acc[b][a][e];
            if (g.accumulate) v += to_f32(gptr(row)[n + e]);
            gptr(row)[n + e] = from_f32<TO>(v);
          }
      }
    }
  }
}

using Mm256 = MmGeom<256, 256, 2, 4, 2>;
using Mm128 = MmGeom<128, 128, 2, 2, 2>;

template <class G, bool BLOCKS, class TO>
hipError_t launch_tiled(const BlockMatmulArgs& a, hipStream_t s) {
  const auto kernel = &block_matmul_kernel<G, BLOCKS, std::is_same<TO, float>::value, TO>;
  constexpr int bytes = 2 * G::SLOT;
  // More LDS than the default limit: raised each time, for whichever device is current.
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                           hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e != hipSuccess) return e;
  const int64_t tiles = (a.m + G::TM - 1) / G::TM * ((a.n + G::TN - 1) / G::TN);
  hipLaunchKernelGGL(kernel, dim3((unsigned)((tiles + 7) / 8 * 8)), dim3(G::NT), bytes, s, a);
  return hipGetLastError();
}

template <bool BLOCKS, class TO>
hipError_t launch_typed(const BlockMatmulArgs& a, hipStream_t s) {
  const int64_t big = (a.m + 255) / 256 * ((a.n + 255) / 256);
  if (big >= 128) return launch_tiled<Mm256, BLOCKS, TO>(a, s);
  return launch_tiled<Mm128, BLOCKS, TO>(a, s);
}

}  // namespace

hipError_t launch_block_matmul(BlockMatmulArgs a, bool b_blocks, bool out_f32, hipStream_t s) {
  a.by_four = op_rows_by_four(a.out, out_f32 ? MALT_FLOAT32 : MALT_BFLOAT16, a.ldo, a.n);
  if (b_blocks) return out_f32 ? launch_typed<true, float>(a, s) : launch_typed<true, bf16_t>(a, s);
  return out_f32 ? launch_typed<false, float>(a, s) : launch_typed<false, bf16_t>(a, s);
}

}  // namespace malt
