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
//   are widened to bf16 on their way from LDS, scale included (both exact down to
//   bf16's smallest number, 2^-133), and v_mfma_f32_16x16x32_bf16, whose sums are
//   off by 1e-8 to 1e-7, multiplies them at half the rate.
//
// Bound by the matrix cores (and their power).  Measured, the library's products without
// block scales beside: 8192 x 5120 x 1280 bf16 73 us, 1.47 PFLOP/s (8-bit library 72);
// 8192 x 1280 x 5120 bf16 67 to 70 us, 1.5 PFLOP/s (57); 8192^3 bf16 2.41 to 2.44 PFLOP/s (2.63);
// 5120 x 1280 x 8192 float32 107 to 117 us, 0.92 to 1.0 PFLOP/s (bf16 library 102).
//
// Tiled kernels: an output tile per workgroup; stages of one block (128 k, 128
// bytes a row) go straight from global memory into a two-slot LDS ring.  Which k
// a lane's 32 bytes are does not matter as long as both operands agree, since
// the block has one scale: a lane takes the 16-byte chunks g and g + 4 of its
// row (g = lane / 16), which hit 16 distinct groups of banks.  The instruction's
// first operand is B, so that a lane ends up with four consecutive columns.
#include <atomic>
#include <type_traits>

#include "block_mma.h"
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

// 4 bytes a lane into LDS, as dma16.
__device__ __forceinline__ void dma4(const i32x4& rsrc, uint32_t voff, uint32_t soff, uint32_t lds_addr) {
  asm volatile("s_nop 0\n\tbuffer_load_dword %0, %1, %2 offen lds"
               :
               : "v"(voff), "s"(rsrc), "s"(soff), "{m0}"(lds_addr)
               : "memory");
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
  static_assert(SLOT % 16 == 0 && 2 * SLOT <= 160 * 1024, "slots are aligned, the ring fits");
};

__device__ __forceinline__ int swz(int row, int chunk) { return row * QB + ((chunk ^ ((row >> 1) & 7)) << 4); }

template <class G, bool BLOCKS, bool WIDE, bool SPLIT, class TO>
__global__ __launch_bounds__(G::NT) __attribute__((amdgpu_waves_per_eu(G::WPE, G::WPE)))
void block_matmul_kernel(BlockMatmulArgs g) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  constexpr int MB = G::MB, NB = G::NB;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / G::WN, wn = wave % G::WN;
  const int blocks_k = (int)((g.k + QB - 1) / QB);
  const int64_t kp = (int64_t)blocks_k * QB;
  // Part of the contraction: blocks k0 .. k0 + KT - 1.
  const int part = SPLIT ? blockIdx.y : 0, k0 = SPLIT ? (int)((int64_t)blocks_k * part / g.parts) : 0;
  const int KT = SPLIT ? (int)((int64_t)blocks_k * (part + 1) / g.parts) - k0 : blocks_k;
  const int64_t tn = (g.n + G::TN - 1) / G::TN, tm = (g.m + G::TM - 1) / G::TM;
  // Each XCD (block index mod 8) takes a run of consecutive tiles, column tiles of
  // a row tile first, so that the operands they share stay in its L2.
  const int64_t tiles = tm * tn, per = (tiles + 7) / 8;
  const int64_t tile = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if ((int64_t)(blockIdx.x >> 3) >= per || tile >= tiles) return;
  const int64_t m0 = tile / tn * G::TM, n0 = tile % tn * G::TN;

  const i32x4 rs_a = buf_rsrc(g.a + m0 * kp + (int64_t)k0 * QB), rs_b = buf_rsrc(g.b + n0 * kp + (int64_t)k0 * QB);
  const int64_t sa_pitch = q_scale_rows(g.m), sb_pitch = q_scale_rows(g.n);
  const i32x4 rs_sa = buf_rsrc(g.a_scales + m0 + k0 * sa_pitch), rs_sb = buf_rsrc(g.b_scales + n0 + k0 * sb_pitch);
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
  // A wave's loads of one stage: its share of the operands and one of scales, so
  // that every wave waits for the same count (several waves load the same scales
  // to the same place).
  constexpr int IN_FLIGHT = G::LOADS + 1;
  const bool b_wave = !BLOCKS && (wave & 1);
  const i32x4 rs_s = b_wave ? rs_sb : rs_sa;
  const int64_t s_pitch = b_wave ? sb_pitch : sa_pitch;
  const int s_lanes = (b_wave ? G::TN : G::TM) / 4, s_dst = G::A_BYTES + G::B_BYTES + (b_wave ? G::TM : 0);
  const uint32_t lds0 = lds_u32(lds);
  auto issue = [&](int kt) {
    const uint32_t at = lds0 + (kt & 1) * G::SLOT, soff = (uint32_t)kt * QB;
#pragma unroll
    for (int q = 0; q < G::LOADS; ++q) dma16(q < G::A_LOADS / G::NW ? rs_a : rs_b, voff[q], soff, at + dst[q]);
    if (lane < s_lanes) dma4(rs_s, 4 * lane, (uint32_t)(kt * s_pitch), at + s_dst);
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
  const uint8_t* const wscale = g.b_scales + (n0 + wn * G::SN) / QB * g.b_row_stride + k0 * g.b_col_stride;

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
  if (KT > 1) {
    issue(1);
    ns::wait_vm_c<IN_FLIGHT>();
  } else {
    ns::wait_vm_c<0>();
  }
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
    // Step s of a stage takes 16-byte chunk s / MB of a lane against row block
    // s % MB of A: two matrix instructions of 8 values for each block of B.  While
    // they run, the next step's values are widened and those of the step after
    // it are read; B's next chunk is widened in the last step of this one, block
    // by block as its products are issued.
    constexpr int S = 2 * MB;
    auto chunk = [&](const char* st, int off, int block) {
      return *reinterpret_cast<const i32x4*>(st + off + block * 16 * QB);
    };
    bf16x8 fa[2][2], fb[NB][2];
    i32x4 ra[2], rb[NB];
    auto open = [&](bf16x8 (&f)[2], const i32x4& r, float sc) {
      f[0] = widen(r[0], r[1], sc);
      f[1] = widen(r[2], r[3], sc);
    };
    open(fa[0], chunk(lds, off_a[0], 0), scale_of(sa[0], 0));
#pragma unroll
    for (int b = 0; b < NB; ++b) open(fb[b], chunk(lds, off_b[0], b), scale_of(sb, BLOCKS ? 0 : b));
    ra[1] = chunk(lds, off_a[0], 1);
    for (int kt = 0; kt < KT; ++kt) {
      const char* st = lds + (kt & 1) * G::SLOT;
      const char* nx = lds + (~kt & 1) * G::SLOT;
      int sa_next[SAW], sb_next = sb;
#pragma unroll
      for (int i = 0; i < SAW; ++i) sa_next[i] = sa[i];
      bool more = true;
#pragma unroll
      for (int q = 0; q < S; ++q) {
        const int h = q / MB, a = q % MB;
        if (q + 2 == S) {   // the last chunk read of this stage lies in registers
          more = next_stage(kt);
          if (more) read_scales(nx, kt + 1, sa_next, sb_next);
        }
        if (q + 2 < S) ra[q & 1] = chunk(st, off_a[(q + 2) / MB], (q + 2) % MB);
        else if (more) ra[q & 1] = chunk(nx, off_a[0], q + 2 - S);
        if (a == MB - 2) {
#pragma unroll
          for (int b = 0; b < NB; ++b)
            if (h == 0) rb[b] = chunk(st, off_b[1], b);
            else if (more) rb[b] = chunk(nx, off_b[0], b);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int b = 0; b < NB; ++b)
            acc[b][a] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[b][i], fa[q & 1][i], acc[b][a], 0, 0, 0);
        const int n = q + 1 < S ? q + 1 : 0;   // what is widened for
        const int* sn = q + 1 < S ? sa : sa_next;
        open(fa[n & 1], ra[n & 1], scale_of(sn[(n % MB) / 4], n % 4));
        if (a == MB - 1)
#pragma unroll
          for (int b = 0; b < NB; ++b) open(fb[b], rb[b], scale_of(h == 0 ? sb : sb_next, BLOCKS ? 0 : b));
        __builtin_amdgcn_sched_barrier(0);
      }
      sb = sb_next;
#pragma unroll
      for (int i = 0; i < SAW; ++i) sa[i] = sa_next[i];
    }
  }

  // acc[b][a][e] = out(m, n + e): m = block a, row lane % 16; n = block b, column 4 (lane / 16).
  if constexpr (SPLIT) {   // this part's sums, tile by tile, for block_sum_kernel
    float* p = g.partial + ((int64_t)part * tiles + tile) * (G::TM * G::TN);
#pragma unroll
    for (int a = 0; a < MB; ++a)
#pragma unroll
      for (int b = 0; b < NB; ++b)
        store4(p + (wm * G::SM + 16 * a + (lane & 15)) * G::TN + wn * G::SN + 16 * b + 4 * (lane >> 4), acc[b][a]);
    return;
  }
  // Two row blocks at a time go through a part of LDS of the wave's own and leave
  // it in whole rows of the wave's columns: 128 or 256 bytes a row, not pieces of 32.
  constexpr int PITCH = G::SN + 4, PASS = 32 * PITCH;   // floats
  static_assert(G::NW * PASS * 4 <= 2 * G::SLOT, "the copies fit the ring");
  float* const mine = reinterpret_cast<float*>(lds) + wave * PASS;
  __syncthreads();   // every wave is done reading the ring
#pragma unroll
  for (int p = 0; p < MB; p += 2) {
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int b = 0; b < NB; ++b)
        *reinterpret_cast<f32x4*>(mine + (16 * a + (lane & 15)) * PITCH + 16 * b + 4 * (lane >> 4)) = acc[b][p + a];
    constexpr int W = sizeof(TO) == 4 ? 4 : 8, PER = G::SN / W;   // columns a lane stores, lanes a row
#pragma unroll
    for (int i = 0; i < 32 * PER / 64; ++i) {
      const int r = (i * 64 + lane) / PER, c = (i * 64 + lane) % PER * W;
      const int64_t m = m0 + wm * G::SM + 16 * p + r, n = n0 + wn * G::SN + c;
      op_f32x4 v[W / 4];
#pragma unroll
      for (int e = 0; e < W / 4; ++e) v[e] = *reinterpret_cast<const f32x4*>(mine + r * PITCH + c + 4 * e);
      if (m >= g.m) continue;
      TO* row = static_cast<TO*>(g.out) + m * g.ldo;
      if (g.accumulate)
#pragma unroll
        for (int e = 0; e < W / 4; ++e) v[e] += row_load4(row, n + 4 * e, g.n);
      if constexpr (W == 8) {
        if (n + 8 <= g.n) {
          const op_u32x4 q = {pack_bf16x2(v[0].x, v[0].y), pack_bf16x2(v[0].z, v[0].w), pack_bf16x2(v[1].x, v[1].y),
                              pack_bf16x2(v[1].z, v[1].w)};
          *reinterpret_cast<MALT_GLOBAL op_u32x4_any*>(gptr(row) + n) = q;
          continue;
        }
      }
#pragma unroll
      for (int e = 0; e < W / 4; ++e) row_store4(row, n + 4 * e, g.n, v[e]);
    }
  }
}

// out (+)= the sum of the parts, in order; four columns a thread.
template <int TM, int TN, class TO>
__global__ __launch_bounds__(256) void block_sum_kernel(BlockMatmulArgs g) {
  const int64_t tn = (g.n + TN - 1) / TN, tm = (g.m + TM - 1) / TM;
  const int64_t row = (int64_t)blockIdx.y * (256 / (TN / 4)) + threadIdx.x / (TN / 4);
  const int64_t n = (int64_t)blockIdx.x * TN + threadIdx.x % (TN / 4) * 4;
  if (row >= g.m || n >= g.n) return;
  const float* p = g.partial + (row / TM * tn + blockIdx.x) * (TM * TN) + row % TM * TN + threadIdx.x % (TN / 4) * 4;
  op_f32x4 v = load4(p);
  for (int i = 1; i < g.parts; ++i) {
    const op_f32x4 x = load4(p + i * (tm * tn * (TM * TN)));
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += x[e];
  }
  TO* out = static_cast<TO*>(g.out) + row * g.ldo;
  if (g.accumulate) v += row_load4(out, n, g.n);
  row_store4(out, n, g.n, v);
}

// Other shapes that were measured and are slower: 128 x 256 tiles, and a fixed interleaving of
// the widened loop's conversions with its matrix instructions.
// Rings of two slots; with three or four, and one workgroup a CU, the 128-tile ran
// 5 to 10% slower: what a stage of few workgroups waits for is LDS, not memory.
using Mm256 = MmGeom<256, 256, 2, 4, 2>;
using Mm128 = MmGeom<128, 128, 2, 2, 2>;   // two workgroups a CU

template <class G, bool BLOCKS, bool SPLIT, class TO>
hipError_t launch_tiled(const BlockMatmulArgs& a, hipStream_t s) {
  const auto kernel = &block_matmul_kernel<G, BLOCKS, std::is_same<TO, float>::value, SPLIT, TO>;
  constexpr int bytes = 2 * G::SLOT;
  // More LDS than the default limit: raised once for each device.
  static std::atomic<uint64_t> raised{0};
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = uint64_t(1) << (dev & 63);
  if (dev > 63 || !(raised.load(std::memory_order_relaxed) & bit)) {
    e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
    raised.fetch_or(bit, std::memory_order_relaxed);
  }
  const int64_t tn = (a.n + G::TN - 1) / G::TN, tiles = (a.m + G::TM - 1) / G::TM * tn;
  hipLaunchKernelGGL(kernel, dim3((unsigned)((tiles + 7) / 8 * 8), (unsigned)a.parts), dim3(G::NT), bytes, s, a);
  if constexpr (SPLIT) {
    constexpr int rows = 256 / (G::TN / 4);
    hipLaunchKernelGGL((block_sum_kernel<G::TM, G::TN, TO>), dim3((unsigned)tn, (unsigned)((a.m + rows - 1) / rows)),
                       dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

template <bool BLOCKS, class TO>
hipError_t launch_typed(const BlockMatmulArgs& a, bool big, hipStream_t s) {
  if (big) return launch_tiled<Mm256, BLOCKS, false, TO>(a, s);
  if (a.parts == 1) return launch_tiled<Mm128, BLOCKS, false, TO>(a, s);
  return launch_tiled<Mm128, BLOCKS, true, TO>(a, s);
}

}  // namespace

// The tile and the parts of the contraction that the estimate below finds fastest.
// Microseconds, fitted to runs over M, N, K from 16 to 8192 (within 20%; in
// brackets the float32 result): a stage of 128 k takes 1.7 [2.4 to 3.2] on a
// 256-tile; on 128-tiles 0.62 [1.02] while there is one a CU, 1.15 [1.9] with two; a
// tile's start and end 9 and 4; joining parts 6 and their bytes at 4 TB/s.
// Measured: 8192 x 1280 x 1280 (160 big tiles) 26 on 256-tiles, 23 on 128-tiles;
// 4096^3 69 and 76; 128 x 128 x 8192 37 in one part, 15 in 16; 1280 x 1280 x 8192
// 43 in one, 41 in two; 1000 x 1501 x 901 12 in one, 18 in two.
BlockMatmulPlan block_matmul_plan(int64_t m, int64_t n, int64_t k, bool out_f32) {
  const int64_t kt = (k + QB - 1) / QB;
  const int64_t big = (m + 255) / 256 * ((n + 255) / 256), small = (m + 127) / 128 * ((n + 127) / 128);
  const double t_big = out_f32 ? 2.4 + 0.8 * (big < 256 ? big / 256.0 : 1.0) : 1.7;
  const double t_one = out_f32 ? 1.02 : 0.62, t_two = out_f32 ? 1.9 : 1.15;
  BlockMatmulPlan best = {true, 1, 0};
  double least = double((big + 255) / 256) * (kt * t_big + 9);
  for (int32_t parts = 1; parts <= 16 && parts <= kt && (parts == 1 || small * parts <= 512); parts += parts < 4 ? 1 : parts < 8 ? 2 : 4) {
    const int64_t full = small * parts / 512, rest = small * parts % 512, stages = (kt + parts - 1) / parts;
    double t = full * (stages * t_two + 4);
    if (rest > 0) t += stages * (t_one + (t_two - t_one) * (rest > 256 ? (rest - 256) / 256.0 : 0.0)) + 4;
    const size_t bytes = parts > 1 ? size_t(parts) * small * (128 * 128 * 4) : 0;
    if (parts > 1) t += 6 + 2 * bytes / 4e6;
    if (t < least) {
      least = t;
      best = {false, parts, bytes};
    }
  }
  return best;
}

hipError_t launch_block_matmul(BlockMatmulArgs a, bool b_blocks, bool out_f32, hipStream_t s) {
  const BlockMatmulPlan p = block_matmul_plan(a.m, a.n, a.k, out_f32);
  a.parts = p.parts;
  if (b_blocks) return out_f32 ? launch_typed<true, float>(a, p.big, s) : launch_typed<true, bf16_t>(a, p.big, s);
  return out_f32 ? launch_typed<false, float>(a, p.big, s) : launch_typed<false, bf16_t>(a, p.big, s);
}

}  // namespace malt
