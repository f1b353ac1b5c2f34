// The tiled products of a linear head's cross entropy:
//
//   first pass    z = x W^T, a tile's largest and sum of 2^(z log2 e) for each row
//   second pass   z again, dz = w (softmax(z) - 1_y), for a piece of the vocabulary
//   gradients     dx += dz W and dW = dz^T x for that piece, in one launch
//
// Bound by the matrix cores: 2 M V K operations a product, four products with both gradients.
// The logits are formed twice because M x V of them in 32 bits would cost as much to write and
// read (twice 4 bytes a logit) as the K products that make one.
//
// 8192 x 50257 x 1280 in bf16, 1.05 T operations a product: first pass 950 us (1110 TFLOP/s; the library's
// product that writes its logits: 939), second 1170 in two pieces, gradients 1700 (1240 TFLOP/s; the library's: 2450).
// A stage of 64 takes a tile 1.40 to 1.46 us with random values and 1.23 with zeros: the power limit.  What the
// second pass takes longer is its writing: a tile's dz, 256 KB both ways, 18 us of 47, while no matrix
// instruction runs on that CU.
//
// A workgroup of eight waves makes one 256 x 256 tile, the pipeline of the Newton-Schulz
// update (ns_common.h): stages of 64 contracted values go straight to LDS, two slots deep.  Where
// there are few tiles or few stages in each, tiles are of 128 x 128, two on a CU, which read twice the LDS for a
// product but leave no CU out and work on one's stages during the other's epilogue: 300 x 1000 x 64 76 -> 37 us a
// step, 200 x 8000 x 512 in float32 168 -> 89, 500 x 2000 x 2000 162 -> 80 (the rules are in model_api.hip).  Both
// sides of every product lie with the contraction along their rows: x and W are transposed once for
// the gradients, dz is written both ways.  (Transposed LDS reads instead: 1.84 us a stage, for one side or
// both; rows of 32 KB apart: 1.70, with a pitch that is no power of two 1.58.)
//
// float32 operands are planes whose sum they are, and a product of two runs as a contraction over
// the pairs of planes that matter, small ones first: float32 sums of exact products.
//   logits: two float16 planes under a power of two for each row, 22 bits; three pairs (low by low is
//     below 2^-22 of the whole, as the planes' own rounding).
//   gradients: three bf16 planes, all 24 bits; six pairs (middle by low and low by low are below
//     2^-24).  dz has no float16 planes: along a row its values are below the label's, so that dx could take
//     three pairs under a power of two for each row, but dW's sums run across rows of unlike size.
// At the matrix cores' 16-bit rate that is three and 1.5 times the float32 instruction's
// (1001 x 50257 x 901: 324, 425 and 1070 us; in one float32 product each the matrix cores would need 4 x 590).
// bf16 gradients take one plane of dz, rounded once more, an error of the size of the result's own
// rounding (two planes where the problem is small, and of a float32 operand).
//
// An XCD's 32 CUs work on 8 x 4 neighbouring tiles at a time, so that the twelve panels they read
// come once from memory and otherwise from its L2.
#include <atomic>

#include "head.h"
#include "ns_common.h"
#include "ops_common.h"

namespace malt {

using namespace ns;

namespace {

using G = NsGeom<HEAD_BK, 2, 32>;
constexpr int BK = G::BK, H = G::H, RB = G::RB, CPR = G::CPR;
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
constexpr float LOG2E = 1.44269504088896340736f;
// A tile of EDGE x EDGE, the waves' 2 x 4 parts of it, and a ring of DEPTH stages.
template <int EDGE, int DEPTH>
struct Shape {
  static constexpr int E = EDGE, STAGES = DEPTH;
  static constexpr int TM = E / 2, TN = E / (NW / 2), NB = TM / 16, NA = TN / 16;
  static constexpr int OPER = E * RB, STAGE = 2 * OPER, RING = STAGES * STAGE;   // bytes
  static constexpr int LOADS = STAGE / 1024 / NW;                                // 1 KB each, a wave's of a stage
  // Behind the ring, so that the next tile's first stages can arrive during a tile's epilogue: rows'
  // records or labels and scales of two tiles, and the waves' statistics or 16 rows of each wave's dz (padded by 8 bytes).
  static constexpr int AT_ROWS = RING, AT_SCALES = AT_ROWS + 2 * E * 16, AT_EPI = AT_SCALES + 2 * E * 4;
  static constexpr int OUT_PITCH = TN * 2 + 8, OUT_WAVE = 16 * OUT_PITCH, JOIN = E * (NW / 2) * 8;
  // A result's 32 columns of a wave's rows (padded by 16 bytes), in the ring's place.
  static constexpr int GRAD_PITCH = 32 * 4 + 16, GRAD_WAVE = TM * GRAD_PITCH;
  static constexpr int EPI = NW * OUT_WAVE > JOIN ? NW * OUT_WAVE : JOIN;
  static constexpr int LDS = AT_EPI + EPI > NW * GRAD_WAVE ? AT_EPI + EPI : NW * GRAD_WAVE;
  static constexpr int PER_CU = 2 * LDS <= 160 * 1024 ? 2 : 1, GROUPS = 256 * PER_CU;   // workgroups that run at a time
  static_assert(PER_CU * LDS <= 160 * 1024 && LOADS * NW * 1024 == STAGE && (RING & (RING - 1)) == 0, "LDS");
  typedef f32x4 Acc[NA][NB];
};
typedef Shape<256, 2> Large;
typedef Shape<128, 2> Small;
typedef Shape<128, 4> Deep;   // for a CU that has one tile at a time: 0.38 us a stage where two slots take 0.55
static_assert(BK == 64 && CPR == 8 && NT == 512, "the loads and reads below");

__host__ __device__ inline int stages_of(const HeadProduct& g) { return (int)((g.k + BK - 1) / BK); }

// Block b's tile (i, j) and part of the contraction, or i < 0.  Blocks b, b + 8, ... run on one XCD:
// it takes an eighth of the tiles, neighbours in an order of bands of eight rows, column by column.
struct TileAt { int i, j, split; };
constexpr int BAND = 8;
__host__ __device__ inline int tile_blocks(int tiles_m, int tiles_n, int splits) {
  return (tiles_m * tiles_n * splits + 7) / 8 * 8;
}
__device__ __forceinline__ TileAt tile_at(int b, int tiles_m, int tiles_n, int splits) {
  const int tiles = tiles_m * tiles_n, all = tiles * splits, per = (all + 7) / 8;
  int t = (b & 7) * per + (b >> 3);
  if ((b >> 3) >= per || t >= all) return {-1, -1, 0};   // so for any block past the last
  const int split = t / tiles;
  t -= split * tiles;
  const int band = t / (BAND * tiles_n), first = band * BAND, rows = tiles_m - first < BAND ? tiles_m - first : BAND;
  t -= first * tiles_n;
  return {first + t % rows, t / rows, split};
}

// One operand's loads of 1 KB each: this wave's.
template <class S>
struct Loader {
  static constexpr int E = S::E, N = S::LOADS / 2;
  const uint16_t* base;   // the tile's first row in plane 0
  uint32_t voff[N];
  int64_t plane, step;

  __device__ __forceinline__ void init(const HeadSide& s, int tile, int wave, int lane) {
    plane = s.plane;
    step = s.step;
    const int64_t row0 = (int64_t)tile * E;
    base = s.p + row0 / HEAD_TILE * s.tile + row0 % HEAD_TILE * s.ld;
    const int last = (int)(s.rows - 1 - row0 < E - 1 ? s.rows - 1 - row0 : E - 1);   // rows past the end repeat the last one
#pragma unroll
    for (int q = 0; q < N; ++q) {
      const int r = (wave + q * NW) * 8 + lane / CPR;
      const int c = (lane % CPR) ^ ((r / G::RPP) % CPR);
      voff[q] = ((uint32_t)(r < last ? r : last) * (uint32_t)s.ld + c * 8) * 2;
    }
  }
  // Stage kt of a plane.
  __device__ __forceinline__ uint64_t at(int p, int kt) const {
    return reinterpret_cast<uint64_t>(base + p * plane + kt * step);
  }
};

// A tile's product: prime() starts the loads of its first stages, arrived() waits for this wave's,
// run() does the rest.
// acc[a][b][e] = C(row0 + wr TM + 16 b + lane % 16, col0 + wc TN + 16 a + 4 (lane / 16) + e).
// HALVES: the planes are float16.
template <bool HALVES, class S>
struct Product {
  static constexpr int NA = S::NA, NB = S::NB, LOADS = S::LOADS, STAGES = S::STAGES;
  const HeadProduct& g;
  char* const lds;
  const int lane, wave;
  Loader<S> la, lb;
  int kt0, KT;   // stages of the contraction, for each pair of planes
  // The next stage to load: its pair of planes, how many stages of that are left, where they lie.
  int pair, left;
  uint64_t at_a, at_b;
  uint32_t at_lds, lds0;

  __device__ __forceinline__ Product(const HeadProduct& g_, char* lds_)
      : g(g_), lds(lds_), lane(threadIdx.x & 63), wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) {}

  __device__ __forceinline__ static i32x4 rsrc(uint64_t at) {   // as buf_rsrc: addresses have 48 bits
    return i32x4{(int)(uint32_t)at, (int)(uint32_t)(at >> 32), -1, 0x00020000};
  }
  __device__ __forceinline__ void issue(int q) const {
    if (q < LOADS / 2) dma16(rsrc(at_a), la.voff[q], 0u, at_lds + q * NW * 1024);
    else dma16(rsrc(at_b), lb.voff[q - LOADS / 2], 0u, at_lds + S::OPER + (q - LOADS / 2) * NW * 1024);
  }
  __device__ __forceinline__ void start_pair() {
    at_a = la.at((int)(g.pair_a >> (4 * pair)) & 15, kt0);
    at_b = lb.at((int)(g.pair_b >> (4 * pair)) & 15, kt0);
    left = KT;
  }
  // Past the stage that was loaded last.
  __device__ __forceinline__ void advance() {
    at_a += 2 * la.step;
    at_b += 2 * lb.step;
    at_lds = lds0 + ((at_lds - lds0 + S::STAGE) & (S::RING - 1));
    if (--left == 0) {
      ++pair;
      start_pair();
    }
  }

  // No wave reads the ring any more.
  __device__ __forceinline__ void prime(int tile_a, int tile_b, int first, int count) {
    kt0 = first;
    KT = count;
    la.init(g.a, tile_a, wave, lane);
    lb.init(g.b, tile_b, wave, lane);
    pair = 0;
    at_lds = lds0 = lds_u32(lds) + wave * 1024;
    start_pair();
    const int total = KT * g.pairs;
#pragma unroll
    for (int s = 0; s < STAGES; ++s)
      if (s < total) {
#pragma unroll
        for (int q = 0; q < LOADS; ++q) issue(q);
        advance();
      }
  }

  __device__ __forceinline__ void arrived() const {
    asm volatile("" ::: "memory");
    wait_vm_c<0>();
  }

  // A ring of loads: at the barrier that closes stage st, stage st + 1 has arrived and every wave is
  // done with the slot of stage st, which then receives stage st + STAGES; half of its loads go out at
  // once, half from among the products that follow.  Fragments are read one sub-step ahead.
  // Loads arrive in order: while as many are under way as stages st + 2 and later have, one of st + 1 cannot be.
  __device__ __forceinline__ static void next_arrived(int later) {
    if constexpr (STAGES > 2) {
      static_assert(STAGES == 4, "the cases below");
      if (later >= 2) wait_vm_c<2 * LOADS>();
      else if (later == 1) wait_vm_c<LOADS>();
      else wait_vm_c<0>();
    } else {
      wait_vm_c<0>();
    }
  }
  __device__ __forceinline__ void run(typename S::Acc& acc) {
    const int wr = wave / (NW / 2), wc = wave % (NW / 2);
    // Block b's fragment lies 16 b rows below block 0's: 16 rows keep the swizzle's phase.
    int oa[H], ob[H];
#pragma unroll
    for (int h = 0; h < H; ++h) {
      oa[h] = G::swz_rk(wr * S::TM + (lane & 15), 4 * h + (lane >> 4));
      ob[h] = S::OPER + G::swz_rk(wc * S::TN + (lane & 15), 4 * h + (lane >> 4));
    }
#pragma unroll
    for (int a = 0; a < NA; ++a)
#pragma unroll
      for (int b = 0; b < NB; ++b) acc[a][b] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int total = KT * g.pairs;
    if (total == 0) return;
    bf16x8 fa[2][NB], fb[2][NA];
    auto read = [&](int buf, const char* st, int h) {
#pragma unroll
      for (int b = 0; b < NB; ++b) fa[buf][b] = *reinterpret_cast<const bf16x8*>(st + oa[h] + b * 16 * RB);
#pragma unroll
      for (int a = 0; a < NA; ++a) fb[buf][a] = *reinterpret_cast<const bf16x8*>(st + ob[h] + a * 16 * RB);
    };
    __builtin_amdgcn_s_barrier();   // every wave's loads have arrived
    asm volatile("" ::: "memory");
    read(0, lds, 0);
    auto stage = [&](const int st, auto steady_tag) {
      constexpr bool steady = decltype(steady_tag)::value;   // stage st + STAGES exists
      const char* const slot = lds + (st & (STAGES - 1)) * S::STAGE;
#pragma unroll
      for (int h = 0; h < H; ++h) {
        const int c = h & 1;
        if (h + 1 < H) {
          read(c ^ 1, slot, h + 1);
        } else if (steady || st + 1 < total) {
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // this wave's reads of the stage are done
          next_arrived(steady ? STAGES - 2 : total - st - 2);
          __builtin_amdgcn_s_barrier();
          asm volatile("" ::: "memory");
          if constexpr (steady) {
#pragma unroll
            for (int q = LOADS / 2; q < LOADS; ++q) issue(q);
          }
          read(c ^ 1, lds + ((st + 1) & (STAGES - 1)) * S::STAGE, 0);
        }
#pragma unroll
        for (int a = 0; a < NA; ++a)
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            if constexpr (HALVES)
              acc[a][b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, fb[c][a]), __builtin_bit_cast(f16x8, fa[c][b]),
                                                                 acc[a][b], 0, 0, 0);
            else
              acc[a][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[c][a], fa[c][b], acc[a][b], 0, 0, 0);
            if (steady && h == H - 1 && a * NB + b < LOADS / 2) issue(a * NB + b);
          }
#pragma unroll
        for (int j = 0; j < NA * NB; ++j) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);   // one product
          __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);   // one LDS read
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (steady) advance();
    };
    int st = 0;
    for (; st < total - STAGES; ++st) stage(st, std::true_type{});
    for (; st < total; ++st) stage(st, std::false_type{});
  }
};

// Over the four lanes that hold a row's columns, 16 and 32 lanes apart: exchanges between registers,
// no round trips through LDS.
template <class F>
__device__ __forceinline__ float across(float v, F&& op) {
  auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = op(__uint_as_float(p[0]), __uint_as_float(p[1]));
  p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return op(__uint_as_float(p[0]), __uint_as_float(p[1]));
}

// A 4 x 4 block of 16-bit values in a lane quad, turned: in, lane p holds column p's rows 0, 1 (x) and 2, 3 (y);
// out, row p's four columns.  `pick` takes the low halves of this lane and the next (even lanes) or the
// high ones of the one before and this (odd): byte permutes and selects, no branches.
__device__ __forceinline__ uint32_t turn_pick(int lane) { return lane & 1 ? 0x03020706u : 0x05040100u; }
__device__ __forceinline__ op_u32x2 turn_quad(uint2 v, uint32_t pick, bool low) {
  const uint32_t x1 = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v.x, 0xB1, 0xF, 0xF, true);   // lane p ^ 1
  const uint32_t y1 = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v.y, 0xB1, 0xF, 0xF, true);
  const uint32_t a = __builtin_amdgcn_perm(x1, v.x, pick), b = __builtin_amdgcn_perm(y1, v.y, pick);   // two columns of rows p % 2, 2 + p % 2
  const uint32_t give = low ? b : a;
  const uint32_t got = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)give, 0x4E, 0xF, 0xF, true);      // lane p ^ 2
  return op_u32x2{low ? a : got, low ? got : b};
}

// A power of two's exponent.
__device__ __forceinline__ int exponent_of(float scale) { return (int)(__float_as_uint(scale) >> 23) - 127; }

// The scales of rows (in LDS, `scales` of this lane's first) and of this lane's columns into its logits: exponents are added
// before they are applied.  Two products, one after the other, would pass through infinity or lose bits below the
// smallest normal number where a large row meets a small one.
template <int NA, int NB>
__device__ __forceinline__ void scale_logits(const float* columns, int c, int g, const float* scales, f32x4 (&acc)[NA][NB]) {
  i32x4 w[NA];
#pragma unroll
  for (int i = 0; i < NA; ++i) {
    const f32x4 s = *reinterpret_cast<const MALT_GLOBAL f32x4*>(gptr(columns) + c + 16 * i + 4 * g);
#pragma unroll
    for (int e = 0; e < 4; ++e) w[i][e] = exponent_of(s[e]);
  }
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int x = exponent_of(scales[16 * b]);
#pragma unroll
    for (int i = 0; i < NA; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[i][b][e] = __builtin_amdgcn_ldexpf(acc[i][b][e], w[i][e] + x);
  }
}

// All waves are done with what they read of LDS.
__device__ __forceinline__ void lds_free() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

__device__ __forceinline__ int label_of(const HeadLabels& l, int64_t r, int64_t vocab) {
  const int64_t y = load_id(l.labels, l.wide, r * l.stride);
  return (uint64_t)y < (uint64_t)vocab ? (int)y : -1;
}

}  // namespace

// A workgroup takes every 32nd tile of its XCD's.  While a tile's sums are formed in registers,
// the next one's first stages arrive.
template <bool HALVES, class S>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(WPE * S::PER_CU, WPE * S::PER_CU)))
void head_first_kernel(HeadLogits a) {
  constexpr int E = S::E, TM = S::TM, TN = S::TN, NA = S::NA, NB = S::NB;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  int block = blockIdx.x;
  TileAt t = tile_at(block, a.g.tiles_m, a.g.tiles_n, 1);
  if (t.i < 0) return;
  Product<HALVES, S> product(a.g, lds);
  const int lane = product.lane, wave = product.wave, wr = wave / (NW / 2), wc = wave % (NW / 2), g = lane >> 4;
  const int KT = stages_of(a.g);
  product.prime(t.i, t.j, 0, KT);
  int* const labels = reinterpret_cast<int*>(lds + S::AT_ROWS);   // [2][row]
  auto row_label = [&](int i) {
    const int64_t m = (int64_t)i * E + threadIdx.x;
    return threadIdx.x < E && m < a.g.m ? label_of(a.rows, m, a.vocab) : -1;
  };
  float* const scales = reinterpret_cast<float*>(lds + S::AT_SCALES);   // [2][row]
  auto row_scale = [&](int i) { return HALVES ? gptr(a.x_scales)[(int64_t)i * E + threadIdx.x % E] : 1.f; };
  int own = row_label(t.i), turn = 0;
  float own_scale = row_scale(t.i);
  product.arrived();
  malt_f32x2* const join = reinterpret_cast<malt_f32x2*>(lds + S::AT_EPI);   // [row][wave column]
  for (;;) {
    const int64_t row0 = (int64_t)t.i * E, col0 = (int64_t)t.j * E;
    const int tile_n = t.j;
    if (threadIdx.x < E) {
      labels[turn * E + threadIdx.x] = own;
      if (HALVES) scales[turn * E + threadIdx.x] = own_scale;
    }
    typename S::Acc acc;
    product.run(acc);
    lds_free();
    block += gridDim.x;
    t = tile_at(block, a.g.tiles_m, a.g.tiles_n, 1);
    if (t.i >= 0) {
      product.prime(t.i, t.j, 0, KT);
      own = row_label(t.i);
      own_scale = row_scale(t.i);
    }
    const int c = (int)col0 + wc * TN, left = a.g.n - c - 4 * g;   // columns there are from this lane's first
    const bool end = a.g.n - c < TN;
    const int rows = a.g.m - (int)row0 - wr * TM;   // this wave's
    if constexpr (HALVES) scale_logits(a.w_scales, c, g, scales + turn * E + wr * TM + (lane & 15), acc);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      if (b % 4 == 0 && 16 * b >= rows) break;
      const int ml = wr * TM + b * 16 + (lane & 15), yl = labels[turn * E + ml] - c;   // the label's place in the wave's columns
      if (__builtin_amdgcn_ballot_w64((unsigned)yl < TN)) {   // few waves meet a label
        float z = 0.f;
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const bool label = yl == 16 * i + 4 * g + e;
            z = label ? acc[i][b][e] : z;
            acc[i][b][e] = label ? -__builtin_inff() : acc[i][b][e];
          }
        if ((unsigned)yl < TN && ((yl >> 2) & 3) == g) gptr(a.at_label)[row0 + ml] = z * LOG2E;
      }
      if (end) {
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][b][e] = 16 * i + e >= left ? -__builtin_inff() : acc[i][b][e];
      }
      float top = acc[0][b][0];
#pragma unroll
      for (int i = 0; i < NA; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) top = fmaxf(top, acc[i][b][e]);
      top = across(top, [](float a, float b) { return fmaxf(a, b); }) * LOG2E;
      const float ref = top == -__builtin_inff() ? 0.f : top;
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < NA; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += __builtin_amdgcn_exp2f(__builtin_fmaf(acc[i][b][e], LOG2E, -ref));
      sum = across(sum, [](float a, float b) { return a + b; });
      if (g == 0) join[ml * (NW / 2) + wc] = malt_f32x2{top, sum};
    }
    product.arrived();
    lds_free();
    const int64_t m = row0 + threadIdx.x;
    if (threadIdx.x < E && m < a.g.m) {
      float top = -__builtin_inff(), sum = 0.f;
#pragma unroll
      for (int i = 0; i < NW / 2; ++i) top = fmaxf(top, join[threadIdx.x * (NW / 2) + i].x);
      const float ref = top == -__builtin_inff() ? 0.f : top;
#pragma unroll
      for (int i = 0; i < NW / 2; ++i) {
        const malt_f32x2 v = join[threadIdx.x * (NW / 2) + i];
        sum += v.y * __builtin_amdgcn_exp2f(v.x - ref);
      }
      gptr(a.partial)[m * a.parts + tile_n] = malt_f32x2{top, sum};
    }
    if (t.i < 0) return;
    turn ^= 1;
  }
}

template <bool HALVES, class S>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(WPE * S::PER_CU, WPE * S::PER_CU)))
void head_second_kernel(HeadLogits a) {
  constexpr int E = S::E, TM = S::TM, TN = S::TN, NA = S::NA, NB = S::NB;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  int block = blockIdx.x;
  TileAt t = tile_at(block, a.g.tiles_m, a.g.tiles_n, 1);
  if (t.i < 0) return;
  Product<HALVES, S> product(a.g, lds);
  const int lane = product.lane, wave = product.wave, wr = wave / (NW / 2), wc = wave % (NW / 2), g = lane >> 4;
  const int KT = stages_of(a.g);
  product.prime(t.i, t.j, 0, KT);
  f32x4* const records = reinterpret_cast<f32x4*>(lds + S::AT_ROWS);   // [2][row]
  auto record = [&](int i) {
    return *reinterpret_cast<const MALT_GLOBAL f32x4*>(
        gptr(reinterpret_cast<const float*>(a.records + (int64_t)i * E + threadIdx.x % E)));
  };
  float* const scales = reinterpret_cast<float*>(lds + S::AT_SCALES);   // [2][row]
  auto row_scale = [&](int i) { return HALVES ? gptr(a.x_scales)[(int64_t)i * E + threadIdx.x % E] : 1.f; };
  f32x4 own = record(t.i);
  float own_scale = row_scale(t.i);
  int turn = 0;
  product.arrived();
  char* const sto = lds + S::AT_EPI + wave * S::OUT_WAVE;
  const uint32_t pick = turn_pick(lane);
  const bool low = (lane & 3) < 2;
  for (;;) {
    const int64_t col0 = (int64_t)t.j * E;
    const int tile_m = t.i, tile_n = t.j;
    if (threadIdx.x < E) {
      records[turn * E + threadIdx.x] = own;
      if (HALVES) scales[turn * E + threadIdx.x] = own_scale;
    }
    typename S::Acc acc;
    product.run(acc);
    lds_free();
    block += gridDim.x;
    t = tile_at(block, a.g.tiles_m, a.g.tiles_n, 1);
    if (t.i >= 0) {
      product.prime(t.i, t.j, 0, KT);
      own = record(t.i);
      own_scale = row_scale(t.i);
    }
    const int c = (int)col0 + wc * TN, left = a.g.n - c - 4 * g;
    const bool end = a.g.n - c < TN;
    // This wave's rows, to the end of the last stage that the gradients read.
    const int rows = (a.g.m - tile_m * E + BK - 1) / BK * BK - wr * TM;
    if constexpr (HALVES) scale_logits(a.w_scales, c, g, scales + turn * E + wr * TM + (lane & 15), acc);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      if (b % 4 == 0 && 16 * b >= rows) break;
      const int ml = wr * TM + b * 16 + (lane & 15);
      const f32x4 s = records[turn * E + ml];
      const int y = __float_as_int(s.w), yl = y < 0 ? -1 : y - (int)a.col0 - c;
#pragma unroll
      for (int i = 0; i < NA; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          acc[i][b][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(acc[i][b][e], LOG2E, -s.x)) * s.y;
      if (__builtin_amdgcn_ballot_w64((unsigned)yl < TN)) {
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const bool label = yl == 16 * i + 4 * g + e;
            acc[i][b][e] = label ? -s.z : acc[i][b][e];
          }
      }
      // Zeros in rows that have no gradient, whatever their logits are, and past the end.
      if (__builtin_amdgcn_ballot_w64(y < 0)) {
        const bool none = y < 0;
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][b][e] = none ? 0.f : acc[i][b][e];
      }
      if (end) {
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][b][e] = 16 * i + e >= left ? 0.f : acc[i][b][e];
      }
    }
    // The next tile's loads are waited for before the stores go out: loads and stores may complete in any
    // order, and waiting for both would put the stores' time between two tiles.
    product.arrived();
    // 16 rows of dz, or 16 columns of as many rows as the wave has columns, meet in the wave's own region of LDS, so
    // that stores cover whole lines (8 bytes a lane straight from the registers: dz_t alone 9 us a tile).
    auto packed = [&](int i, int b) { return uint2{pack_bf16x2(acc[i][b][0], acc[i][b][1]), pack_bf16x2(acc[i][b][2], acc[i][b][3])}; };
    constexpr int GB = TN / 16, CHUNKS = TN / 8, ROWS = 64 / CHUNKS;   // 16 bytes each; rows a store covers
    const int col = tile_n * E + wc * TN;
    auto leave = [&](bf16_t* out) {
      // The wave's LDS instructions run in order.
      asm volatile("" ::: "memory");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int it = 0; it < 16 / ROWS; ++it) {
        const int r = lane / CHUNKS + ROWS * it, ch = lane % CHUNKS;
        const char* src = sto + r * S::OUT_PITCH + ch * 16;
        const uint2 lo = *reinterpret_cast<const uint2*>(src);
        const uint2 hi = *reinterpret_cast<const uint2*>(src + 8);
        const u32x4 v = {lo.x, lo.y, hi.x, hi.y};
        *reinterpret_cast<MALT_GLOBAL u32x4*>(gptr(out) + r * BK + ch * 8) = v;
      }
      asm volatile("" ::: "memory");
      __builtin_amdgcn_wave_barrier();
    };
    for (int p = 0; p < a.dz_planes; ++p) {
#pragma unroll
      for (int b0 = 0; b0 < NB; b0 += GB) {
        if (16 * b0 >= rows) break;
        const int row = tile_m * E + wr * TM + 16 * b0;
        if (a.dz) {
          bf16_t* const dz = a.dz + p * a.dz_plane + row / HEAD_TILE * a.dz_tile + col / BK * HEAD_BLOCK + row % HEAD_TILE * BK + col % BK;
#pragma unroll
          for (int b = 0; b < GB; ++b) {
#pragma unroll
            for (int i = 0; i < NA; ++i) *reinterpret_cast<uint2*>(sto + (lane & 15) * S::OUT_PITCH + (4 * g + i * 16) * 2) = packed(i, b0 + b);
            leave(dz + 16 * b * BK);
          }
        }
        if (a.dz_t) {
          bf16_t* const dz_t = a.dz_t + p * a.dz_plane + col / HEAD_TILE * a.dz_t_tile + row / BK * HEAD_BLOCK + col % HEAD_TILE * BK + row % BK;
#pragma unroll
          for (int i = 0; i < NA; ++i) {
            // Lane p of a quad takes column p of its four rows.
#pragma unroll
            for (int b = 0; b < GB; ++b)
              *reinterpret_cast<op_u32x2*>(sto + (4 * g + (lane & 3)) * S::OUT_PITCH + (16 * b + (lane & 12)) * 2) =
                  turn_quad(packed(i, b0 + b), pick, low);
            leave(dz_t + 16 * i * BK);
          }
        }
        if (p + 1 < a.dz_planes) {
#pragma unroll
          for (int b = b0; b < b0 + GB; ++b)
#pragma unroll
            for (int i = 0; i < NA; ++i) {
              const uint2 v = packed(i, b);
              acc[i][b][0] -= bf16_lo(v.x);
              acc[i][b][1] -= bf16_hi(v.x);
              acc[i][b][2] -= bf16_lo(v.y);
              acc[i][b][3] -= bf16_hi(v.y);
            }
        }
      }
    }
    if (t.i < 0) return;
    turn ^= 1;
  }
}

namespace {

// Four columns of a result, `width` of which there are, from their sums.
template <class T>
__device__ __forceinline__ void write4(const HeadOut& o, float scale, bool none, T* out, int64_t width, op_f32x4 v) {
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = none || scale == 0.f ? 0.f : v[e] * scale;
  if (o.accumulate) {
    const op_f32x4 u = row_load4(out, 0, width);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += u[e];
  }
  row_store4(out, 0, width, v);
}
// Rows that have no gradient.
__device__ __forceinline__ bool row_without(const HeadOut& o, const HeadGrads& a, int64_t m) {
  return o.mask_rows && gptr(reinterpret_cast<const int32_t*>(a.records + m))[3] < 0;
}
__device__ __forceinline__ float scale_of(const HeadGrads& a) { return a.scale_at ? a.scale * gptr(a.scale_at)[0] : a.scale; }

// A wave's sub-tile leaves through its own part of LDS, 32 of its columns at a time, so that a
// store covers eight rows' 128 bytes, and in a loop: straight from the registers it is 30 KB of code,
// run once a tile.
template <class T, class S>
__device__ __forceinline__ void write_out(const HeadOut& o, const HeadGrads& a, int split, int64_t row0, int64_t col0, char* lds,
                                          const typename S::Acc& acc) {
  constexpr int TM = S::TM, TN = S::TN, NB = S::NB;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = wave / (NW / 2), wc = wave % (NW / 2);
  const float scale = scale_of(a);
  char* const own = lds + wave * S::GRAD_WAVE;
  const int64_t m0 = row0 + wr * TM + (lane >> 3);
  const int rows = (int)(o.g.m - m0);   // there are, from this lane's first
  uint32_t none = 0;                    // bit i: row 8 i has no gradient
  if (o.mask_rows) {
#pragma unroll
    for (int i = 0; i < TM / 8; ++i) none |= (8 * i < rows && row_without(o, a, m0 + 8 * i) ? 1u : 0u) << i;
  }
#pragma unroll
  for (int slice = 0; slice < TN / 32; ++slice) {
    // The wave's LDS instructions run in order.
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int b = 0; b < NB; ++b)
        *reinterpret_cast<f32x4*>(own + (16 * b + (lane & 15)) * S::GRAD_PITCH + (16 * i + 4 * (lane >> 4)) * 4) = acc[2 * slice + i][b];
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
    const int64_t n = col0 + wc * TN + 32 * slice + 4 * (lane & 7);
    if (n >= o.g.n) continue;
    const char* from = own + (lane >> 3) * S::GRAD_PITCH + (lane & 7) * 16;
    const int width = (int)(o.g.n - n);   // columns there are from this lane's first
    float* part = o.partial + ((int64_t)split * o.g.m + m0) * o.g.n + n;
    T* out = static_cast<T*>(o.out) + m0 * o.ldo + n;
#pragma unroll 4
    for (int i = 0; i < TM / 8; ++i, from += 8 * S::GRAD_PITCH, part += 8 * (int64_t)o.g.n, out += 8 * o.ldo) {
      if (8 * i >= rows) break;
      const f32x4 x = *reinterpret_cast<const f32x4*>(from);
      op_f32x4 v = {x.x, x.y, x.z, x.w};
      if (o.add_partial) {
        const op_f32x4 u = row_load4(part, 0, width);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += u[e];
      }
      if (o.write_partial) row_store4(part, 0, width, v);
      else write4(o, scale, (none >> i) & 1, out, width, v);
    }
  }
}

}  // namespace

template <class S>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(WPE * S::PER_CU, WPE * S::PER_CU)))
void head_grads_kernel(HeadGrads a) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  int b = blockIdx.x, which = 0;
  const int first = tile_blocks(a.part[0].g.tiles_m, a.part[0].g.tiles_n, a.part[0].splits);
  if (a.parts > 1 && b >= first) {
    b -= first;
    which = 1;
  }
  const HeadOut& o = a.part[which];
  const TileAt t = tile_at(b, o.g.tiles_m, o.g.tiles_n, o.splits);
  if (t.i < 0) return;
  const int split = t.split;
  const int64_t row0 = (int64_t)t.i * S::E, col0 = (int64_t)t.j * S::E;
  const int KT = stages_of(o.g), kt0 = (int)((int64_t)KT * split / o.splits), kt1 = (int)((int64_t)KT * (split + 1) / o.splits);
  typename S::Acc acc;
  Product<false, S> product(o.g, lds);
  product.prime(t.i, t.j, kt0, kt1 - kt0);
  product.arrived();
  product.run(acc);
  lds_free();
  if (o.f32) write_out<float, S>(o, a, split, row0, col0, lds, acc);
  else write_out<bf16_t, S>(o, a, split, row0, col0, lds, acc);
}

// The sums of contractions' parts, four columns a thread: one result's, then the other's.  Of many parts
// a wave takes a quarter each, or few outputs would wait for one load after another (74 x 431, 64 parts: 30 -> 9 us).
constexpr int SUM_MANY = 8, SUM_WAVES = 4;
__host__ __device__ inline int sum_quads(const HeadOut& o) { return o.splits >= SUM_MANY ? 64 : 64 * SUM_WAVES; }   // of a workgroup
template <class T>
__device__ __forceinline__ void sum4(const HeadOut& o, const HeadGrads& a, int64_t block, op_f32x4 (&join)[SUM_WAVES][64]) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const bool many = o.splits >= SUM_MANY;   // the same for a workgroup
  const int64_t i = block * sum_quads(o) + (many ? lane : threadIdx.x), per = (o.g.n + 3) / 4, m = i / per, n = i % per * 4;
  const int first = many ? wave : 0, step = many ? SUM_WAVES : 1;
  op_f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (m < o.g.m) {
    const float* const p = o.partial + m * o.g.n;
#pragma unroll 4
    for (int s = first; s < o.splits; s += step) {
      const op_f32x4 u = row_load4(p + s * (int64_t)o.g.m * o.g.n, n, o.g.n);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += u[e];
    }
  }
  if (many) {
    join[wave][lane] = v;
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int w = 1; w < SUM_WAVES; ++w)
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += join[w][lane][e];
  }
  if (m < o.g.m) write4(o, scale_of(a), row_without(o, a, m), static_cast<T*>(o.out) + m * o.ldo + n, o.g.n - n, v);
}
__global__ __launch_bounds__(64 * SUM_WAVES) void head_sum_kernel(HeadGrads a, int first_blocks) {
  __shared__ op_f32x4 join[SUM_WAVES][64];
  const bool second = (int)blockIdx.x >= first_blocks;
  const HeadOut& o = a.part[second ? 1 : 0];
  const int64_t block = blockIdx.x - (second ? first_blocks : 0);
  if (o.f32) sum4<float>(o, a, block, join);
  else sum4<bf16_t>(o, a, block, join);
}

namespace {
template <class S>
hipError_t raise_limits() {
  for (const void* f : {reinterpret_cast<const void*>(&head_first_kernel<false, S>), reinterpret_cast<const void*>(&head_first_kernel<true, S>),
                        reinterpret_cast<const void*>(&head_second_kernel<false, S>), reinterpret_cast<const void*>(&head_second_kernel<true, S>),
                        reinterpret_cast<const void*>(&head_grads_kernel<S>)}) {
    const hipError_t e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, S::LDS);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
}  // namespace

// The kernels use more dynamic LDS than the default limit: raised once for each device.
hipError_t head_setup() {
  static std::atomic<uint64_t> raised{0};
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = uint64_t(1) << (dev & 63);
  if (dev <= 63 && raised.load(std::memory_order_relaxed) & bit) return hipSuccess;
  e = raise_limits<Large>();
  if (e == hipSuccess) e = raise_limits<Small>();
  if (e == hipSuccess) e = raise_limits<Deep>();
  if (e != hipSuccess) return e;
  if (dev <= 63) raised.fetch_or(bit, std::memory_order_relaxed);
  return hipSuccess;
}

namespace {
template <class S>
void logits_of(const HeadLogits& a, bool second, int blocks, hipStream_t s) {
  const dim3 grid((unsigned)(blocks < S::GROUPS ? blocks : S::GROUPS));
  if (second && a.x_scales) hipLaunchKernelGGL((head_second_kernel<true, S>), grid, dim3(NT), S::LDS, s, a);
  else if (second) hipLaunchKernelGGL((head_second_kernel<false, S>), grid, dim3(NT), S::LDS, s, a);
  else if (a.x_scales) hipLaunchKernelGGL((head_first_kernel<true, S>), grid, dim3(NT), S::LDS, s, a);
  else hipLaunchKernelGGL((head_first_kernel<false, S>), grid, dim3(NT), S::LDS, s, a);
}
}  // namespace

hipError_t launch_head_logits(const HeadLogits& a, int edge, bool second, hipStream_t s) {
  const int blocks = tile_blocks(a.g.tiles_m, a.g.tiles_n, 1);
  if (edge == 256) logits_of<Large>(a, second, blocks, s);
  else if (blocks > Deep::GROUPS) logits_of<Small>(a, second, blocks, s);
  else logits_of<Deep>(a, second, blocks, s);
  return hipGetLastError();
}

hipError_t launch_head_grads(const HeadGrads& a, int edge, hipStream_t s) {
  int blocks = 0;
  for (int i = 0; i < a.parts; ++i) blocks += tile_blocks(a.part[i].g.tiles_m, a.part[i].g.tiles_n, a.part[i].splits);
  const dim3 grid((unsigned)blocks);
  if (edge == 256) hipLaunchKernelGGL(head_grads_kernel<Large>, grid, dim3(NT), Large::LDS, s, a);
  else if (blocks > Deep::GROUPS) hipLaunchKernelGGL(head_grads_kernel<Small>, grid, dim3(NT), Small::LDS, s, a);
  else hipLaunchKernelGGL(head_grads_kernel<Deep>, grid, dim3(NT), Deep::LDS, s, a);
  return hipGetLastError();
}

hipError_t launch_head_sum(const HeadGrads& a, bool first, bool second, hipStream_t s) {
  auto blocks = [&](int i) {
    const int quads = sum_quads(a.part[i]);
    return (int)(((int64_t)a.part[i].g.m * ((a.part[i].g.n + 3) / 4) + quads - 1) / quads);
  };
  const int n = first ? blocks(0) : 0, all = n + (second ? blocks(1) : 0);
  if (all == 0) return hipSuccess;
  hipLaunchKernelGGL(head_sum_kernel, dim3((unsigned)all), dim3(256), 0, s, a, n);
  return hipGetLastError();
}

}  // namespace malt
