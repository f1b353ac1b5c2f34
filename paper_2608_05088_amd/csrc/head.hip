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
// A workgroup of eight waves makes one 256 x 256 tile, the pipeline of the Newton-Schulz
// update (ns_common.h): stages of 64 contracted values go straight to LDS, two slots deep.  Rows with
// the contraction contiguous ("rows") are read as they lie, an operand whose rows are the
// contraction ("columns") through transposed LDS reads, so that nothing is transposed in memory.
//
// float32 operands are three bf16 planes whose sum they are.  A product of two is the six plane
// products that matter (high by low and middle by low are below 2^-26 of it), small ones first,
// run as a contraction six times as long: float32 sums of exact products, at 2.5 times the rate
// of the float32 matrix instruction.  bf16 gradients take dz and the operands as single
// planes: dz is rounded once more, an error of the size of the result's own rounding.
//
// Tiles are dealt to the eight XCDs in blocks of 8 x 4, so that the panels of the tiles that run
// on one XCD at a time are few enough for its L2.
#include <atomic>

#include "head.h"
#include "ns_common.h"
#include "ops_common.h"

namespace malt {

using namespace ns;

namespace {

using G = NsGeom<HEAD_BK, 2, 32>;
constexpr int BK = G::BK, STAGES = G::STAGES, H = G::H, RB = G::RB, CPR = G::CPR, LOADS = G::LOADS;
constexpr int NB = TM / 16, NA = TN / 16;
constexpr float LOG2E = 1.44269504088896340736f;
constexpr int OUT_PITCH = TN * 2 + 8;   // dz's staging: a wave's sub-tile, rows padded by 8 bytes
constexpr int STAGING = NW * TM * OUT_PITCH;
constexpr int LDS_BYTES = G::RING_BYTES > STAGING ? G::RING_BYTES : STAGING;
static_assert(LDS_BYTES <= 160 * 1024, "LDS budget");
static_assert(BK == 64 && CPR == 8 && LOADS == 8, "the loads below");

enum Side { ROWS, COLS };   // ROWS: [row][k]; COLS: [k][row]

struct TileAt { int i, j; };

// Block b's tile of tiles_m x tiles_n, or i < 0.  Blocks b, b + 8, ... run on one XCD.
constexpr int SUPER_M = 8, SUPER_N = 4;
__host__ __device__ inline int supers(int tiles_m, int tiles_n) {
  return ((tiles_m + SUPER_M - 1) / SUPER_M) * ((tiles_n + SUPER_N - 1) / SUPER_N);
}
__host__ __device__ inline int tile_blocks(int tiles_m, int tiles_n) {
  return (supers(tiles_m, tiles_n) + 7) / 8 * 8 * SUPER_M * SUPER_N;
}
__device__ __forceinline__ TileAt tile_at(int b, int tiles_m, int tiles_n) {
  const int xcd = b & 7, slot = b >> 3;
  const int super = slot / (SUPER_M * SUPER_N) * 8 + xcd, in = slot % (SUPER_M * SUPER_N);
  const int sm = (tiles_m + SUPER_M - 1) / SUPER_M;
  const int i = super % sm * SUPER_M + in % SUPER_M, j = super / sm * SUPER_N + in / SUPER_M;
  return i < tiles_m && j < tiles_n ? TileAt{i, j} : TileAt{-1, -1};
}

// One operand's loads: 32 of 1 KB a stage, four of them this wave's.
template <Side S>
struct Loader {
  const uint16_t* base;   // the tile's first row (ROWS) or column (COLS) of plane 0
  uint32_t voff[LOADS / 2];
  uint32_t ld;            // elements
  int64_t rows;           // COLS: contraction rows there are
  int64_t plane;

  __device__ __forceinline__ void init(const HeadSide& s, int64_t row0, int wave, int lane) {
    ld = (uint32_t)s.ld;
    plane = s.plane;
    if constexpr (S == ROWS) {
      base = s.p + row0 * s.ld;
      const int last = (int)(s.rows - 1 - row0 < 255 ? s.rows - 1 - row0 : 255);   // rows past the end repeat the last one
#pragma unroll
      for (int q = 0; q < LOADS / 2; ++q) {
        const int r = (wave + q * NW) * 8 + lane / CPR;
        const int c = (lane % CPR) ^ ((r / G::RPP) % CPR);
        voff[q] = ((uint32_t)(r < last ? r : last) * ld + c * 8) * 2;
      }
    } else {
      base = s.p + row0;
      rows = s.rows;
      const int last = (int)(s.cols - 8 - row0 < 248 ? s.cols - 8 - row0 : 248);   // columns past the end repeat the last eight
#pragma unroll
      for (int q = 0; q < LOADS / 2; ++q) {
        const int k = (wave + q * NW) * 2 + lane / 32;
        const int c = swz_chunk<3>(k, lane % 32) * 8;
        voff[q] = ((uint32_t)k * ld + (c < last ? c : last)) * 2;
      }
    }
  }
  // Load q of stage kt of a plane.
  __device__ __forceinline__ void load(int p, int kt, int q, int wave, int lane, uint32_t lds) const {
    const uint16_t* at = base + p * plane;
    uint32_t v = voff[q];
    if constexpr (S == ROWS) {
      at += kt * BK;
    } else {
      const int64_t k0 = (int64_t)kt * BK;
      at += k0 * ld;
      if (k0 + BK > rows) {   // rows of the contraction past the end repeat the last one: the other side is zero there
        const int k = (wave + q * NW) * 2 + lane / 32, last = (int)(rows - 1 - k0);
        if (k > last) v -= (uint32_t)(k - last) * ld * 2;
      }
    }
    dma16(buf_rsrc(at), v, 0u, lds);
  }
  __device__ static constexpr int dst(int wave, int q) { return (wave + q * NW) * 1024; }
};

// A wave's fragments of one operand: N blocks of 16 rows from row `first` of the tile.
template <Side S, int N>
struct Reader {
  int off[S == ROWS ? H : N * 2];

  __device__ __forceinline__ void init(int first, int lane) {
    if constexpr (S == ROWS) {
#pragma unroll
      for (int h = 0; h < H; ++h) off[h] = G::swz_rk(first + (lane & 15), 4 * h + (lane >> 4));
    } else {
      const int r = (lane & 15) >> 2, q = lane & 3;
#pragma unroll
      for (int a = 0; a < N; ++a)
#pragma unroll
        for (int r2 = 0; r2 < 2; ++r2) off[2 * a + r2] = swz_kn<3>(8 * (lane >> 4) + 4 * r2 + r, first + a * 16 + 4 * q);
    }
  }
  __device__ __forceinline__ bf16x8 read(const char* st, int h, int a) const {
    if constexpr (S == ROWS) {
      return *reinterpret_cast<const bf16x8*>(st + off[h] + a * 16 * RB);
    } else {
      const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t*)(st + off[2 * a] + h * 32 * KN_ROW));
      const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t*)(st + off[2 * a + 1] + h * 32 * KN_ROW));
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  }
};

// acc[a][b][e] = C(row0 + wr TM + 16 b + lane % 16, col0 + wc TN + 16 a + 4 (lane / 16) + e).
template <Side SA, Side SB>
__device__ __forceinline__ void product(const HeadProduct& g, int64_t row0, int64_t col0, char* lds, f32x4 (&acc)[NA][NB]) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = wave / (NW / 2), wc = wave % (NW / 2);
  Loader<SA> la;
  Loader<SB> lb;
  la.init(g.a, row0, wave, lane);
  lb.init(g.b, col0, wave, lane);
  Reader<SA, NB> ra;
  Reader<SB, NA> rb;
  ra.init(wr * TM, lane);
  rb.init(wc * TN, lane);
#pragma unroll
  for (int a = 0; a < NA; ++a)
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[a][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  bf16x8 fa[2][NB], fb[2][NA];
  const int KT = (int)((g.k + BK - 1) / BK);
  const int total = KT * g.pairs;
  pipeline<G, 1, LOADS / 2>(
      total, LOADS, lds,
      [&](int st, int q) {
        // The pair of planes, the stage of the contraction.
        const int p = (st >= KT) + (st >= 2 * KT) + (st >= 3 * KT) + (st >= 4 * KT) + (st >= 5 * KT), kt = st - p * KT;
        const uint32_t at = lds_u32(lds + (st % STAGES) * G::STAGE_BYTES);
        if (q < LOADS / 2) la.load((int)(g.pair_a >> (4 * p)) & 15, kt, q, wave, lane, at + la.dst(wave, q));
        else lb.load((int)(g.pair_b >> (4 * p)) & 15, kt, q - LOADS / 2, wave, lane, at + G::OPER_BYTES + lb.dst(wave, q - LOADS / 2));
      },
      [&](int buf, const char* st, int h) {
#pragma unroll
        for (int b = 0; b < NB; ++b) fa[buf][b] = ra.read(st, h, b);
#pragma unroll
        for (int a = 0; a < NA; ++a) fb[buf][a] = rb.read(st + G::OPER_BYTES, h, a);
      },
      [](int, int, const char*) {},
      [&](int buf, auto&& after) {
#pragma unroll
        for (int a = 0; a < NA; ++a)
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            acc[a][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[buf][a], fa[buf][b], acc[a][b], 0, 0, 0);
            after(a * NB + b);
          }
      });
}

__device__ __forceinline__ int64_t label_of(const HeadLabels& l, int64_t r, int64_t vocab) {
  const int64_t y = load_id(l.labels, l.wide, r * l.stride);
  return (uint64_t)y < (uint64_t)vocab ? y : -1;
}

}  // namespace

__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(WPE, WPE)))
void head_first_kernel(HeadLogits a) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const TileAt t = tile_at(blockIdx.x, a.g.tiles_m, a.g.tiles_n);
  if (t.i < 0) return;
  const int64_t row0 = (int64_t)t.i * HEAD_TILE, col0 = (int64_t)t.j * HEAD_TILE;
  f32x4 acc[NA][NB];
  product<ROWS, ROWS>(a.g, row0, col0, lds, acc);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = wave / (NW / 2), wc = wave % (NW / 2), g = lane >> 4;
  malt_f32x2* const join = reinterpret_cast<malt_f32x2*>(lds);   // [row][wave column]
  __syncthreads();   // every wave is done with the ring
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int ml = wr * TM + b * 16 + (lane & 15);
    const int64_t m = row0 + ml, c = col0 + wc * TN + 4 * g;
    const int64_t y = m < a.g.m ? label_of(a.rows, m, a.vocab) : -1;
    // The label's and the end's place from this lane's first column.
    const int yl = y < 0 ? -1 : (int)(y - c), left = (int)(a.g.n - c);
    float top = -__builtin_inff(), sum = 0.f;
#pragma unroll
    for (int i = 0; i < NA; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float z = acc[i][b][e] * LOG2E;
        if (yl == 16 * i + e) gptr(a.at_label)[m] = z;
        if (yl == 16 * i + e || 16 * i + e >= left) z = -__builtin_inff();
        acc[i][b][e] = z;
        top = fmaxf(top, z);
      }
    top = fmaxf(top, __shfl_xor(top, 16, 64));
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    const float ref = top == -__builtin_inff() ? 0.f : top;
#pragma unroll
    for (int i = 0; i < NA; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum += __builtin_amdgcn_exp2f(acc[i][b][e] - ref);
    sum += __shfl_xor(sum, 16, 64);
    sum += __shfl_xor(sum, 32, 64);
    if (g == 0) join[ml * (NW / 2) + wc] = malt_f32x2{top, sum};
  }
  __syncthreads();
  const int64_t m = row0 + threadIdx.x;
  if (threadIdx.x < HEAD_TILE && m < a.g.m) {
    float top = -__builtin_inff(), sum = 0.f;
#pragma unroll
    for (int i = 0; i < NW / 2; ++i) top = fmaxf(top, join[threadIdx.x * (NW / 2) + i].x);
    const float ref = top == -__builtin_inff() ? 0.f : top;
#pragma unroll
    for (int i = 0; i < NW / 2; ++i) {
      const malt_f32x2 v = join[threadIdx.x * (NW / 2) + i];
      sum += v.y * __builtin_amdgcn_exp2f(v.x - ref);
    }
    gptr(a.partial)[m * a.parts + t.j] = malt_f32x2{top, sum};
  }
}

__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(WPE, WPE)))
void head_second_kernel(HeadLogits a) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const TileAt t = tile_at(blockIdx.x, a.g.tiles_m, a.g.tiles_n);
  if (t.i < 0) return;
  const int64_t row0 = (int64_t)t.i * HEAD_TILE, col0 = (int64_t)t.j * HEAD_TILE;
  f32x4 acc[NA][NB];
  product<ROWS, ROWS>(a.g, row0, col0, lds, acc);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = wave / (NW / 2), wc = wave % (NW / 2), g = lane >> 4;
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int64_t m = row0 + wr * TM + b * 16 + (lane & 15), c = col0 + wc * TN + 4 * g;
    HeadRow s = {0.f, 0.f, 0.f, 0.f};
    int64_t y = -1;
    if (m < a.g.m) {
      y = label_of(a.rows, m, a.vocab);
      const f32x4 v = *reinterpret_cast<const MALT_GLOBAL f32x4*>(gptr(reinterpret_cast<const float*>(a.stats + m)));
      s = HeadRow{v.x, v.y, v.z, 0.f};
      if (a.rows.weights) {
        const float w = gptr(a.rows.weights)[m * a.rows.weight_stride];
        s.inverse *= w;
        s.others *= w;
        if (w == 0.f) y = -1;
      }
    }
    const int yl = (int)(y - a.col0 - c), left = (int)(a.g.n - c);
#pragma unroll
    for (int i = 0; i < NA; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float q = __builtin_amdgcn_exp2f(acc[i][b][e] * LOG2E - s.top) * s.inverse;
        // Zeros in rows that have no gradient, whatever their logits are, and past the end.
        acc[i][b][e] = y < 0 || 16 * i + e >= left ? 0.f : yl == 16 * i + e ? -s.others : q;
      }
  }
  __syncthreads();   // every wave is done with the ring
  char* const sto = lds + wave * (TM * OUT_PITCH);
  const int sr0 = lane & 15, sc0 = 4 * g;
  for (int p = 0; p < a.dz_planes; ++p) {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < NA; ++i) {
        uint2 pk;
        pk.x = pack_bf16x2(acc[i][b][0], acc[i][b][1]);
        pk.y = pack_bf16x2(acc[i][b][2], acc[i][b][3]);
        *reinterpret_cast<uint2*>(sto + (sr0 + b * 16) * OUT_PITCH + (sc0 + i * 16) * 2) = pk;
        acc[i][b][0] -= bf16_lo(pk.x);
        acc[i][b][1] -= bf16_hi(pk.x);
        acc[i][b][2] -= bf16_lo(pk.y);
        acc[i][b][3] -= bf16_hi(pk.y);
      }
    // The wave's own region: its LDS instructions run in order.
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
    bf16_t* const dz = a.dz + p * a.dz_plane;
#pragma unroll 4
    for (int it = 0; it < TM * 8 / 64; ++it) {
      const int r = lane / 8 + 8 * it, ch = lane % 8;
      const char* src = sto + r * OUT_PITCH + ch * 16;
      const uint2 lo = *reinterpret_cast<const uint2*>(src);
      const uint2 hi = *reinterpret_cast<const uint2*>(src + 8);
      const u32x4 v = {lo.x, lo.y, hi.x, hi.y};
      *reinterpret_cast<MALT_GLOBAL u32x4*>(gptr(dz) + (row0 + wr * TM + r) * a.dz_ld + col0 + wc * TN + ch * 8) = v;
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
  }
}

namespace {

template <class T>
__device__ __forceinline__ void write_out(const HeadOut& o, const HeadGrads& a, float scale, int64_t row0, int64_t col0,
                                          const f32x4 (&acc)[NA][NB]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wr = wave / (NW / 2), wc = wave % (NW / 2);
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int64_t m = row0 + wr * TM + b * 16 + (lane & 15);
    if (m >= o.g.m) continue;
    bool none = false;
    if (o.mask_rows)
      none = label_of(a.rows, m, a.vocab) < 0 || (a.rows.weights && gptr(a.rows.weights)[m * a.rows.weight_stride] == 0.f);
#pragma unroll
    for (int i = 0; i < NA; ++i) {
      const int64_t n = col0 + wc * TN + i * 16 + 4 * (lane >> 4);
      if (n >= o.g.n) continue;
      op_f32x4 v = {acc[i][b][0], acc[i][b][1], acc[i][b][2], acc[i][b][3]};
      if (o.add_partial) {
        const op_f32x4 u = row_load4(o.partial + m * o.g.n, n, o.g.n);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += u[e];
      }
      if (o.write_partial) {
        row_store4(o.partial + m * o.g.n, n, o.g.n, v);
        continue;
      }
      T* const out = static_cast<T*>(o.out) + m * o.ldo;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = none || scale == 0.f ? 0.f : v[e] * scale;
      if (o.accumulate) {
        const op_f32x4 u = row_load4(out, n, o.g.n);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += u[e];
      }
      row_store4(out, n, o.g.n, v);
    }
  }
}

}  // namespace

__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(WPE, WPE)))
void head_grads_kernel(HeadGrads a) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  int b = blockIdx.x, which = 0;
  const int first = tile_blocks(a.part[0].g.tiles_m, a.part[0].g.tiles_n);
  if (a.parts > 1 && b >= first) {
    b -= first;
    which = 1;
  }
  const HeadOut& o = a.part[which];
  const TileAt t = tile_at(b, o.g.tiles_m, o.g.tiles_n);
  if (t.i < 0) return;
  const int64_t row0 = (int64_t)t.i * HEAD_TILE, col0 = (int64_t)t.j * HEAD_TILE;
  f32x4 acc[NA][NB];
  if (o.form == 0) product<ROWS, COLS>(o.g, row0, col0, lds, acc);
  else product<COLS, COLS>(o.g, row0, col0, lds, acc);
  float scale = a.scale;
  if (a.scale_at) scale *= gptr(a.scale_at)[0];
  if (o.f32) write_out<float>(o, a, scale, row0, col0, acc);
  else write_out<bf16_t>(o, a, scale, row0, col0, acc);
}

// The kernels use more dynamic LDS than the default limit: raised once for each device.
hipError_t head_setup() {
  static std::atomic<uint64_t> raised{0};
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = uint64_t(1) << (dev & 63);
  if (dev <= 63 && raised.load(std::memory_order_relaxed) & bit) return hipSuccess;
  for (const void* f : {reinterpret_cast<const void*>(&head_first_kernel), reinterpret_cast<const void*>(&head_second_kernel),
                        reinterpret_cast<const void*>(&head_grads_kernel)}) {
    e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, LDS_BYTES);
    if (e != hipSuccess) return e;
  }
  if (dev <= 63) raised.fetch_or(bit, std::memory_order_relaxed);
  return hipSuccess;
}

hipError_t launch_head_logits(const HeadLogits& a, bool second, hipStream_t s) {
  const dim3 grid((unsigned)tile_blocks(a.g.tiles_m, a.g.tiles_n));
  if (second) hipLaunchKernelGGL(head_second_kernel, grid, dim3(NT), LDS_BYTES, s, a);
  else hipLaunchKernelGGL(head_first_kernel, grid, dim3(NT), LDS_BYTES, s, a);
  return hipGetLastError();
}

hipError_t launch_head_grads(const HeadGrads& a, hipStream_t s) {
  int blocks = tile_blocks(a.part[0].g.tiles_m, a.part[0].g.tiles_n);
  if (a.parts > 1) blocks += tile_blocks(a.part[1].g.tiles_m, a.part[1].g.tiles_n);
  hipLaunchKernelGGL(head_grads_kernel, dim3((unsigned)blocks), dim3(NT), LDS_BYTES, s, a);
  return hipGetLastError();
}

}  // namespace malt
