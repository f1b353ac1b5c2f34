// Token table: rows looked up by id and scaled, and the table's gradient by
// sorted tokens.
//
//   out[t, :] = s table[id_t, :]            (zeros for an id outside the table)
//   dtable[v, :] (+)= s sum_{t : id_t = v} grad[t, :]
//
// Both are bound by memory.  The gradient sorts the tokens by id, stably, so
// every row's sum is taken in the order of its tokens: the result does not
// depend on how the work was scheduled.  A row with few tokens is summed by the
// wave that writes it; the sorted tokens of longer rows (one id in sixteen may
// be the same word, and padding half of all) are summed in chunks by waves of
// their own, whose sums a second launch joins.
//
// Measured (a large copy reaches 5.17 TB/s on the same card):
//   lookup of 8192 x 1280, float32 to bf16: 8.9 us, 7 TB/s with what the caches hold;
//   gradient of 8192 x 1024 float32 tokens, 50257 rows: 53 us, of which 36 to fill the table's
//   206 MB while the tokens are sorted, 11 the sums and 6 their joins; 4.5 TB/s (43 in all
//   where the caches still hold part of the table);
//   gradient of 491520 x 768 bf16 tokens into float32: 256 us, of which 41 for the sort's
//   seven launches, 14 for joins and 201 for the sums (861 MB), 4.3 TB/s; the same where
//   equal ids lie together; 263 where all are one id.
// Joining a row in the wave that writes it, chunks in a launch before, took 41 and 268 us,
// and 514 with one id.
#include "embed.h"
#include "ops_common.h"

namespace malt {

namespace {

constexpr int DIGIT = 8, BINS = 1 << DIGIT;
constexpr int STRIP = 256;     // columns a wave takes, four a lane
constexpr int GROUP = 16;      // chunks
constexpr int JOIN_WAVES = 8, JOIN_ALONE = 16;
constexpr int FILL_VECS = 4;   // groups of four columns a thread fills with zeros

// ------------------------------------------------------------------- lookup
template <class TI, class TO>
__global__ __launch_bounds__(256) void embed_lookup_kernel(EmbedLookupArgs a) {
  // 2^lanes_log2 lanes take a token (a wave at most), four columns a lane at a time.
  const int lanes = 1 << a.lanes_log2;
  const int64_t t = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> a.lanes_log2;
  if (t >= a.tokens) return;
  const int64_t id = load_id(a.ids, a.wide_ids, t);
  const bool there = id >= 0 && id < a.vocab;
  const TI* row = static_cast<const TI*>(a.table) + (there ? id : 0) * a.table_ld;
  TO* out = static_cast<TO*>(a.out) + t * a.out_ld;
  for (int c = 4 * (threadIdx.x & (lanes - 1)); c < a.width; c += 16 * lanes) {
    op_f32x4 v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      v[u] = op_f32x4{0.f, 0.f, 0.f, 0.f};
      if (there) v[u] = row_load4(row, c + 4 * u * lanes, a.width);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[u][e] = there ? v[u][e] * a.scale : 0.f;
      row_store4(out, c + 4 * u * lanes, a.width, v[u]);
    }
  }
}

// --------------------------------------------------------------------- sort
// Keys: the id, or `vocab` for an id outside the table (sorted past the rest).
__device__ __forceinline__ uint32_t token_key(const EmbedGradArgs& a, int64_t t) {
  const int64_t id = load_id(a.ids, a.wide_ids, t);
  return id >= 0 && id < a.vocab ? (uint32_t)id : (uint32_t)a.vocab;
}

// Lanes of the wave whose digit equals this lane's.
__device__ __forceinline__ uint64_t same_digit(uint32_t d, bool valid) {
  const uint64_t all = __ballot(valid);
  uint32_t lo = (uint32_t)all, hi = (uint32_t)(all >> 32);
#pragma unroll
  for (int b = 0; b < DIGIT; ++b) {
    const uint32_t x = (uint32_t)((int32_t)(d << (31 - b)) >> 31);   // bit b, all over
    const uint64_t s = __ballot(x != 0);
    lo &= ~((uint32_t)s ^ x);
    hi &= ~((uint32_t)(s >> 32) ^ x);
  }
  return (uint64_t)hi << 32 | lo;
}

__device__ __forceinline__ int lanes_below(uint64_t m) {
  return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0));
}

// Ranks of one wave's R rounds of 64 keys among the wave's keys of the same
// digit, in (round, lane) order; hist (this wave's BINS counters, zeroed)
// receives the digits' counts.
template <int R>
__device__ __forceinline__ void wave_ranks(const uint32_t (&key)[R], int shift, int rounds, int n, int lane,
                                           uint32_t* hist, uint32_t (&rank)[R]) {
#pragma unroll
  for (int r = 0; r < R; ++r)
    if (r < rounds) {
      const bool valid = r * 64 + lane < n;
      const uint32_t d = (key[r] >> shift) & (BINS - 1);
      const uint64_t m = same_digit(d, valid);
      const int below = lanes_below(m);
      uint32_t before = 0;
      if (valid) before = hist[d];
      asm volatile("" ::: "memory");   // a wave's LDS accesses are in order
      if (valid && below == 0) hist[d] = before + (uint32_t)__popcll(m);
      asm volatile("" ::: "memory");
      rank[r] = before + (uint32_t)below;
      __builtin_amdgcn_sched_barrier(0);   // one round's masks at a time: all of them together would not fit the registers
    }
}

// Exclusive sum over the threads 0 .. BINS - 1 of a workgroup (every thread calls;
// the others pass 0); `part` holds BINS / 64 values.
__device__ __forceinline__ uint32_t bins_exclusive(uint32_t v, int tid, uint32_t* part) {
  uint32_t x = v;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const uint32_t y = (uint32_t)__shfl_up((int)x, off, 64);
    if ((tid & 63) >= off) x += y;
  }
  if (tid < BINS && (tid & 63) == 63) part[tid >> 6] = x;
  __syncthreads();
  uint32_t base = 0;
#pragma unroll
  for (int w = 0; w < BINS / 64; ++w)
    if (w < (tid >> 6)) base += part[w];
  __syncthreads();
  return base + x - v;
}

// Many tokens: each pass of the sort takes one digit in three kernels: every
// block's counts of the digits, their sums over the blocks for each digit, and
// the keys' places.  The first also empties the table rows' segments.
template <bool FIRST>
__global__ __launch_bounds__(SORT_THREADS) void sort_count_kernel(EmbedGradArgs a, int shift, const uint32_t* keys) {
  __shared__ uint32_t hist[BINS];
  hist[threadIdx.x] = 0;
  if (FIRST)
    for (int64_t v = (int64_t)blockIdx.x * SORT_THREADS + threadIdx.x; v < a.vocab; v += (int64_t)gridDim.x * SORT_THREADS)
      gptr(reinterpret_cast<op_u32x2*>(a.seg))[v] = op_u32x2{0u, 0u};
  __syncthreads();
  const int64_t base = (int64_t)blockIdx.x * SORT_TILE;
  for (int i = threadIdx.x; i < SORT_TILE; i += SORT_THREADS) {
    if (base + i >= a.tokens) break;
    const uint32_t k = FIRST ? token_key(a, base + i) : gptr(keys)[base + i];
    atomicAdd(&hist[(k >> shift) & (BINS - 1)], 1u);
  }
  __syncthreads();
  gptr(a.table)[(int64_t)threadIdx.x * gridDim.x + blockIdx.x] = hist[threadIdx.x];
}

// Workgroup d: exclusive sums over the blocks of digit d's counts, in place, and
// the digit's total behind the table.
__global__ __launch_bounds__(256) void sort_scan_kernel(uint32_t* table, int blocks) {
  __shared__ uint32_t part[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t* const row = table + (int64_t)blockIdx.x * blocks;
  uint32_t carry = 0;
  for (int i0 = 0; i0 < blocks; i0 += 256) {
    const uint32_t v = i0 + tid < blocks ? gptr(row)[i0 + tid] : 0;
    uint32_t x = v;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const uint32_t y = (uint32_t)__shfl_up((int)x, off, 64);
      if (lane >= off) x += y;
    }
    if (lane == 63) part[wave] = x;
    __syncthreads();
    uint32_t base = carry;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if (w < wave) base += part[w];
      carry += part[w];
    }
    if (i0 + tid < blocks) gptr(row)[i0 + tid] = base + x - v;
    __syncthreads();
  }
  if (tid == 0) gptr(table)[(int64_t)BINS * blocks + blockIdx.x] = carry;
}

template <bool FIRST>
__global__ __launch_bounds__(SORT_THREADS) void sort_place_kernel(EmbedGradArgs a, int shift, const uint32_t* keys,
                                                                  const uint32_t* index, uint32_t* keys_out,
                                                                  uint32_t* index_out) {
  constexpr int NW = SORT_THREADS / 64, R = SORT_TILE / SORT_THREADS;
  static_assert(SORT_THREADS == BINS, "a thread for each digit");
  __shared__ uint32_t hist[NW][BINS], part[BINS / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int i = tid; i < NW * BINS; i += SORT_THREADS) (&hist[0][0])[i] = 0;
  const int64_t base = (int64_t)blockIdx.x * SORT_TILE + (int64_t)wave * (R * 64);
  const int64_t left = a.tokens - base;
  const int n = left < 0 ? 0 : left > R * 64 ? R * 64 : (int)left;
  uint32_t key[R], idx[R], rank[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    key[r] = idx[r] = 0;
    const int i = r * 64 + lane;
    if (i < n) {
      key[r] = FIRST ? token_key(a, base + i) : gptr(keys)[base + i];
      idx[r] = FIRST ? (uint32_t)(base + i) : gptr(index)[base + i];
    }
  }
  __syncthreads();
  wave_ranks(key, shift, R, n, lane, hist[wave], rank);
  const uint32_t start = bins_exclusive(gptr(a.table)[(int64_t)BINS * gridDim.x + tid], tid, part);
  {   // thread d: places of digit d's keys, wave after wave
    uint32_t at = start + gptr(a.table)[(int64_t)tid * gridDim.x + blockIdx.x];
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const uint32_t c = hist[w][tid];
      hist[w][tid] = at;
      at += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < R; ++r)
    if (r * 64 + lane < n) {
      const uint32_t p = hist[wave][(key[r] >> shift) & (BINS - 1)] + rank[r];
      gptr(keys_out)[p] = key[r];
      gptr(index_out)[p] = idx[r];
    }
}

__global__ __launch_bounds__(256) void embed_segments_kernel(EmbedGradArgs a) {
  const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (j >= a.tokens) return;
  const uint32_t k = gptr(a.keys)[j];
  if (k >= (uint32_t)a.vocab) return;
  if (j == 0 || gptr(a.keys)[j - 1] != k) gptr(a.seg)[2 * (int64_t)k] = (uint32_t)j;
  if (j + 1 == a.tokens || gptr(a.keys)[j + 1] != k) gptr(a.seg)[2 * (int64_t)k + 1] = (uint32_t)(j + 1);
}

// Zeros for FILL_VECS x 1024 groups of four columns from block b's on.
template <class TO>
__device__ __forceinline__ void fill_rows(const EmbedGradArgs& a, int64_t b) {
  const op_f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  TO* const out = static_cast<TO*>(a.dtable);
  // Rows without gaps are one long row.
  const bool one = a.dtable_ld == a.width;
  const int64_t width = one ? a.vocab * a.width : a.width, per = (width + 3) / 4, all = one ? per : per * a.vocab;
#pragma unroll
  for (int u = 0; u < FILL_VECS; ++u) {
    const int64_t i = (b * FILL_VECS + u) * 1024 + threadIdx.x;
    if (i < all) {
      const int64_t row = one ? 0 : i / per;
      row_store4(out + row * a.dtable_ld, 4 * (i - row * per), width, zero);
    }
  }
}

// Up to SORT_ONE tokens (what its registers hold; 8000 tokens, 50257 x 768: 38 us, and 62 by
// the kernels above): all passes in the LDS of workgroup 0, and the segments.
// Wave w's keys are a run of them, so ranks by wave are stable.  Meanwhile the
// other workgroups fill the table with zeros: a sort of 8000 tokens takes one CU 17 us
// (ids of two digits; 27 of three), the rest of the chip 26 to 36 for the 200 MB of a table.
template <class TO>
__global__ __launch_bounds__(1024) void sort_one_kernel(EmbedGradArgs a, int bits, uint32_t* keys_out, uint32_t* order_out) {
  constexpr int NW = 16, R = SORT_ONE / 1024;
  __shared__ uint32_t skey[SORT_ONE];
  __shared__ uint16_t sidx[SORT_ONE];
  __shared__ uint32_t hist[NW][BINS], part[BINS / 64];
  if (blockIdx.x > 0) {
    fill_rows<TO>(a, blockIdx.x - 1);
    return;
  }
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int tokens = (int)a.tokens;
  const int rounds = (tokens + 1023) / 1024;
  const int base = wave * rounds * 64;
  const int left = tokens - base, n = left < 0 ? 0 : left < rounds * 64 ? left : rounds * 64;
  uint32_t key[R], idx[R], rank[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    key[r] = 0;
    idx[r] = (uint32_t)(base + r * 64 + lane);
    if (r * 64 + lane < n) key[r] = token_key(a, base + r * 64 + lane);
  }
  for (int shift = 0; shift < bits; shift += DIGIT) {
    for (int i = tid; i < NW * BINS; i += 1024) (&hist[0][0])[i] = 0;
    __syncthreads();
    wave_ranks(key, shift, rounds, n, lane, hist[wave], rank);
    __syncthreads();
    uint32_t total = 0;
    if (tid < BINS)
#pragma unroll
      for (int w = 0; w < NW; ++w) total += hist[w][tid];
    uint32_t at = bins_exclusive(tid < BINS ? total : 0, tid, part);
    if (tid < BINS)
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const uint32_t c = hist[w][tid];
        hist[w][tid] = at;
        at += c;
      }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (r * 64 + lane < n) {
        const uint32_t p = hist[wave][(key[r] >> shift) & (BINS - 1)] + rank[r];
        skey[p] = key[r];
        sidx[p] = (uint16_t)idx[r];
      }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (r * 64 + lane < n) {
        key[r] = skey[base + r * 64 + lane];
        idx[r] = sidx[base + r * 64 + lane];
      }
  }
#pragma unroll
  for (int r = 0; r < R; ++r)
    if (r * 64 + lane < n) {
      const int j = base + r * 64 + lane;
      const uint32_t k = key[r];
      gptr(keys_out)[j] = k;
      gptr(order_out)[j] = idx[r];
      if (k < (uint32_t)a.vocab) {
        if (j == 0 || skey[j - 1] != k) gptr(a.seg)[2 * (int64_t)k] = (uint32_t)j;
        if (j + 1 == tokens || skey[j + 1] != k) gptr(a.seg)[2 * (int64_t)k + 1] = (uint32_t)(j + 1);
      }
    }
}

// --------------------------------------------------------------------- sums
// s += up to 8 rows of grad, whose loads are all in flight together; at(u) is
// the u-th token's number (wave-uniform, u < n).  (16 rows in flight were slower, 4 no
// faster.  For the second gradient above, 8 columns a lane of bf16 instead of 4: 285 -> 320
// us; whole rows of three strips a wave: 277 -> 305; registers then leave room for fewer waves.)
template <class TG, class At>
__device__ __forceinline__ void add_rows(op_f32x4& s, const TG* grad, int64_t ld, int n, int c0, int lane, int width,
                                         At&& at) {
  op_f32x4 v[8];
#pragma unroll
  for (int u = 0; u < 8; ++u) {
    v[u] = op_f32x4{0.f, 0.f, 0.f, 0.f};
    if (u < n) v[u] = row_load4(grad + (int64_t)at(u) * ld, c0 + 4 * lane, width);
  }
#pragma unroll
  for (int u = 0; u < 8; ++u)
    if (u < n)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] += v[u][e];
}

// Rows order[j .. end) of grad, columns of one strip, added in that order.
template <class TG>
__device__ __forceinline__ op_f32x4 sum_rows(const TG* grad, int64_t ld, const uint32_t* order, int64_t j, int64_t end,
                                             int c0, int lane, int width) {
  op_f32x4 s = {0.f, 0.f, 0.f, 0.f};
  for (; j < end; j += 64) {
    const int n = end - j < 64 ? (int)(end - j) : 64;
    const uint32_t mine = lane < n ? gptr(order)[j + lane] : 0;   // 64 tokens' numbers in one load
    for (int i = 0; i < n; i += 8)
      add_rows(s, grad, ld, n - i < 8 ? n - i : 8, c0, lane, width,
                    [&](int u) { return (uint32_t)__builtin_amdgcn_readlane((int)mine, i + u); });
  }
  return s;
}

template <class TO>
__device__ __forceinline__ void finish_row(const EmbedGradArgs& a, TO* out, int c0, int lane, op_f32x4 x) {
  if (a.accumulate) {
    const op_f32x4 old = row_load4(out, c0 + 4 * lane, a.width);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = old[i] + a.scale * x[i];
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] *= a.scale;
  }
  row_store4(out, c0 + 4 * lane, a.width, x);
}

// The strips of a row are neighbouring waves: a row of a gradient is then read as a
// whole (rows and strips in different dimensions of the grid: 284 us at 491520 x 768
// bf16, so 269).  The grid's waves, W a workgroup, run through x and then y, since
// either takes fewer than 2^32 threads.
template <int W>
__device__ __forceinline__ uint32_t wave_of_grid() {
  return (blockIdx.y * gridDim.x + blockIdx.x) * W + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
}
template <int W>
static dim3 waves_grid(int64_t waves) {
  const int64_t blocks = (waves + W - 1) / W, x = blocks < (1 << 24) / W ? blocks : (1 << 24) / W;
  return dim3((unsigned)x, (unsigned)((blocks + x - 1) / x));
}

// A chunk of the sorted tokens, one strip: partial sums of the segments longer than a
// chunk.  Such a segment holds the chunk's first or last token, so a chunk has two
// slots: 0 for the segment its first token belongs to, 1 for one that starts after it.
template <class TG>
__device__ __forceinline__ void chunk_sums(const EmbedGradArgs& a, int64_t chunk, int c0, int lane) {
  const int64_t j0 = chunk * a.chunk, j1 = j0 + a.chunk < a.tokens ? j0 + a.chunk : a.tokens;
  const uint32_t first = a.keys[j0], last = a.keys[j1 - 1];
  float* part = a.part + chunk * 2 * a.part_ld + c0 + 4 * lane;
  const TG* grad = static_cast<const TG*>(a.grad);
  if (first < (uint32_t)a.vocab) {
    const int64_t s = a.seg[2 * (int64_t)first], e = a.seg[2 * (int64_t)first + 1];
    if (e - s > a.chunk) store4(part, sum_rows(grad, a.grad_ld, a.order, j0, e < j1 ? e : j1, c0, lane, a.width));
  }
  if (last != first && last < (uint32_t)a.vocab) {
    const int64_t s = a.seg[2 * (int64_t)last], e = a.seg[2 * (int64_t)last + 1];
    if (e - s > a.chunk) store4(part + a.part_ld, sum_rows(grad, a.grad_ld, a.order, s, j1, c0, lane, a.width));
  }
}

// GROUP chunks of one row, one strip: their sums in one.  (Padding may be half of all tokens.)
__global__ __launch_bounds__(256) void embed_group_kernel(EmbedGradArgs a) {
  const uint32_t w = wave_of_grid<4>(), strips = (uint32_t)(a.width + STRIP - 1) / STRIP;
  const int64_t g = w / strips, j0 = g * GROUP * a.chunk;
  const int c = (int)(w % strips) * STRIP + 4 * (threadIdx.x & 63);
  if (g >= a.chunks / GROUP) return;
  const uint32_t v = a.keys[j0];
  if (v >= (uint32_t)a.vocab) return;
  if (a.seg[2 * (int64_t)v + 1] < j0 + GROUP * a.chunk) return;
  const float* p = a.part + g * GROUP * 2 * a.part_ld + c;
  op_f32x4 y[GROUP];
#pragma unroll
  for (int i = 0; i < GROUP; ++i) y[i] = load4(p + i * 2 * a.part_ld);
#pragma unroll
  for (int i = 1; i < GROUP; ++i) y[0] += y[i];
  store4(a.groups + g * a.part_ld + c, y[0]);
}

// The sums that make up row v, [s, e) of the sorted tokens, and piece q of `of` of them:
// its chunks, or groups in the place of the chunks they hold.
struct RowParts {
  int64_t s, k0, n0, g0, ng, n;
  __device__ __forceinline__ RowParts(const EmbedGradArgs& a, int64_t s_, int64_t e) : s(s_), k0(s_ / a.chunk) {
    const int64_t k1 = (e - 1) / a.chunk + 1, width = (int64_t)GROUP * a.chunk;
    g0 = (s + width - 1) / width;
    ng = a.groups ? e / width - g0 : 0;
    if (ng < 0) ng = 0;
    n0 = ng > 0 ? g0 * GROUP - k0 : k1 - k0;
    n = ng > 0 ? n0 + ng + k1 - (g0 + ng) * GROUP : n0;
  }
  __device__ __forceinline__ op_f32x4 sum(const EmbedGradArgs& a, int q, int of, int c) const {
    op_f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int64_t i = n * q / of; i < n * (q + 1) / of; ++i) {
      const int64_t k = i < n0 ? k0 + i : k0 + i + ng * (GROUP - 1);
      const float* p = i >= n0 && i < n0 + ng ? a.groups + (g0 + i - n0) * a.part_ld
                                              : a.part + (2 * k + (s > k * a.chunk ? 1 : 0)) * a.part_ld;
      x += load4(p + c);
    }
    return x;
  }
};

// Rows of more than a chunk, one strip: a wave joins the row that starts in its chunk,
// if one does (it holds the chunk's last token).  A row of more than JOIN_ALONE parts
// is left to the workgroup, whose waves take a run of them each.
template <class TO>
__global__ __launch_bounds__(64 * JOIN_WAVES) void embed_join_kernel(EmbedGradArgs a) {
  __shared__ op_f32x4 sums[JOIN_WAVES][64];
  __shared__ uint32_t large[JOIN_WAVES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c0 = blockIdx.y * STRIP;
  const int64_t chunk = (int64_t)blockIdx.x * JOIN_WAVES + wave;
  uint32_t left = (uint32_t)a.vocab;
  if (chunk < a.chunks) {
    const int64_t j0 = chunk * a.chunk, j1 = j0 + a.chunk < a.tokens ? j0 + a.chunk : a.tokens;
    const uint32_t v = a.keys[j1 - 1];
    if (v < (uint32_t)a.vocab) {
      const int64_t s = a.seg[2 * (int64_t)v], e = a.seg[2 * (int64_t)v + 1];
      if (s >= j0 && e - s > a.chunk) {
        const RowParts r(a, s, e);
        if (r.n > JOIN_ALONE) left = v;
        else finish_row(a, static_cast<TO*>(a.dtable) + (int64_t)v * a.dtable_ld, c0, lane, r.sum(a, 0, 1, c0 + 4 * lane));
      }
    }
  }
  if (lane == 0) large[wave] = left;
  __syncthreads();
  for (int w = 0; w < JOIN_WAVES; ++w) {
    const uint32_t v = __builtin_amdgcn_readfirstlane(large[w]);
    if (v >= (uint32_t)a.vocab) continue;
    sums[wave][lane] = RowParts(a, a.seg[2 * (int64_t)v], a.seg[2 * (int64_t)v + 1]).sum(a, wave, JOIN_WAVES, c0 + 4 * lane);
    __syncthreads();
    if (wave == 0) {
      op_f32x4 x = sums[0][lane];
#pragma unroll
      for (int q = 1; q < JOIN_WAVES; ++q) x += sums[q][lane];
      finish_row(a, static_cast<TO*>(a.dtable) + (int64_t)v * a.dtable_ld, c0, lane, x);
    }
    __syncthreads();
  }
}

// Up to FIRST_MOST tokens: no sort.  A workgroup for each token and strip looks
// the tokens over, an eighth of them a wave; if its token is the first with its
// id, the waves sum the rows they met and join the sums in the tokens' order.
// Rows without tokens are zeros already.
template <class TG, class TO>
__global__ __launch_bounds__(512) void embed_first_kernel(EmbedGradArgs a) {
  constexpr int NW = 8, G = FIRST_MOST / 64 / NW;
  __shared__ op_f32x4 sums[NW][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t0 = blockIdx.x, c0 = blockIdx.y * STRIP, tokens = (int)a.tokens;
  const int64_t v = load_id(a.ids, a.wide_ids, t0);
  if (v < 0 || v >= a.vocab) return;
  const int groups = (tokens + 64 * NW - 1) / (64 * NW), base = wave * groups * 64;
  uint64_t met[G];
  bool earlier = false;
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const int t = base + g * 64 + lane;
    const bool same = g < groups && t < tokens && load_id(a.ids, a.wide_ids, t) == v;
    earlier |= same && t < t0;
    met[g] = __ballot(same);
  }
  if (__syncthreads_or(earlier)) return;
  op_f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int g = 0; g < G; ++g) {
    uint64_t m = met[g];
    while (m) {
      const int n = __popcll(m);
      uint32_t t[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        t[u] = m ? (uint32_t)(base + g * 64 + __builtin_ctzll(m)) : 0;
        m &= m - 1;   // 0 stays 0
      }
      add_rows(x, static_cast<const TG*>(a.grad), a.grad_ld, n < 8 ? n : 8, c0, lane, a.width, [&](int u) { return t[u]; });
    }
  }
  sums[wave][lane] = x;
  __syncthreads();
  if (wave != 0) return;
#pragma unroll
  for (int w = 1; w < NW; ++w) x += sums[w][lane];
  finish_row(a, static_cast<TO*>(a.dtable) + v * a.dtable_ld, c0, lane, x);
}

template <class TO>
__global__ __launch_bounds__(1024) void embed_fill_kernel(EmbedGradArgs a) {
  fill_rows<TO>(a, blockIdx.x);
}

// A wave takes a row and a strip.  (Several neighbouring rows a wave: frequent ids are
// neighbours, 268 -> 274 us with two and 322 with four.)  How it comes by the row and its tokens is one of three:
enum Source {
  EVERY,      // every row of the table, with its segment of the sorted tokens (empty: zeros)
  MET,        // every sorted token that is the first of its row (the other rows are zeros already)
  LOOK        // every row, written anew; few tokens, all of which the wave looks over itself
};
// Waves of a workgroup.  Rows of unequal length go better by one (491520 x 768: 263 us with
// four, 256 with one), waves of which most have nothing to do by four (8192 x 1024: 42.8 and 44.4).
template <int SOURCE>
constexpr int ROW_WAVES = SOURCE == EVERY ? 1 : 4;
template <class TG, class TO, int SOURCE>
__global__ __launch_bounds__(64 * ROW_WAVES<SOURCE>) void embed_rows_kernel(EmbedGradArgs a) {
  const int lane = threadIdx.x & 63;
  const uint32_t w = wave_of_grid<ROW_WAVES<SOURCE>>(), strips = (uint32_t)(a.width + STRIP - 1) / STRIP;
  const int c0 = (int)(w % strips) * STRIP;
  if (SOURCE != LOOK && w / strips < (uint32_t)a.chunks) return chunk_sums<TG>(a, w / strips, c0, lane);
  const int64_t i = w / strips - (SOURCE != LOOK ? a.chunks : 0);
  op_f32x4 x = {0.f, 0.f, 0.f, 0.f};
  int64_t v = i;
  if constexpr (SOURCE == LOOK) {
    if (i >= a.vocab) return;
    uint64_t met[FEW / 64], any = 0;
#pragma unroll
    for (int b = 0; b < FEW / 64; ++b) {
      const int t = b * 64 + lane;
      met[b] = b * 64 < a.tokens ? __ballot(t < a.tokens && load_id(a.ids, a.wide_ids, t) == v) : 0;
      any |= met[b];
    }
    if (any) {
#pragma unroll
      for (int b = 0; b < FEW / 64; ++b) {
        uint64_t m = met[b];
        while (m) {
          const int n = __popcll(m);
          uint32_t t[8];
#pragma unroll
          for (int u = 0; u < 8; ++u) {
            t[u] = m ? (uint32_t)(b * 64 + __builtin_ctzll(m)) : 0;
            m &= m - 1;   // 0 stays 0
          }
          add_rows(x, static_cast<const TG*>(a.grad), a.grad_ld, n < 8 ? n : 8, c0, lane, a.width, [&](int u) { return t[u]; });
        }
      }
    }
  } else {
    int64_t s, e;
    if constexpr (SOURCE == MET) {
      if (i >= a.tokens) return;
      const uint32_t k = a.keys[i];
      if (k >= (uint32_t)a.vocab || (i > 0 && a.keys[i - 1] == k)) return;
      v = k;
      s = i;
      e = a.seg[2 * v + 1];
    } else {
      if (i >= a.vocab) return;
      s = a.seg[2 * v];
      e = a.seg[2 * v + 1];
      if (s == e && a.accumulate) return;
    }
    if (e - s > a.chunk) return;   // joined later
    if (s != e) x = sum_rows(static_cast<const TG*>(a.grad), a.grad_ld, a.order, s, e, c0, lane, a.width);
  }
  finish_row(a, static_cast<TO*>(a.dtable) + v * a.dtable_ld, c0, lane, x);
}

}  // namespace

// -------------------------------------------------------------------- launch
hipError_t launch_embed_lookup(EmbedLookupArgs a, bool table_f32, bool out_f32, hipStream_t s) {
  a.lanes_log2 = 0;
  while (a.lanes_log2 < 6 && (4 << a.lanes_log2) < a.width) ++a.lanes_log2;
  const int64_t blocks = (a.tokens + (256 >> a.lanes_log2) - 1) / (256 >> a.lanes_log2);
  const dim3 grid((unsigned)blocks), threads(256);
  if (table_f32 && out_f32) hipLaunchKernelGGL((embed_lookup_kernel<float, float>), grid, threads, 0, s, a);
  else if (table_f32) hipLaunchKernelGGL((embed_lookup_kernel<float, bf16_t>), grid, threads, 0, s, a);
  else if (out_f32) hipLaunchKernelGGL((embed_lookup_kernel<bf16_t, float>), grid, threads, 0, s, a);
  else hipLaunchKernelGGL((embed_lookup_kernel<bf16_t, bf16_t>), grid, threads, 0, s, a);
  return hipGetLastError();
}

EmbedGradLayout embed_grad_layout(int64_t tokens, int64_t vocab, int64_t width) {
  EmbedGradLayout L = {};
  auto take = [&](size_t bytes) {
    const size_t at = L.bytes;
    L.bytes += (bytes + 255) & ~size_t(255);
    return at;
  };
  if (tokens <= FEW) return L;
  // Shorter chunks have more sums to join, longer ones a longer last wave.  Measured: 20000
  // x 100 in chunks of 16, 32, 64: 49, 49, 58 us; 491520 x 768 in 32, 64, 128: 289, 269, 263.
  L.chunk = 16;
  while (tokens / L.chunk >= 4096) L.chunk *= 2;
  L.blocks = (tokens + SORT_TILE - 1) / SORT_TILE;
  L.part_ld = (width + STRIP - 1) / STRIP * STRIP;
  for (size_t& k : L.keys) k = take(4 * size_t(tokens));
  for (size_t& k : L.index) k = take(4 * size_t(tokens));
  L.table = take(4 * size_t(BINS) * (L.blocks + 1));
  L.seg = take(8 * size_t(vocab));
  const int64_t chunks = (tokens + L.chunk - 1) / L.chunk;
  L.part = take(8 * size_t(chunks) * L.part_ld);
  if (chunks >= 1024) L.groups = take(4 * size_t(chunks / GROUP) * L.part_ld);
  return L;
}

template <class TG, class TO, int SOURCE>
static void rows_typed(const EmbedGradArgs& a, hipStream_t s) {
  const int64_t rows = SOURCE == MET ? a.tokens : a.vocab;
  const unsigned strips = (unsigned)((a.width + STRIP - 1) / STRIP);
  hipLaunchKernelGGL((embed_rows_kernel<TG, TO, SOURCE>), waves_grid<ROW_WAVES<SOURCE>>((a.chunks + rows) * strips),
                     dim3(64 * ROW_WAVES<SOURCE>), 0, s, a);
  if (SOURCE == LOOK) return;
  if (a.groups) hipLaunchKernelGGL(embed_group_kernel, waves_grid<4>(a.chunks / GROUP * strips), dim3(256), 0, s, a);
  hipLaunchKernelGGL((embed_join_kernel<TO>), dim3((unsigned)((a.chunks + JOIN_WAVES - 1) / JOIN_WAVES), strips),
                     dim3(64 * JOIN_WAVES), 0, s, a);
}

// Workgroups that fill the table with zeros.
static unsigned fill_blocks(const EmbedGradArgs& a) {
  const int64_t vecs = a.dtable_ld == a.width ? (a.vocab * a.width + 3) / 4 : a.vocab * ((a.width + 3) / 4);
  return (unsigned)((vecs + FILL_VECS * 1024 - 1) / (FILL_VECS * 1024));
}

template <class TG, class TO>
static void grad_typed(EmbedGradArgs a, const EmbedGradLayout& L, char* ws, hipStream_t s) {
  const unsigned strips = (unsigned)((a.width + STRIP - 1) / STRIP);
  // One launch while the rows' looks at all tokens are few.  Measured, us in one launch and
  // in the two below: 256 tokens, 1173 x 429: 10.5 and 13; 64, 50257 x 768: 23.6 and 23.9;
  // 256, 50257 x 768: 32 and 24.
  if (a.tokens <= FEW && !a.accumulate && a.vocab * a.tokens <= LOOK_MOST) return rows_typed<TG, TO, LOOK>(a, s);
  // The search for the first token of an id grows with the square of the tokens, and
  // what it saves (the sort) is hidden where a large table is filled with zeros at the
  // same time.  Measured: 1000 tokens, 1173 x 429: 14 us and 24 sorted; 2048, 40298 x 39:
  // 15 and 30; 4096, 1173 x 429: 39 and 31; 1000, 50257 x 768: 35 and 32.
  const bool first = a.tokens <= FIRST_MOST && a.tokens * strips <= FIRST_MOST &&
                     (a.accumulate || a.vocab * a.width * (int64_t)sizeof(TO) <= (int64_t)64 << 20);
  if (a.tokens <= FEW || first) {
    if (!a.accumulate) hipLaunchKernelGGL((embed_fill_kernel<TO>), dim3(fill_blocks(a)), dim3(1024), 0, s, a);
    hipLaunchKernelGGL((embed_first_kernel<TG, TO>), dim3((unsigned)a.tokens, strips), dim3(512), 0, s, a);
    return;
  }
  uint32_t* keys[2] = {reinterpret_cast<uint32_t*>(ws + L.keys[0]), reinterpret_cast<uint32_t*>(ws + L.keys[1])};
  uint32_t* index[2] = {reinterpret_cast<uint32_t*>(ws + L.index[0]), reinterpret_cast<uint32_t*>(ws + L.index[1])};
  a.table = reinterpret_cast<uint32_t*>(ws + L.table);
  a.seg = reinterpret_cast<uint32_t*>(ws + L.seg);
  a.part = reinterpret_cast<float*>(ws + L.part);
  a.part_ld = L.part_ld;
  a.chunk = L.chunk;
  a.chunks = (a.tokens + a.chunk - 1) / a.chunk;
  if (L.groups) a.groups = reinterpret_cast<float*>(ws + L.groups);
  int bits = 1;   // keys run up to vocab
  while ((int64_t(1) << bits) <= a.vocab) ++bits;
  int to = 0;
  const bool one = a.tokens <= SORT_ONE;
  if (one) {
    const unsigned fill = a.accumulate ? 0 : fill_blocks(a);
    hipLaunchKernelGGL((sort_one_kernel<TO>), dim3(1 + fill), dim3(1024), 0, s, a, bits, keys[0], index[0]);
    to = 1;
  } else {
    const dim3 grid((unsigned)L.blocks), threads(SORT_THREADS);
    for (int shift = 0; shift < bits; shift += DIGIT, to ^= 1) {
      const uint32_t *k = keys[to ^ 1], *i = index[to ^ 1];
      if (shift == 0) hipLaunchKernelGGL(sort_count_kernel<true>, grid, threads, 0, s, a, shift, k);
      else hipLaunchKernelGGL(sort_count_kernel<false>, grid, threads, 0, s, a, shift, k);
      hipLaunchKernelGGL(sort_scan_kernel, dim3(BINS), dim3(256), 0, s, a.table, int(L.blocks));
      if (shift == 0) hipLaunchKernelGGL(sort_place_kernel<true>, grid, threads, 0, s, a, shift, k, i, keys[to], index[to]);
      else hipLaunchKernelGGL(sort_place_kernel<false>, grid, threads, 0, s, a, shift, k, i, keys[to], index[to]);
    }
  }
  a.keys = keys[to ^ 1];
  a.order = index[to ^ 1];
  if (!one) hipLaunchKernelGGL(embed_segments_kernel, dim3((unsigned)((a.tokens + 255) / 256)), dim3(256), 0, s, a);
  if (one) rows_typed<TG, TO, MET>(a, s);
  else rows_typed<TG, TO, EVERY>(a, s);
}

hipError_t launch_embed_grad(const EmbedGradArgs& a, const EmbedGradLayout& L, char* ws, bool grad_f32, bool out_f32,
                             hipStream_t s) {
  if (grad_f32 && out_f32) grad_typed<float, float>(a, L, ws, s);
  else if (grad_f32) grad_typed<float, bf16_t>(a, L, ws, s);
  else if (out_f32) grad_typed<bf16_t, float>(a, L, ws, s);
  else grad_typed<bf16_t, bf16_t>(a, L, ws, s);
  return hipGetLastError();
}

}  // namespace malt
