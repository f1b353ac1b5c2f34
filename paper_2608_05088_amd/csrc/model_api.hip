// C entry points of the operators in front of the layers and behind them: the norm, the head's loss,
// AdamW.  What the kernels take for granted is checked here, on the host, before anything is
// enqueued.
#include <math.h>

#include <algorithm>
#include <new>
#include <numeric>
#include <vector>

#include "adamw.h"
#include "block_fp8.h"
#include "head.h"
#include "norm.h"
#include "ops_check.h"

using namespace malt;

namespace {

struct Buf {
  const void* p;
  size_t n;
};

bool number(double x) { return x >= -1.7976931348623157e308 && x <= 1.7976931348623157e308; }

// ------------------------------------------------------------------------ AdamW
// Buffers of a call, sorted: no written one may overlap another.
struct Span {
  uintptr_t at, end;
  bool written;
};

malt_status_t check_spans(std::vector<Span>& spans) {
  std::sort(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.at < b.at; });
  uintptr_t read_end = 0, write_end = 0;
  for (const Span& s : spans) {
    if (s.at < write_end || (s.written && s.at < read_end))
      return fail(MALT_ERR_ALIAS, "two of the tensors overlap, or one is named twice");
    uintptr_t& e = s.written ? write_end : read_end;
    if (s.end > e) e = s.end;
  }
  return MALT_OK;
}

malt_status_t check_adam_tensor(int i, int64_t n, const void* state, int bits) {
  if (n < 0 || n > ADAM_MAX_NUMEL) return fail(MALT_ERR_SHAPE, "tensor %d: %lld elements", i, (long long)n);
  if (bits != 8 && bits != 32) return fail(MALT_ERR_INVALID_ARG, "tensor %d: moments of %d bits (8 and 32 there are)", i, bits);
  if (n > 0 && !state) return fail(MALT_ERR_INVALID_ARG, "tensor %d: state is NULL", i);
  if (!op_aligned(state, 4)) return fail(MALT_ERR_ALIGNMENT, "tensor %d: state is not 4-byte aligned", i);
  return MALT_OK;
}

// Tensors by launches: `run` is called with each launch's arguments and grid.
template <class Fill, class Run>
malt_status_t adam_launches(AdamArgs& a, int count, const int64_t* numel, Fill&& fill, Run&& run) {
  int64_t chunks = 0;
  a.count = 0;
  a.first = 0;
  auto flush = [&]() -> malt_status_t {
    if (a.count == 0) return MALT_OK;
    const hipError_t e = run(a, (uint32_t)chunks);
    a.count = 0;
    chunks = 0;
    return e == hipSuccess ? MALT_OK : hip_fail(e, "launching the AdamW step");
  };
  for (int i = 0; i < count; ++i) {
    const int64_t own = (numel[i] + ADAM_CHUNK - 1) / ADAM_CHUNK;
    if (own == 0) continue;
    // A grid holds fewer than 2^32 threads, 256 a chunk; a launch's tensors are neighbours in the call.
    if (a.count > 0 && (a.count == ADAM_TENSORS || chunks + own > (int64_t(1) << 23) || a.first + a.count != i)) MALT_TRY(flush());
    if (a.count == 0) a.first = i;
    a.chunk[a.count] = (uint32_t)chunks;
    fill(a.t[a.count], i);
    ++a.count;
    chunks += own;
  }
  return flush();
}

// ------------------------------------------------------------------------- head
constexpr int64_t kHeadRows = 65536, kHeadInner = 65536, kHeadVocab = int64_t(1) << 22, kHeadWeight = int64_t(1) << 33;
constexpr int64_t kHeadPiece = int64_t(1) << 28;   // elements of a piece's dz, of its transpose and of W^T's piece, all planes

int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

struct HeadPlan {
  bool few;              // the first pass in one launch on the weights as they lie
  bool grads;
  bool halves;           // logits from float16 planes
  int x_halves, w_halves;
  bool pack_w;           // otherwise the products read the weights as they lie
  int dz_planes, dx_z, dx_w, dw_z, dw_x;   // bf16 planes of the gradients' products
  int64_t rows_pad, cols_pad;
  int64_t piece;         // vocabulary columns of a piece, a multiple of the tile
  int pieces;
  bool turn_pieces;      // W^T is packed by pieces, in one place
  int first_edge, second_edge, grad_edge;   // of the tiles
  int parts;             // of a row's statistics
  int dx_splits, dw_splits;   // parts of the gradients' contractions
  size_t partial, at_label, records, x, w, x_scales, w_scales, x_t, w_t, dz, dz_t, dx, dw, bytes;
};

// Pairs of planes that make a product of `na` by `nb` planes (of two or three at most), small ones first.
void head_pairs(HeadProduct& g, int na, int nb, int planes) {
  g.pairs = 0;
  g.pair_a = g.pair_b = 0;
  for (int s = planes - 1; s >= 0; --s)
    for (int i = s < na ? s : na - 1; i >= 0; --i) {
      const int j = s - i;
      if (j >= nb) break;
      g.pair_a |= (uint32_t)i << (4 * g.pairs);
      g.pair_b |= (uint32_t)j << (4 * g.pairs);
      ++g.pairs;
    }
}
int head_pair_count(int na, int nb, int planes) {
  HeadProduct g;
  head_pairs(g, na, nb, planes);
  return g.pairs;
}

// The tiles' edge of a pass over rows x cols logits, from what tiles take.  A CU runs one tile of 256 at a time, 1.43 us
// a stage, or two of 128, 0.78; `big` and `small`: what is done after the stages, in us.  us, tiles of 128 | 256:
//   first pass   300 x 1000 x 64 6 | 11, 512 x 50257 x 768 45 | 52, 8192 x 50257 x 768 659 | 622
//   second       300 x 1000 x 64 9 | 26, 2000 x 12000 x 768 54 | 62, 8192 x 50257 x 1280 762 | 660 (half of it; by now 586)
int head_edge(int64_t rows, int64_t cols, int64_t stages, double big, double small) {
  auto rounds = [&](int64_t e) { return double((up(rows, e) / e * (up(cols, e) / e) + 255) / 256); };
  if (rounds(256) > 64) return 256;   // little to win, and a row's statistics take twice the workspace
  return 0.5 * rounds(128) * (0.78 * double(stages) + small) < rounds(256) * (1.43 * double(stages) + big) ? 128 : 256;
}

// Parts for dx's contraction where dW's tiles, `small` stages each, fill the CUs that dx's parts leave free and
// follow them: those that end first by this count, one workgroup a CU.  A tile's epilogue counts as 6 stages, `extra`
// what a part costs in writing and reading it.  us a step, against even shares: 3000 x 20000 x 1000 in float32 2024 | 2187,
// 400 x 30000 x 1024 621 | 646, 1001 x 50257 x 901 2034 | 2020 (idle CUs leave the others power), bf16 within 1%.
int head_parts(int64_t tiles, int64_t stages, int64_t small_tiles, int64_t small, double extra, int64_t most) {
  double best = 0;
  int at = 0;
  for (int64_t n = 1; n <= most && n * tiles <= 256; ++n) {
    const int64_t l1 = (stages + n - 1) / n + 6, l2 = small + 6, busy = n * tiles;
    auto done = [&](int64_t t) { return (256 - busy) * (t / l2) + busy * ((t - l1) / l2); };
    int64_t t = l1;
    while (done(t) < small_tiles) t = std::min((t / l2 + 1) * l2, t + l2 - (t - l1) % l2);
    const double cost = double(t) + extra * double(n > 1 ? n : 0);
    if (at == 0 || cost < best) {
      best = cost;
      at = int(n);
    }
  }
  return at;
}

HeadPlan head_plan(const malt_linear_loss_t& a) {
  HeadPlan L = {};
  const bool x32 = a.x_type == MALT_FLOAT32, w32 = a.weight_type == MALT_FLOAT32;
  L.few = a.rows <= HEAD_FEW;
  L.grads = a.dx || a.dweight;
  L.halves = x32 || w32;
  L.x_halves = x32 ? HEAD_HALVES : 1;
  L.w_halves = w32 ? HEAD_HALVES : 1;
  // Planes of dz and of the other side, by the result's type.  bf16: one of dz, whose rounding is of the result's
  // own size (together 1.41 times it); two below 2^32 products, where that costs under 10 us.  The other side's
  // float32 values: two, since a third rounding would make that 1.73.
  const bool dw32 = a.dweight_type == MALT_FLOAT32;
  const int coarse = double(a.rows) * double(a.vocab) * double(a.inner) < 0x1p32 ? 2 : 1;
  L.dx_z = x32 ? HEAD_PLANES : coarse;
  L.dx_w = w32 ? (x32 ? HEAD_PLANES : 2) : 1;
  L.dw_z = dw32 ? HEAD_PLANES : coarse;
  L.dw_x = x32 ? (dw32 ? HEAD_PLANES : 2) : 1;
  L.dz_planes = std::max(a.dx ? L.dx_z : 1, a.dweight ? L.dw_z : 1);
  L.rows_pad = up(a.rows, HEAD_TILE);
  L.cols_pad = up(a.inner, HEAD_BK);
  // As they lie: rows of whole stages, 16-byte pieces, a tile's offsets in 32 bits.
  L.pack_w = L.halves || a.inner % HEAD_BK || a.ldw % 8 || a.ldw > (int64_t(1) << 22) || !op_aligned(a.weight, 16);
  size_t end = 0;
  auto take = [&](size_t bytes) {
    const size_t at = end;
    end += align256(bytes);
    return at;
  };
  const int64_t stages = L.cols_pad / HEAD_BK * head_pair_count(L.x_halves, L.w_halves, HEAD_HALVES);
  L.first_edge = head_edge(a.rows, a.vocab, stages, 8.5, 3.8);
  L.parts = L.few ? head_few_parts(a.vocab, a.inner) : int(up(a.vocab, L.first_edge) / L.first_edge);
  if (!a.stats_given) {
    L.partial = take(size_t(a.rows) * L.parts * 8);
    L.at_label = take(size_t(a.rows) * 4);
  }
  if (a.rows > 0 && (L.grads || !L.few)) {
    L.x = take(size_t(L.x_halves) * L.rows_pad * L.cols_pad * 2);
    if (L.pack_w) L.w = take(size_t(L.w_halves) * up(a.vocab, HEAD_TILE) * L.cols_pad * 2);
    if (L.halves) {
      L.x_scales = take(size_t(L.rows_pad) * 4);
      L.w_scales = take(size_t(up(a.vocab, HEAD_TILE)) * 4);
    }
  }
  if (L.grads) {
    // Pieces of like size, as few as keep dz and W^T within their shares of memory.  Half the share would be 7% slower (8192 x
    // 50257 x 1280 in bf16: 3890 -> 4150 us a step in twice the pieces, 1024 x 131072 x 2048 in float32 8650 -> 9620).
    // W^T is packed at once where all of it is within its share (a launch for each piece: 3890 -> 3930), by pieces otherwise
    // (1024 x 131072 x 2048 in float32: 3.6 -> 2.0 GB of workspace, 8650 -> 8710 us).
    const int64_t all = up(a.vocab, HEAD_TILE), across_w = a.dx && a.rows > 0 ? up(a.inner, HEAD_TILE) * L.dx_w : 0;
    L.turn_pieces = across_w * all > kHeadPiece;
    const int64_t column = std::max(L.rows_pad * L.dz_planes, L.turn_pieces ? across_w : 0);   // elements
    int64_t most = L.rows_pad > 0 ? kHeadPiece / column / HEAD_TILE * HEAD_TILE : all;
    if (most < HEAD_TILE) most = HEAD_TILE;
    const int64_t pieces = (all + most - 1) / most;
    L.piece = up((all + pieces - 1) / pieces, HEAD_TILE);
    // Whole rounds of 256 CUs before the last piece's (8192 rows x 50257: 13 and 12 instead of 13 and 13).
    const int64_t whole = 256 / std::gcd(L.rows_pad / HEAD_TILE, int64_t(256)) * HEAD_TILE;
    if (pieces > 1 && up(L.piece, whole) <= most) L.piece = up(L.piece, whole);
    L.pieces = int((all + L.piece - 1) / L.piece);
    L.records = take(size_t(L.rows_pad) * sizeof(HeadRow));
    if (a.dx) {
      L.w_t = take(size_t(across_w) * (L.turn_pieces ? L.piece : all) * 2);
      L.dz = take(size_t(L.dz_planes) * L.rows_pad * L.piece * 2);
    }
    if (a.dweight) {
      L.x_t = take(size_t(L.dw_x) * up(a.inner, HEAD_TILE) * L.rows_pad * 2);
      L.dz_t = take(size_t(L.dz_planes) * L.rows_pad * L.piece * 2);
    }
    // A product of few tiles and a long contraction is cut into parts, so that no workgroup has more
    // stages than a CU's share of them all, and 16 at the least (a part costs its tile in float32, written and read).
    const int64_t dx_stages = L.piece / HEAD_BK * head_pair_count(L.dx_z, L.dx_w, x32 ? HEAD_PLANES : 2);
    const int64_t dw_stages = up(a.rows, HEAD_BK) / HEAD_BK *
                              head_pair_count(L.dw_z, L.dw_x, dw32 ? HEAD_PLANES : 2);
    L.second_edge = head_edge(a.rows, std::min(L.piece, a.vocab), stages, 4 + 14 * L.dz_planes, 4 + 9 * L.dz_planes);
    // Of the gradients: by their stages of 256-tiles on each of 256 CUs.  us, tiles of 128 | 256: 500 x 2000 x 2000 (below 36) 24 | 35,
    // 2000 x 12000 x 768 (35) 83 | 101, 512 x 50257 x 768 (37) 119 | 119, 400 x 30000 x 1024 in float32 (165) 401 | 330.
    const int64_t wide = up(a.inner, HEAD_TILE) / HEAD_TILE;
    const int64_t work = wide * ((a.dx ? L.rows_pad / HEAD_TILE * dx_stages : 0) + (a.dweight ? L.piece / HEAD_TILE * dw_stages : 0));
    L.grad_edge = work <= 36 * 256 ? 128 : 256;
    const int64_t across = up(a.inner, L.grad_edge) / L.grad_edge;
    const int64_t dx_tiles = a.dx ? up(a.rows, L.grad_edge) / L.grad_edge * across : 0, dw_tiles = a.dweight ? L.piece / L.grad_edge * across : 0;
    int64_t share = (dx_tiles * dx_stages + dw_tiles * dw_stages) / (L.grad_edge == 256 ? 256 : 512);
    if (share < 16) share = 16;
    auto parts = [&](int64_t stages, int64_t contraction) {
      int64_t n = (stages + share - 1) / share;
      if (n > contraction / HEAD_BK) n = contraction / HEAD_BK;
      return int(n < 1 ? 1 : n > 64 ? 64 : n);
    };
    L.dx_splits = a.dx ? parts(dx_stages, L.piece) : 1;
    L.dw_splits = a.dweight ? parts(dw_stages, a.rows) : 1;
    if (L.grad_edge == 256 && a.dx && a.dweight && L.dw_splits == 1) {
      const double extra = double(a.rows) * double(a.inner) * 8 / 5.1e6 / 1.43;   // stages
      const int n = head_parts(dx_tiles, dx_stages, dw_tiles, dw_stages, extra, std::min<int64_t>(64, L.piece / HEAD_BK));
      if (n > 0) L.dx_splits = n;
    }
    if (a.dx && (L.pieces > 1 || L.dx_splits > 1)) L.dx = take(size_t(L.dx_splits) * a.rows * a.inner * 4);
    if (L.dw_splits > 1) L.dw = take(size_t(L.dw_splits) * L.piece * a.inner * 4);
  }
  L.bytes = end;
  return L;
}

// A packed operand of `rows` (a multiple of the tile) by `cols` (of the stage).
HeadSide packed_side(const uint16_t* p, int64_t rows, int64_t cols) {
  return {p, rows * cols, cols / HEAD_BK * HEAD_BLOCK, HEAD_BLOCK, HEAD_BK, rows};
}

malt_status_t check_head(const malt_linear_loss_t* a) {
  if (!a) return fail(MALT_ERR_INVALID_ARG, "args is NULL");
  if (a->rows < 0 || a->rows > kHeadRows) return fail(MALT_ERR_SHAPE, "%lld rows (at most %lld)", (long long)a->rows, (long long)kHeadRows);
  if (a->inner < 1 || a->inner > kHeadInner) return fail(MALT_ERR_SHAPE, "rows of %lld values (at most %lld)", (long long)a->inner, (long long)kHeadInner);
  if (a->vocab < 1 || a->vocab > kHeadVocab || a->vocab > kHeadWeight / a->inner)
    return fail(MALT_ERR_SHAPE, "a weight of %lld x %lld", (long long)a->vocab, (long long)a->inner);
  // A grid holds fewer than 2^32 threads, 512 for each 256 x 256 tile.
  if (a->rows > 0 && up(a->rows, HEAD_TILE) * up(a->vocab, HEAD_TILE) > (int64_t(1) << 38))
    return fail(MALT_ERR_SHAPE, "%lld rows over a vocabulary of %lld", (long long)a->rows, (long long)a->vocab);
  const Mat x = {"x", a->x, a->x_type, a->rows, a->inner, a->ldx}, w = {"weight", a->weight, a->weight_type, a->vocab, a->inner, a->ldw},
            dx = {"dx", a->dx, a->x_type, a->rows, a->inner, a->lddx},
            dw = {"dweight", a->dweight, a->dweight_type, a->vocab, a->inner, a->lddw};
  MALT_TRY(check_mat(x));
  MALT_TRY(check_mat(w));
  MALT_TRY(check_ids("labels", a->labels, a->label_type, a->rows));
  if (a->label_stride < 0 || a->label_stride > kMaxPitch) return fail(MALT_ERR_SHAPE, "labels: stride %lld", (long long)a->label_stride);
  if (a->dx) MALT_TRY(check_mat(dx));
  if (a->dweight) MALT_TRY(check_mat(dw));
  if (a->accumulate != 0 && a->accumulate != 1) return fail(MALT_ERR_INVALID_ARG, "accumulate must be 0 or 1");
  if (a->stats_given != 0 && a->stats_given != 1) return fail(MALT_ERR_INVALID_ARG, "stats_given must be 0 or 1");
  if (a->stats_given && !a->stats && a->rows > 0) return fail(MALT_ERR_INVALID_ARG, "stats is NULL");
  if (a->stats_given && a->losses) return fail(MALT_ERR_INVALID_ARG, "losses are formed with the statistics, not from them");
  if (!a->losses && !a->stats && !a->dx && !a->dweight) return fail(MALT_ERR_INVALID_ARG, "nothing is wanted");
  if (a->weights && (a->weight_stride < 0 || a->weight_stride > kMaxPitch)) return fail(MALT_ERR_SHAPE, "weights: stride %lld", (long long)a->weight_stride);
  if (!op_aligned(a->losses, 4) || !op_aligned(a->weights, 4)) return fail(MALT_ERR_ALIGNMENT, "losses or weights not 4-byte aligned");
  if (!op_aligned(a->stats, 16)) return fail(MALT_ERR_ALIGNMENT, "stats not 16-byte aligned");
  const size_t rows = size_t(a->rows);
  const size_t label_bytes = rows ? ((rows - 1) * a->label_stride + 1) * (a->label_type == MALT_INT64 ? 8 : 4) : 0;
  const size_t weight_bytes = a->weights && rows ? ((rows - 1) * a->weight_stride + 1) * 4 : 0;
  const Buf out[] = {{a->losses, a->losses ? 4 * rows : 0}, {a->stats, a->stats && !a->stats_given ? rows * sizeof(HeadRow) : 0},
                     {a->dx, a->dx ? dx.bytes() : 0}, {a->dweight, a->dweight ? dw.bytes() : 0}};
  const Buf in[] = {{a->x, x.bytes()}, {a->weight, w.bytes()}, {a->labels, label_bytes}, {a->weights, weight_bytes},
                    {a->stats, a->stats_given ? rows * sizeof(HeadRow) : 0}};
  for (int i = 0; i < 4; ++i) {
    for (const Buf& b : in)
      if (op_overlap(out[i].p, out[i].n, b.p, b.n)) return fail(MALT_ERR_ALIAS, "an output overlaps an input");
    for (int j = 0; j < i; ++j)
      if (op_overlap(out[i].p, out[i].n, out[j].p, out[j].n)) return fail(MALT_ERR_ALIAS, "two outputs overlap");
  }
  return MALT_OK;
}

}  // namespace

extern "C" {

// ------------------------------------------------------------------------ AdamW
malt_status_t malt_adamw_state_size(int64_t numel, int32_t bits, size_t* bytes) {
  if (!bytes) return fail(MALT_ERR_INVALID_ARG, "output pointer is NULL");
  MALT_TRY(check_adam_tensor(0, numel, bytes, bits));
  *bytes = size_t(adam_state_bytes(numel, bits));
  return MALT_OK;
}

malt_status_t malt_adamw_step(const malt_adamw_tensors_t* t, const malt_adamw_t* h, void* stream) {
  if (!t || !h) return fail(MALT_ERR_INVALID_ARG, "args is NULL");
  if (t->count < 0) return fail(MALT_ERR_INVALID_ARG, "%d tensors", t->count);
  if (t->count > 0 && (!t->numel || !t->params || !t->param_types || !t->grads || !t->grad_types || !t->states || !t->state_bits))
    return fail(MALT_ERR_INVALID_ARG, "a list of the tensors is NULL");
  if (!(h->lr >= 0 && number(h->lr))) return fail(MALT_ERR_INVALID_ARG, "lr must be a number, 0 or more");
  if (!(h->beta1 >= 0 && h->beta1 < 1 && h->beta2 >= 0 && h->beta2 < 1)) return fail(MALT_ERR_INVALID_ARG, "betas must be in [0, 1)");
  if (!((float)h->eps >= 0x1p-126f && number(h->eps))) return fail(MALT_ERR_INVALID_ARG, "eps must be at least 2^-126");
  if (!(h->weight_decay >= 0 && number(h->weight_decay))) return fail(MALT_ERR_INVALID_ARG, "weight_decay must be a number, 0 or more");
  if (h->step < 1) return fail(MALT_ERR_INVALID_ARG, "step counts from 1 (got %lld)", (long long)h->step);
  if (!number(h->grad_scale)) return fail(MALT_ERR_INVALID_ARG, "grad_scale must be a number");
  if (!op_aligned(h->grad_scale_at, 4)) return fail(MALT_ERR_ALIGNMENT, "grad_scale_at is not 4-byte aligned");
  try {
    std::vector<Span> spans;
    spans.reserve(3 * size_t(t->count) + 1);
    auto span = [&](const void* p, size_t n, bool written) {
      if (n) spans.push_back({reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + n, written});
    };
    for (int i = 0; i < t->count; ++i) {
      const int64_t n = t->numel[i];
      MALT_TRY(check_adam_tensor(i, n, t->states[i], t->state_bits[i]));
      const Mat p = {"param", t->params[i], t->param_types[i], 1, n, n}, g = {"grad", t->grads[i], t->grad_types[i], 1, n, n};
      for (const Mat* m : {&p, &g}) {
        if (!op_dtype_ok(m->type)) return fail(MALT_ERR_INVALID_ARG, "tensor %d: %s: unknown element type %d", i, m->name, m->type);
        if (n > 0 && !m->p) return fail(MALT_ERR_INVALID_ARG, "tensor %d: %s is NULL", i, m->name);
        if (!op_aligned(m->p, m->elem())) return fail(MALT_ERR_ALIGNMENT, "tensor %d: %s is not aligned to its elements", i, m->name);
      }
      span(p.p, p.bytes(), true);
      span(g.p, g.bytes(), false);
      span(t->states[i], size_t(adam_state_bytes(n, t->state_bits[i])), true);
    }
    span(h->grad_scale_at, h->grad_scale_at ? 4 : 0, false);
    MALT_TRY(check_spans(spans));
  } catch (const std::bad_alloc&) {
    return fail(MALT_ERR_HIP, "out of host memory");
  }
  AdamArgs a;
  a.b1 = (float)h->beta1;
  a.c1 = (float)(1.0 - h->beta1);
  a.b2 = (float)h->beta2;
  a.c2 = (float)(1.0 - h->beta2);
  a.shrink = (float)(1.0 - h->lr * h->weight_decay);
  a.rate = (float)(h->lr / (1.0 - pow(h->beta1, (double)h->step)));
  a.root = (float)(1.0 / sqrt(1.0 - pow(h->beta2, (double)h->step)));
  a.eps = (float)h->eps;
  a.grad_scale = (float)h->grad_scale;
  a.grad_scale_at = h->grad_scale_at;
  a.seed_lo = (uint32_t)h->seed;
  a.seed_hi = (uint32_t)(h->seed >> 32);
  return adam_launches(
      a, t->count, t->numel,
      [&](AdamTensor& d, int i) {
        d.param = t->params[i];
        d.grad = t->grads[i];
        d.state = t->states[i];
        d.numel = t->numel[i] | (t->param_types[i] == MALT_FLOAT32 ? ADAM_P_F32 : 0) |
                  (t->grad_types[i] == MALT_FLOAT32 ? ADAM_G_F32 : 0) | (t->state_bits[i] == 8 ? ADAM_8BIT : 0);
      },
      [&](const AdamArgs& args, uint32_t chunks) { return launch_adamw(args, chunks, static_cast<hipStream_t>(stream)); });
}

malt_status_t malt_adamw_moments(int32_t count, const int64_t* numel, const void* const* states, float* const* moments, void* stream) {
  if (count < 0) return fail(MALT_ERR_INVALID_ARG, "%d tensors", count);
  if (count > 0 && (!numel || !states || !moments)) return fail(MALT_ERR_INVALID_ARG, "a list of the tensors is NULL");
  try {
    std::vector<Span> spans;
    spans.reserve(2 * size_t(count));
    for (int i = 0; i < count; ++i) {
      MALT_TRY(check_adam_tensor(i, numel[i], states[i], 8));
      if (numel[i] == 0) continue;
      if (!moments[i]) return fail(MALT_ERR_INVALID_ARG, "tensor %d: moments is NULL", i);
      if (!op_aligned(moments[i], 4)) return fail(MALT_ERR_ALIGNMENT, "tensor %d: moments not 4-byte aligned", i);
      const uintptr_t s = reinterpret_cast<uintptr_t>(states[i]), m = reinterpret_cast<uintptr_t>(moments[i]);
      spans.push_back({s, s + size_t(adam_state_bytes(numel[i], 8)), false});
      spans.push_back({m, m + 8 * size_t(numel[i]), true});
    }
    MALT_TRY(check_spans(spans));
  } catch (const std::bad_alloc&) {
    return fail(MALT_ERR_HIP, "out of host memory");
  }
  AdamArgs a = {};
  return adam_launches(
      a, count, numel,
      [&](AdamTensor& d, int i) {
        d.param = moments[i];
        d.grad = nullptr;
        d.state = const_cast<void*>(states[i]);
        d.numel = numel[i];
      },
      [&](const AdamArgs& args, uint32_t chunks) { return launch_adamw_moments(args, chunks, static_cast<hipStream_t>(stream)); });
}

// ------------------------------------------------------------------------- norm
malt_status_t malt_rms_norm(const malt_rms_norm_t* p, void* stream) {
  if (!p) return fail(MALT_ERR_INVALID_ARG, "args is NULL");
  // One workgroup for each row at most, 1024 threads: a grid holds fewer than 2^32 threads.
  if (p->rows < 0 || p->rows > (int64_t(1) << 21)) return fail(MALT_ERR_SHAPE, "%lld rows", (long long)p->rows);
  if (p->width < 1 || p->width > NORM_MAX_WIDTH) return fail(MALT_ERR_SHAPE, "rows of %lld values (at most %lld)", (long long)p->width, (long long)NORM_MAX_WIDTH);
  if (!(p->eps >= 0 && number(p->eps))) return fail(MALT_ERR_INVALID_ARG, "eps must be a number, 0 or more");
  const Mat x = {"x", p->x, p->type, p->rows, p->width, p->ldx}, r = {"residual", p->residual, p->type, p->rows, p->width, p->ldr},
            s = {"sum", p->sum, p->type, p->rows, p->width, p->lds}, y = {"y", p->y, p->y_type, p->rows, p->width, p->ldy},
            w = {"weight", p->weight, p->weight_type, 1, p->width, p->width};
  MALT_TRY(check_mat(x));
  MALT_TRY(check_mat(w));
  if (!p->residual != !p->sum) return fail(MALT_ERR_INVALID_ARG, "residual and sum come together");
  if (p->residual) {
    MALT_TRY(check_mat(r));
    MALT_TRY(check_mat(s));
  }
  if (!p->values != !p->scales) return fail(MALT_ERR_INVALID_ARG, "values and scales come in pairs");
  if (!p->y == !p->values && p->rows > 0) return fail(MALT_ERR_INVALID_ARG, "the output is y or values and scales");
  if (p->y) MALT_TRY(check_mat(y));
  if (!op_aligned(p->values, 16) || !op_aligned(p->scales, 16)) return fail(MALT_ERR_ALIGNMENT, "8-bit values or scales not 16-byte aligned");
  if (!op_aligned(p->rstd, 4)) return fail(MALT_ERR_ALIGNMENT, "rstd is not 4-byte aligned");
  if (p->rows == 0) return MALT_OK;
  const size_t nv = p->values ? size_t(p->rows) * q_pad(p->width) : 0, ns = p->values ? size_t(q_pad(p->width) / QB) * q_scale_rows(p->rows) : 0;
  const Buf out[] = {{p->sum, p->sum ? s.bytes() : 0}, {p->y, p->y ? y.bytes() : 0}, {p->values, nv}, {p->scales, ns},
                     {p->rstd, p->rstd ? 4 * size_t(p->rows) : 0}};
  const Buf in[] = {{p->x, x.bytes()}, {p->residual, p->residual ? r.bytes() : 0}, {p->weight, w.bytes()}};
  for (int i = 0; i < 5; ++i) {
    for (const Buf& b : in)
      if (op_overlap(out[i].p, out[i].n, b.p, b.n)) return fail(MALT_ERR_ALIAS, "an output overlaps an input");
    for (int j = 0; j < i; ++j)
      if (op_overlap(out[i].p, out[i].n, out[j].p, out[j].n)) return fail(MALT_ERR_ALIAS, "two outputs overlap");
  }
  NormArgs a = {};
  a.x = p->x;
  a.residual = p->residual;
  a.weight = p->weight;
  a.sum = p->sum;
  a.y = p->y;
  a.values = static_cast<uint8_t*>(p->values);
  a.scales = static_cast<uint8_t*>(p->scales);
  a.rstd = p->rstd;
  a.rows = p->rows;
  a.ldx = p->ldx;
  a.ldr = p->ldr;
  a.lds = p->lds;
  a.ldy = p->ldy;
  a.width = (int32_t)p->width;
  a.w_f32 = p->weight_type == MALT_FLOAT32;
  a.y_f32 = p->y_type == MALT_FLOAT32;
  a.eps = p->eps;
  return launched(launch_norm(a, p->type == MALT_FLOAT32, static_cast<hipStream_t>(stream)), "launching the norm");
}

malt_status_t malt_rms_norm_grad_size(int64_t rows, int64_t width, int32_t need_dweight, size_t* workspace_bytes) {
  if (!workspace_bytes) return fail(MALT_ERR_INVALID_ARG, "output pointer is NULL");
  if (rows < 0 || rows > (int64_t(1) << 21)) return fail(MALT_ERR_SHAPE, "%lld rows", (long long)rows);
  if (width < 1 || width > NORM_MAX_WIDTH) return fail(MALT_ERR_SHAPE, "rows of %lld values (at most %lld)", (long long)width, (long long)NORM_MAX_WIDTH);
  *workspace_bytes = need_dweight ? size_t(norm_grad_parts(rows, width)) * width * 4 : 0;
  return MALT_OK;
}

malt_status_t malt_rms_norm_grad(const malt_rms_norm_grad_t* p, void* workspace, size_t workspace_bytes, void* stream) {
  if (!p) return fail(MALT_ERR_INVALID_ARG, "args is NULL");
  size_t need;
  MALT_TRY(malt_rms_norm_grad_size(p->rows, p->width, p->dweight != nullptr, &need));
  const Mat h = {"h", p->h, p->type, p->rows, p->width, p->ldh}, dy = {"dy", p->dy, p->dy_type, p->rows, p->width, p->lddy},
            ds = {"dsum", p->dsum, p->type, p->rows, p->width, p->ldds}, dx = {"dx", p->dx, p->type, p->rows, p->width, p->lddx},
            w = {"weight", p->weight, p->weight_type, 1, p->width, p->width}, dw = {"dweight", p->dweight, p->weight_type, 1, p->width, p->width};
  MALT_TRY(check_mat(h));
  MALT_TRY(check_mat(dy));
  MALT_TRY(check_mat(w));
  if (p->dsum) MALT_TRY(check_mat(ds));
  if (p->dx) MALT_TRY(check_mat(dx));
  if (p->dweight) MALT_TRY(check_mat(dw));
  if (!p->dx && !p->dweight) return fail(MALT_ERR_INVALID_ARG, "neither dx nor dweight is wanted");
  if (p->rows > 0 && !p->rstd) return fail(MALT_ERR_INVALID_ARG, "rstd is NULL");
  if (!op_aligned(p->rstd, 4)) return fail(MALT_ERR_ALIGNMENT, "rstd is not 4-byte aligned");
  MALT_TRY(check_workspace(workspace, workspace_bytes, need));
  const Buf out[] = {{p->dx, p->dx ? dx.bytes() : 0}, {p->dweight, p->dweight ? dw.bytes() : 0}, {workspace, need}};
  const Buf in[] = {{p->h, h.bytes()}, {p->dy, dy.bytes()}, {p->dsum, p->dsum ? ds.bytes() : 0}, {p->weight, w.bytes()}, {p->rstd, 4 * size_t(p->rows)}};
  for (int i = 0; i < 3; ++i) {
    for (const Buf& b : in)
      if (op_overlap(out[i].p, out[i].n, b.p, b.n)) return fail(MALT_ERR_ALIAS, "an output or the workspace overlaps an input");
    for (int j = 0; j < i; ++j)
      if (op_overlap(out[i].p, out[i].n, out[j].p, out[j].n)) return fail(MALT_ERR_ALIAS, "two outputs overlap, or one and the workspace");
  }
  NormGradArgs a = {};
  a.h = p->h;
  a.weight = p->weight;
  a.rstd = p->rstd;
  a.dy = p->dy;
  a.dsum = p->dsum;
  a.dx = p->dx;
  a.partial = p->dweight ? static_cast<float*>(workspace) : nullptr;
  a.dweight = p->dweight;
  a.rows = p->rows;
  a.ldh = p->ldh;
  a.ldy = p->lddy;
  a.lds = p->ldds;
  a.ldx = p->lddx;
  a.width = (int32_t)p->width;
  a.parts = norm_grad_parts(p->rows, p->width);
  a.w_f32 = p->weight_type == MALT_FLOAT32;
  a.dy_f32 = p->dy_type == MALT_FLOAT32;
  return launched(launch_norm_grad(a, p->type == MALT_FLOAT32, static_cast<hipStream_t>(stream)), "launching the norm's gradient");
}

// ------------------------------------------------------------------------- head
malt_status_t malt_linear_loss_size(const malt_linear_loss_t* args, size_t* workspace_bytes) {
  if (!workspace_bytes) return fail(MALT_ERR_INVALID_ARG, "output pointer is NULL");
  MALT_TRY(check_head(args));
  *workspace_bytes = head_plan(*args).bytes;
  return MALT_OK;
}

malt_status_t malt_linear_loss(const malt_linear_loss_t* args, void* workspace, size_t workspace_bytes, void* stream_) {
  MALT_TRY(check_head(args));
  const malt_linear_loss_t& a = *args;
  const HeadPlan L = head_plan(a);
  MALT_TRY(check_workspace(workspace, workspace_bytes, L.bytes));
  const size_t rows = size_t(a.rows);
  const Mat x = {"x", a.x, a.x_type, a.rows, a.inner, a.ldx}, w = {"weight", a.weight, a.weight_type, a.vocab, a.inner, a.ldw},
            dx = {"dx", a.dx, a.x_type, a.rows, a.inner, a.lddx}, dw = {"dweight", a.dweight, a.dweight_type, a.vocab, a.inner, a.lddw};
  const Buf others[] = {{a.x, x.bytes()}, {a.weight, w.bytes()},
                        {a.labels, rows ? ((rows - 1) * a.label_stride + 1) * (a.label_type == MALT_INT64 ? 8 : 4) : 0},
                        {a.weights, a.weights && rows ? ((rows - 1) * a.weight_stride + 1) * 4 : 0},
                        {a.losses, a.losses ? 4 * rows : 0}, {a.stats, a.stats ? rows * sizeof(HeadRow) : 0},
                        {a.dx, a.dx ? dx.bytes() : 0}, {a.dweight, a.dweight ? dw.bytes() : 0}};
  for (const Buf& b : others)
    if (op_overlap(workspace, L.bytes, b.p, b.n)) return fail(MALT_ERR_ALIAS, "workspace overlaps another buffer");
  if (a.rows == 0 && (!a.dweight || a.accumulate)) return MALT_OK;
  const hipStream_t s = static_cast<hipStream_t>(stream_);
  char* const ws = static_cast<char*>(workspace);
  const bool per_row = a.weights && a.weight_stride > 0;   // one for all rows is a factor of the result
  const HeadLabels labels = {a.labels, a.label_type == MALT_INT64, a.label_stride, per_row ? a.weights : nullptr, a.weight_stride};
  const bool f32x = a.x_type == MALT_FLOAT32, f32w = a.weight_type == MALT_FLOAT32;
  if (L.grads || !L.few) MALT_TRY(launched(head_setup(), "raising the head's LDS limit"));

  // What is packed: the logits' sides, and for the gradients the transposes.
  const bool want_dx = a.dx && a.rows > 0, want_dw = a.dweight && a.rows > 0;
  HeadPrepare prepare = {};
  prepare.halves = L.halves;
  prepare.scales[0] = reinterpret_cast<float*>(ws + L.x_scales);
  prepare.scales[1] = reinterpret_cast<float*>(ws + L.w_scales);
  HeadSide wside = {static_cast<const uint16_t*>(a.weight), 0, HEAD_TILE * a.ldw, HEAD_BK, (int32_t)a.ldw, a.vocab}, w_t = {}, x_t = {};
  if (a.rows > 0 && (L.grads || !L.few)) {
    HeadPack x = {}, w = {};
    x.x = a.x;
    x.rows = a.rows;
    x.cols = w.cols = a.inner;
    x.ld = a.ldx;
    x.labels = labels;
    x.finite = w.finite = L.halves;
    x.vocab = a.vocab;
    w.x = a.weight;
    w.rows = a.vocab;
    w.ld = a.ldw;
    auto straight = [&](HeadPack p, size_t at, int64_t rows, int planes) {
      p.out = reinterpret_cast<uint16_t*>(ws + at);
      p.out_rows = rows;
      p.out_cols = L.cols_pad;
      p.plane = rows * L.cols_pad;
      p.planes = planes;
      return p;
    };
    auto turned = [&](HeadPack p, size_t at, int64_t cols, int planes) {
      p.out = reinterpret_cast<uint16_t*>(ws + at);
      p.out_rows = a.inner;
      p.out_cols = cols;
      p.plane = up(a.inner, HEAD_TILE) * cols;
      p.planes = planes;
      return p;
    };
    prepare.part[0] = straight(x, L.x, L.rows_pad, L.x_halves);
    prepare.part[0].labels.weights = nullptr;   // the losses of rows without weight are formed all the same
    if (want_dw) {
      prepare.part[1] = turned(x, L.x_t, L.rows_pad, L.dw_x);
      x_t = packed_side(prepare.part[1].out, up(a.inner, HEAD_TILE), L.rows_pad);
      x_t.rows = a.inner;
    }
    if (L.pack_w) {
      prepare.part[2] = straight(w, L.w, up(a.vocab, HEAD_TILE), L.w_halves);
      wside = packed_side(prepare.part[2].out, up(a.vocab, HEAD_TILE), L.cols_pad);
    }
    if (want_dx) {
      const int64_t cols = L.turn_pieces ? L.piece : up(a.vocab, HEAD_TILE);   // the last piece's may end before it does
      prepare.part[3] = turned(w, L.w_t, cols, L.dx_w);
      prepare.part[3].rows = std::min(cols, a.vocab);
      w_t = packed_side(prepare.part[3].out, up(a.inner, HEAD_TILE), cols);
      w_t.rows = a.inner;
    }
    MALT_TRY(launched(launch_head_prepare(prepare, f32x, f32w, s), "packing the head's operands"));
  }

  HeadLogits z = {};
  z.g.a = packed_side(reinterpret_cast<const uint16_t*>(ws + L.x), L.rows_pad, L.cols_pad);
  z.g.b = wside;
  z.g.m = (int32_t)a.rows;
  z.g.k = L.cols_pad;
  head_pairs(z.g, L.x_halves, L.w_halves, HEAD_HALVES);
  if (L.halves) {
    z.x_scales = prepare.scales[0];
    z.w_scales = prepare.scales[1];
  }
  z.rows = labels;
  z.vocab = a.vocab;
  HeadRow* const records = reinterpret_cast<HeadRow*>(ws + L.records);
  z.records = records;
  if (a.rows > 0 && !a.stats_given) {
    malt_f32x2* const partial = reinterpret_cast<malt_f32x2*>(ws + L.partial);
    float* const at_label = reinterpret_cast<float*>(ws + L.at_label);
    if (L.few) {
      HeadFew f = {};
      f.x = a.x;
      f.w = a.weight;
      f.ldx = a.ldx;
      f.ldw = a.ldw;
      f.vocab = a.vocab;
      f.m = (int32_t)a.rows;
      f.k = (int32_t)a.inner;
      f.parts = L.parts;
      f.rows = labels;
      f.partial = partial;
      f.at_label = at_label;
      MALT_TRY(launched(launch_head_few(f, f32x, f32w, s), "launching the head's logits of few rows"));
    } else {
      HeadLogits first = z;
      first.g.n = (int32_t)a.vocab;
      first.g.tiles_m = int(up(a.rows, L.first_edge) / L.first_edge);
      first.g.tiles_n = int(up(a.vocab, L.first_edge) / L.first_edge);
      first.partial = partial;
      first.at_label = at_label;
      first.parts = L.parts;
      MALT_TRY(launched(launch_head_logits(first, L.first_edge, false, s), "launching the head's logits"));
    }
    const HeadJoin join = {labels, a.rows, L.rows_pad, a.vocab, partial, L.parts, at_label, reinterpret_cast<HeadRow*>(a.stats),
                           L.grads ? records : nullptr, a.losses};
    MALT_TRY(launched(launch_head_join(join, s), "joining the head's statistics"));
  }
  if (!L.grads) return MALT_OK;
  if (a.rows > 0 && a.stats_given)
    MALT_TRY(launched(launch_head_records(labels, a.rows, L.rows_pad, a.vocab, reinterpret_cast<const HeadRow*>(a.stats), records, s),
                      "preparing the head's rows"));

  HeadGrads gr = {};
  gr.records = records;
  gr.scale = a.weights ? 1.f : a.weight_value;
  gr.scale_at = per_row ? nullptr : a.weights;
  uint16_t *const dz = reinterpret_cast<uint16_t*>(ws + L.dz), *const dz_t = reinterpret_cast<uint16_t*>(ws + L.dz_t);
  for (int p = 0; p < L.pieces; ++p) {
    const int64_t v0 = p * L.piece, n = a.vocab - v0 < L.piece ? a.vocab - v0 : L.piece;
    if (want_dx && L.turn_pieces && p > 0) {
      HeadPrepare next = {};
      next.part[3] = prepare.part[3];
      next.part[3].x = static_cast<const char*>(a.weight) + size_t(v0) * a.ldw * w.elem();
      next.part[3].rows = n;
      MALT_TRY(launched(launch_head_prepare(next, f32x, f32w, s), "packing a piece of the head's weight"));
    }
    if (a.rows > 0) {
      HeadLogits second = z;
      second.g.b.p += v0 / HEAD_TILE * wside.tile;
      second.g.b.rows -= v0;
      second.g.n = (int32_t)n;
      second.g.tiles_m = int(up(a.rows, L.second_edge) / L.second_edge);
      second.g.tiles_n = int(up(n, L.second_edge) / L.second_edge);
      second.col0 = v0;
      if (L.halves) second.w_scales += v0;
      second.dz = a.dx ? dz : nullptr;
      second.dz_t = a.dweight ? dz_t : nullptr;
      second.dz_plane = L.rows_pad * L.piece;
      second.dz_tile = L.piece / HEAD_BK * HEAD_BLOCK;
      second.dz_t_tile = L.rows_pad / HEAD_BK * HEAD_BLOCK;
      second.dz_planes = L.dz_planes;
      MALT_TRY(launched(launch_head_logits(second, L.second_edge, true, s), "launching the logits' gradient"));
    }
    gr.parts = 0;
    if (want_dx) {
      HeadOut& o = gr.part[gr.parts++];
      o = HeadOut{};
      o.g.a = packed_side(dz, L.rows_pad, L.piece);
      o.g.b = w_t;
      if (!L.turn_pieces) o.g.b.p += v0 / HEAD_BK * HEAD_BLOCK;
      o.g.m = (int32_t)a.rows;
      o.g.n = (int32_t)a.inner;
      o.g.k = n;
      o.g.tiles_m = int(up(a.rows, L.grad_edge) / L.grad_edge);
      o.g.tiles_n = int(up(a.inner, L.grad_edge) / L.grad_edge);
      head_pairs(o.g, L.dx_z, L.dx_w, f32x ? HEAD_PLANES : 2);
      o.out = a.dx;
      o.ldo = a.lddx;
      o.partial = reinterpret_cast<float*>(ws + L.dx);
      o.splits = L.dx_splits;
      o.add_partial = p > 0;
      o.write_partial = o.splits > 1 || p + 1 < L.pieces;
      o.f32 = f32x;
      o.mask_rows = true;
    }
    if (a.dweight) {
      HeadOut& o = gr.part[gr.parts++];
      o = HeadOut{};
      const bool fine = a.dweight_type == MALT_FLOAT32;
      o.g.a = packed_side(dz_t, L.piece, L.rows_pad);
      o.g.b = x_t;
      o.g.m = (int32_t)n;
      o.g.n = (int32_t)a.inner;
      o.g.k = a.rows;
      o.g.tiles_m = int(up(n, L.grad_edge) / L.grad_edge);
      o.g.tiles_n = int(up(a.inner, L.grad_edge) / L.grad_edge);
      head_pairs(o.g, L.dw_z, L.dw_x, fine ? HEAD_PLANES : 2);
      o.out = static_cast<char*>(a.dweight) + v0 * a.lddw * op_dtype_bytes(a.dweight_type);
      o.ldo = a.lddw;
      o.partial = reinterpret_cast<float*>(ws + L.dw);
      o.splits = L.dw_splits;
      o.write_partial = o.splits > 1;
      o.f32 = fine;
      o.accumulate = a.accumulate != 0;
    }
    MALT_TRY(launched(launch_head_grads(gr, L.grad_edge, s), "launching the head's gradients"));
    bool sums[2] = {false, false};
    for (int i = 0; i < gr.parts; ++i) sums[i] = gr.part[i].splits > 1 && (!gr.part[i].mask_rows || p + 1 == L.pieces);
    MALT_TRY(launched(launch_head_sum(gr, sums[0], sums[1], s), "joining the head's gradients"));
  }
  return MALT_OK;
}

}  // extern "C"
