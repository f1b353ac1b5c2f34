// C entry points of the operators around the optimizer step: what the kernels
// take for granted is checked here, on the host, before anything is enqueued.
#include <math.h>

#include "block_fp8.h"
#include "distill.h"
#include "embed.h"
#include "ops_check.h"

using namespace malt;

namespace {

// A grid holds fewer than 2^32 threads: 64 for each token or table row, 1024 for
// each row of logits, 512 for each 256 x 256 output tile.
constexpr int64_t kMaxTokens = int64_t(1) << 25;
constexpr int64_t kMaxRows = int64_t(1) << 21;
constexpr int64_t kMaxVocab = int64_t(1) << 30;
constexpr int64_t kMaxBlockDim = int64_t(1) << 22;
constexpr int64_t kMaxProduct = int64_t(1) << 37;

malt_status_t check_table(int64_t tokens, int64_t vocab, int64_t width) {
  if (tokens < 0 || tokens > kMaxTokens) return fail(MALT_ERR_SHAPE, "%lld tokens", (long long)tokens);
  if (vocab < 1 || vocab > kMaxTokens) return fail(MALT_ERR_SHAPE, "a table of %lld rows", (long long)vocab);
  if (width < 1 || width > (int64_t(1) << 20) || vocab > kMaxMatrix / width)
    return fail(MALT_ERR_SHAPE, "a table of %lld x %lld", (long long)vocab, (long long)width);
  return MALT_OK;
}

}  // namespace

extern "C" {

malt_status_t malt_embed_lookup(const void* ids, malt_index_t id_type, int64_t tokens, const void* table,
                                malt_dtype_t table_type, int64_t vocab, int64_t width, int64_t table_ld, float scale,
                                void* out, malt_dtype_t out_type, int64_t out_ld, void* stream) {
  MALT_TRY(check_table(tokens, vocab, width));
  MALT_TRY(check_ids("ids", ids, id_type, tokens));
  const Mat t = {"table", table, table_type, vocab, width, table_ld}, o = {"out", out, out_type, tokens, width, out_ld};
  MALT_TRY(check_mat(t));
  MALT_TRY(check_mat(o));
  if (tokens == 0) return MALT_OK;
  const size_t id_bytes = size_t(tokens) * (id_type == MALT_INT64 ? 8 : 4);
  if (op_overlap(out, o.bytes(), table, t.bytes()) || op_overlap(out, o.bytes(), ids, id_bytes))
    return fail(MALT_ERR_ALIAS, "out overlaps the table or the ids");
  EmbedLookupArgs a = {};
  a.ids = ids;
  a.table = table;
  a.out = out;
  a.tokens = tokens;
  a.vocab = vocab;
  a.table_ld = table_ld;
  a.out_ld = out_ld;
  a.width = int32_t(width);
  a.wide_ids = id_type == MALT_INT64;
  a.scale = scale;
  return launched(launch_embed_lookup(a, table_type == MALT_FLOAT32, out_type == MALT_FLOAT32,
                                      static_cast<hipStream_t>(stream)),
                  "launching the table lookup");
}

malt_status_t malt_embed_grad_size(int64_t tokens, int64_t vocab, int64_t width, size_t* workspace_bytes) {
  if (!workspace_bytes) return fail(MALT_ERR_INVALID_ARG, "output pointer is NULL");
  MALT_TRY(check_table(tokens, vocab, width));
  *workspace_bytes = embed_grad_layout(tokens, vocab, width).bytes;
  return MALT_OK;
}

malt_status_t malt_embed_grad(const void* ids, malt_index_t id_type, int64_t tokens, const void* grad,
                              malt_dtype_t grad_type, int64_t grad_ld, float scale, int32_t accumulate, void* dtable,
                              malt_dtype_t dtable_type, int64_t vocab, int64_t width, int64_t dtable_ld,
                              void* workspace, size_t workspace_bytes, void* stream) {
  MALT_TRY(check_table(tokens, vocab, width));
  MALT_TRY(check_ids("ids", ids, id_type, tokens));
  if (accumulate != 0 && accumulate != 1) return fail(MALT_ERR_INVALID_ARG, "accumulate must be 0 or 1");
  const Mat g = {"grad", grad, grad_type, tokens, width, grad_ld},
            d = {"dtable", dtable, dtable_type, vocab, width, dtable_ld};
  MALT_TRY(check_mat(g));
  MALT_TRY(check_mat(d));
  const EmbedGradLayout L = embed_grad_layout(tokens, vocab, width);
  MALT_TRY(check_workspace(workspace, workspace_bytes, L.bytes));
  const size_t id_bytes = size_t(tokens) * (id_type == MALT_INT64 ? 8 : 4);
  if (op_overlap(dtable, d.bytes(), grad, g.bytes()) || op_overlap(dtable, d.bytes(), ids, id_bytes))
    return fail(MALT_ERR_ALIAS, "dtable overlaps the gradient or the ids");
  if (op_overlap(workspace, L.bytes, dtable, d.bytes()) || op_overlap(workspace, L.bytes, grad, g.bytes()) ||
      op_overlap(workspace, L.bytes, ids, id_bytes))
    return fail(MALT_ERR_ALIAS, "workspace overlaps another buffer");
  EmbedGradArgs a = {};
  a.ids = ids;
  a.grad = grad;
  a.dtable = dtable;
  a.tokens = tokens;
  a.vocab = vocab;
  a.grad_ld = grad_ld;
  a.dtable_ld = dtable_ld;
  a.width = int32_t(width);
  a.wide_ids = id_type == MALT_INT64;
  a.accumulate = accumulate != 0;
  a.scale = scale;
  if (tokens == 0 && accumulate) return MALT_OK;
  return launched(launch_embed_grad(a, L, static_cast<char*>(workspace), grad_type == MALT_FLOAT32,
                                    dtable_type == MALT_FLOAT32, static_cast<hipStream_t>(stream)),
                  "launching the table gradient");
}

malt_status_t malt_distill(const malt_distill_t* p, void* stream) {
  if (!p) return fail(MALT_ERR_INVALID_ARG, "args is NULL");
  if (p->rows < 0 || p->rows > kMaxRows) return fail(MALT_ERR_SHAPE, "%lld rows", (long long)p->rows);
  if (p->vocab < 1 || p->vocab > kMaxVocab) return fail(MALT_ERR_SHAPE, "a vocabulary of %lld", (long long)p->vocab);
  if (p->n_top < 0 || p->n_top > DISTILL_MAX_TOP)
    return fail(MALT_ERR_SHAPE, "%lld teacher entries a row (at most %d)", (long long)p->n_top, DISTILL_MAX_TOP);
  if (!(p->tau >= 0x1p-60f && p->tau <= 0x1p60f)) return fail(MALT_ERR_INVALID_ARG, "tau must be in [2^-60, 2^60]");
  if (!(p->alpha >= 0.f && p->alpha <= 1.f)) return fail(MALT_ERR_INVALID_ARG, "alpha must be in [0, 1]");
  const Mat z = {"logits", p->logits, p->dtype, p->rows, p->vocab, p->ld},
            top = {"top", p->top, p->top_type, p->n_top > 0 ? p->rows : 0, p->n_top, p->top_ld},
            d = {"dlogits", p->dlogits, p->dtype, p->rows, p->vocab, p->dld};
  MALT_TRY(check_mat(z));
  if (p->n_top > 0) {
    MALT_TRY(check_mat(top));
    MALT_TRY(check_ids("top_ids", p->top_ids, p->id_type, p->rows));
    if (p->id_ld < p->n_top || p->id_ld > kMaxPitch) return fail(MALT_ERR_SHAPE, "top_ids: row pitch %lld", (long long)p->id_ld);
  }
  if (p->labels) MALT_TRY(check_ids("labels", p->labels, p->label_type, p->rows));
  if (p->labels && (p->label_stride < 0 || p->label_stride > kMaxPitch))
    return fail(MALT_ERR_SHAPE, "labels: stride %lld", (long long)p->label_stride);
  if (!p->losses && !p->dlogits) return fail(MALT_ERR_INVALID_ARG, "neither losses nor dlogits is wanted");
  if (!op_aligned(p->losses, 4) || !op_aligned(p->weights, 4)) return fail(MALT_ERR_ALIGNMENT, "losses or weights not 4-byte aligned");
  if (p->weights && (p->weight_stride < 0 || p->weight_stride > kMaxPitch))
    return fail(MALT_ERR_SHAPE, "weights: stride %lld", (long long)p->weight_stride);
  if (p->dlogits) MALT_TRY(check_mat(d));
  if (p->rows == 0) return MALT_OK;
  const size_t id_bytes = p->n_top > 0 ? (size_t(p->rows - 1) * p->id_ld + p->n_top) * (p->id_type == MALT_INT64 ? 8 : 4) : 0;
  const size_t label_bytes = p->labels ? (size_t(p->rows - 1) * p->label_stride + 1) * (p->label_type == MALT_INT64 ? 8 : 4) : 0;
  const size_t weight_bytes = p->weights ? (size_t(p->rows - 1) * p->weight_stride + 1) * 4 : 0;
  const size_t loss_bytes = p->losses ? 4 * size_t(p->rows) : 0;
  struct Buf { const void* p; size_t n; };
  const Buf in[] = {{p->top, top.bytes()}, {p->top_ids, id_bytes}, {p->labels, label_bytes}, {p->weights, weight_bytes}};
  for (const Buf& b : in) {
    if (op_overlap(p->losses, loss_bytes, b.p, b.n)) return fail(MALT_ERR_ALIAS, "losses overlap an input");
    if (p->dlogits && op_overlap(p->dlogits, d.bytes(), b.p, b.n)) return fail(MALT_ERR_ALIAS, "dlogits overlap an input");
  }
  if (op_overlap(p->losses, loss_bytes, p->logits, z.bytes())) return fail(MALT_ERR_ALIAS, "losses overlap the logits");
  if (p->dlogits) {
    if (op_overlap(p->losses, loss_bytes, p->dlogits, d.bytes())) return fail(MALT_ERR_ALIAS, "losses overlap dlogits");
    const bool in_place = p->dlogits == p->logits && p->dld == p->ld;
    if (!in_place && op_overlap(p->dlogits, d.bytes(), p->logits, z.bytes()))
      return fail(MALT_ERR_ALIAS, "dlogits overlap the logits in part");
  }
  DistillArgs a = {};
  a.logits = p->logits;
  a.top = p->top;
  a.top_ids = p->top_ids;
  a.labels = p->labels;
  a.weight = p->weights;
  a.losses = p->losses;
  a.dlogits = p->dlogits;
  a.rows = p->rows;
  a.vocab = p->vocab;
  a.ld = p->ld;
  a.top_ld = p->top_ld;
  a.id_ld = p->id_ld;
  a.weight_stride = p->weight_stride;
  a.label_stride = p->label_stride;
  a.dld = p->dld;
  a.n_top = int32_t(p->n_top);
  a.wide_ids = p->id_type == MALT_INT64;
  a.top_f32 = p->top_type == MALT_FLOAT32;
  a.wide_labels = p->label_type == MALT_INT64;
  a.tau = p->tau;
  a.alpha = p->alpha;
  a.weight_value = p->weight;
  return launched(launch_distill(a, p->dtype == MALT_FLOAT32, static_cast<hipStream_t>(stream)),
                  "launching the distillation loss");
}

malt_status_t malt_block_size(int64_t rows, int64_t cols, size_t* value_bytes, size_t* scale_bytes) {
  if (!value_bytes || !scale_bytes) return fail(MALT_ERR_INVALID_ARG, "output pointer is NULL");
  if (rows < 1 || cols < 1 || rows > kMaxBlockDim || cols > kMaxBlockDim)
    return fail(MALT_ERR_SHAPE, "an 8-bit operand of %lld x %lld", (long long)rows, (long long)cols);
  *value_bytes = size_t(rows) * q_pad(cols);
  *scale_bytes = size_t(q_pad(cols) / QB) * q_scale_rows(rows);
  return MALT_OK;
}

static malt_status_t quantize(const char* what, const void* x, malt_dtype_t type, int64_t rows, int64_t cols, int64_t ld,
                              void* values, void* scales, void* t_values, void* t_scales, void* block_scales, void* stream) {
  size_t nv, ns, tv, ts;
  MALT_TRY(malt_block_size(rows, cols, &nv, &ns));
  MALT_TRY(malt_block_size(cols, rows, &tv, &ts));
  const Mat m = {what, x, type, rows, cols, ld};
  MALT_TRY(check_mat(m));
  if (!values && !t_values) return fail(MALT_ERR_INVALID_ARG, "neither values nor t_values is wanted");
  if (!block_scales && (!values != !scales || !t_values != !t_scales))
    return fail(MALT_ERR_INVALID_ARG, "values and scales come in pairs");
  const size_t nb = size_t(q_pad(rows) / QB) * (q_pad(cols) / QB);
  struct Buf { const void* p; size_t n; };
  const Buf out[] = {{values, nv}, {scales, ns}, {t_values, tv}, {t_scales, ts}, {block_scales, nb}};
  for (int i = 0; i < 5; ++i) {
    if (!out[i].p) continue;
    if (i < 4 && !op_aligned(out[i].p, 16)) return fail(MALT_ERR_ALIGNMENT, "8-bit values or scales not 16-byte aligned");
    if (op_overlap(out[i].p, out[i].n, x, m.bytes())) return fail(MALT_ERR_ALIAS, "an output overlaps %s", what);
    for (int j = 0; j < i; ++j)
      if (out[j].p && op_overlap(out[i].p, out[i].n, out[j].p, out[j].n)) return fail(MALT_ERR_ALIAS, "two outputs overlap");
  }
  QuantArgs a = {};
  a.x = x;
  a.rows = rows;
  a.cols = cols;
  a.ld = ld;
  a.values = static_cast<uint8_t*>(values);
  a.scales = static_cast<uint8_t*>(scales);
  a.t_values = static_cast<uint8_t*>(t_values);
  a.t_scales = static_cast<uint8_t*>(t_scales);
  a.block_scales = static_cast<uint8_t*>(block_scales);
  return launched(launch_block_quant(a, type == MALT_FLOAT32, static_cast<hipStream_t>(stream)), "launching the 8-bit conversion");
}

malt_status_t malt_block_quantize(const void* x, malt_dtype_t type, int64_t rows, int64_t cols, int64_t ld,
                                  void* values, void* scales, void* t_values, void* t_scales, void* stream) {
  return quantize("x", x, type, rows, cols, ld, values, scales, t_values, t_scales, nullptr, stream);
}

malt_status_t malt_block_quantize_weight(const void* w, malt_dtype_t type, int64_t rows, int64_t cols, int64_t ld,
                                         void* values, void* block_scales, void* t_values, void* stream) {
  if (!block_scales) return fail(MALT_ERR_INVALID_ARG, "block_scales is NULL");
  return quantize("w", w, type, rows, cols, ld, values, nullptr, t_values, nullptr, block_scales, stream);
}

malt_status_t malt_block_matmul_size(int64_t m, int64_t n, int64_t k, malt_dtype_t out_type, size_t* workspace_bytes) {
  if (!workspace_bytes) return fail(MALT_ERR_INVALID_ARG, "output pointer is NULL");
  if (!op_dtype_ok(out_type)) return fail(MALT_ERR_INVALID_ARG, "unknown element type %d", int(out_type));
  size_t v, s;
  MALT_TRY(malt_block_size(m, k, &v, &s));
  MALT_TRY(malt_block_size(n, k, &v, &s));
  if (m > kMaxProduct / n) return fail(MALT_ERR_SHAPE, "a product of %lld x %lld", (long long)m, (long long)n);
  *workspace_bytes = block_matmul_plan(m, n, k, out_type == MALT_FLOAT32).bytes;
  return MALT_OK;
}

malt_status_t malt_block_matmul(int64_t m, int64_t n, int64_t k, const void* a_values, const void* a_scales,
                                const void* b_values, const void* b_scales, int32_t b_blocks, int64_t b_row_stride,
                                int64_t b_col_stride, void* out, malt_dtype_t out_type, int64_t ldo,
                                int32_t accumulate, void* workspace, size_t workspace_bytes, void* stream) {
  size_t av, as, bv, bs, need;
  MALT_TRY(malt_block_size(m, k, &av, &as));
  MALT_TRY(malt_block_size(n, k, &bv, &bs));
  MALT_TRY(malt_block_matmul_size(m, n, k, out_type, &need));
  if (!a_values || !a_scales || !b_values || !b_scales) return fail(MALT_ERR_INVALID_ARG, "an operand is NULL");
  if (!op_aligned(a_values, 16) || !op_aligned(a_scales, 16) || !op_aligned(b_values, 16) || (!b_blocks && !op_aligned(b_scales, 16)))
    return fail(MALT_ERR_ALIGNMENT, "an operand is not 16-byte aligned");
  if (b_blocks != 0 && b_blocks != 1) return fail(MALT_ERR_INVALID_ARG, "b_blocks must be 0 or 1");
  if (accumulate != 0 && accumulate != 1) return fail(MALT_ERR_INVALID_ARG, "accumulate must be 0 or 1");
  if (as > 0xffffffffull || bs > 0xffffffffull) return fail(MALT_ERR_SHAPE, "an operand's scales exceed 4 GiB");
  if (b_blocks) {
    if (b_row_stride < 1 || b_col_stride < 1 || b_row_stride > kMaxPitch || b_col_stride > kMaxPitch)
      return fail(MALT_ERR_SHAPE, "strides %lld, %lld of a weight's scales", (long long)b_row_stride, (long long)b_col_stride);
    bs = size_t((q_pad(n) / QB - 1) * b_row_stride + (q_pad(k) / QB - 1) * b_col_stride + 1);
  }
  const Mat o = {"out", out, out_type, m, n, ldo};
  MALT_TRY(check_mat(o));
  if (op_overlap(out, o.bytes(), a_values, av) || op_overlap(out, o.bytes(), a_scales, as) ||
      op_overlap(out, o.bytes(), b_values, bv) || op_overlap(out, o.bytes(), b_scales, bs))
    return fail(MALT_ERR_ALIAS, "out overlaps an operand");
  MALT_TRY(check_workspace(workspace, workspace_bytes, need));
  if (op_overlap(workspace, need, out, o.bytes()) || op_overlap(workspace, need, a_values, av) ||
      op_overlap(workspace, need, a_scales, as) || op_overlap(workspace, need, b_values, bv) ||
      op_overlap(workspace, need, b_scales, bs))
    return fail(MALT_ERR_ALIAS, "workspace overlaps another buffer");
  BlockMatmulArgs g = {};
  g.m = m;
  g.n = n;
  g.k = k;
  g.a = static_cast<const uint8_t*>(a_values);
  g.a_scales = static_cast<const uint8_t*>(a_scales);
  g.b = static_cast<const uint8_t*>(b_values);
  g.b_scales = static_cast<const uint8_t*>(b_scales);
  g.b_row_stride = b_row_stride;
  g.b_col_stride = b_col_stride;
  g.out = out;
  g.ldo = ldo;
  g.accumulate = accumulate != 0;
  g.partial = static_cast<float*>(workspace);
  return launched(launch_block_matmul(g, b_blocks != 0, out_type == MALT_FLOAT32, static_cast<hipStream_t>(stream)),
                  "launching the 8-bit product");
}

malt_status_t malt_block_linear_size(int64_t m, int64_t n, int64_t k, malt_dtype_t out_type, size_t* workspace_bytes) {
  size_t product, values, scales;
  MALT_TRY(malt_block_matmul_size(m, n, k, out_type, workspace_bytes));
  product = *workspace_bytes;
  MALT_TRY(malt_block_size(m, k, &values, &scales));
  *workspace_bytes = m <= BLOCK_FEW ? 0 : align256(product) + values + scales;
  return MALT_OK;
}

malt_status_t malt_block_linear(const void* x, malt_dtype_t x_type, int64_t m, int64_t k, int64_t ldx,
                                const void* w_values, const void* w_scales, int64_t n, void* out,
                                malt_dtype_t out_type, int64_t ldo, void* workspace, size_t workspace_bytes,
                                void* stream) {
  size_t need, values, scales, wv, ws;
  MALT_TRY(malt_block_linear_size(m, n, k, out_type, &need));
  MALT_TRY(malt_block_size(m, k, &values, &scales));
  MALT_TRY(malt_block_size(n, k, &wv, &ws));
  ws = size_t(q_pad(n) / QB) * (q_pad(k) / QB);
  const Mat xm = {"x", x, x_type, m, k, ldx}, o = {"out", out, out_type, m, n, ldo};
  MALT_TRY(check_mat(xm));
  MALT_TRY(check_mat(o));
  if (!w_values || !w_scales) return fail(MALT_ERR_INVALID_ARG, "the weight is NULL");
  if (!op_aligned(w_values, 16)) return fail(MALT_ERR_ALIGNMENT, "the weight's values are not 16-byte aligned");
  if (op_overlap(out, o.bytes(), x, xm.bytes()) || op_overlap(out, o.bytes(), w_values, wv) ||
      op_overlap(out, o.bytes(), w_scales, ws))
    return fail(MALT_ERR_ALIAS, "out overlaps x or the weight");
  MALT_TRY(check_workspace(workspace, workspace_bytes, need));
  if (op_overlap(workspace, need, out, o.bytes()) || op_overlap(workspace, need, x, xm.bytes()) ||
      op_overlap(workspace, need, w_values, wv) || op_overlap(workspace, need, w_scales, ws))
    return fail(MALT_ERR_ALIAS, "workspace overlaps another buffer");
  if (m <= BLOCK_FEW) {
    BlockLinearArgs g = {};
    g.x = x;
    g.m = m;
    g.n = n;
    g.k = k;
    g.ldx = ldx;
    g.w = static_cast<const uint8_t*>(w_values);
    g.w_scales = static_cast<const uint8_t*>(w_scales);
    g.out = out;
    g.ldo = ldo;
    return launched(launch_block_linear(g, x_type == MALT_FLOAT32, out_type == MALT_FLOAT32, static_cast<hipStream_t>(stream)),
                    "launching the 8-bit layer");
  }
  char* const q = static_cast<char*>(workspace) + (need - values - scales);
  MALT_TRY(malt_block_quantize(x, x_type, m, k, ldx, q, q + values, nullptr, nullptr, stream));
  return malt_block_matmul(m, n, k, q, q + values, w_values, w_scales, 1, q_pad(k) / QB, 1, out, out_type, ldo, 0,
                           workspace, need - values - scales, stream);
}

malt_status_t malt_block_linear_operand(const void* x_values, const void* x_scales, int64_t m, int64_t k,
                                        const void* w_values, const void* w_scales, int64_t n, void* out,
                                        malt_dtype_t out_type, int64_t ldo, void* workspace, size_t workspace_bytes,
                                        void* stream) {
  if (m > BLOCK_FEW)
    return malt_block_matmul(m, n, k, x_values, x_scales, w_values, w_scales, 1, q_pad(k > 0 ? k : 1) / QB, 1, out, out_type, ldo,
                             0, workspace, workspace_bytes, stream);
  size_t need, values, scales, wv, ws;
  MALT_TRY(malt_block_matmul_size(m, n, k, out_type, &need));
  MALT_TRY(malt_block_size(m, k, &values, &scales));
  MALT_TRY(malt_block_size(n, k, &wv, &ws));
  ws = size_t(q_pad(n) / QB) * (q_pad(k) / QB);
  if (!x_values || !x_scales || !w_values || !w_scales) return fail(MALT_ERR_INVALID_ARG, "an operand is NULL");
  if (!op_aligned(x_values, 16) || !op_aligned(x_scales, 16) || !op_aligned(w_values, 16))
    return fail(MALT_ERR_ALIGNMENT, "an operand is not 16-byte aligned");
  const Mat o = {"out", out, out_type, m, n, ldo};
  MALT_TRY(check_mat(o));
  if (op_overlap(out, o.bytes(), x_values, values) || op_overlap(out, o.bytes(), x_scales, scales) ||
      op_overlap(out, o.bytes(), w_values, wv) || op_overlap(out, o.bytes(), w_scales, ws))
    return fail(MALT_ERR_ALIAS, "out overlaps an operand");
  BlockLinearArgs g = {};
  g.x = x_values;
  g.x_scales = static_cast<const uint8_t*>(x_scales);
  g.m = m;
  g.n = n;
  g.k = k;
  g.ldx = q_pad(k);
  g.w = static_cast<const uint8_t*>(w_values);
  g.w_scales = static_cast<const uint8_t*>(w_scales);
  g.out = out;
  g.ldo = ldo;
  return launched(launch_block_linear(g, false, out_type == MALT_FLOAT32, static_cast<hipStream_t>(stream)),
                  "launching the 8-bit layer");
}

// A layer's buffers: what is kept for the backward pass, and the workspaces.
struct LayerLayout {
  size_t xt, xt_scales, wt, w_scales, kept;              // kept: x^T, W^T, W's block scales
  size_t q, q_scales, w, forward_product, forward;       // forward: x, W, the product's partial sums
  size_t g, g_scales, gt, gt_scales, backward_product, backward;
};

// w_t: the weight lies k x n, and so does its gradient.
static LayerLayout layer_layout(int64_t m, int64_t n, int64_t k, bool w_t, bool y_f32, bool dx_f32, bool dw_f32, bool need_x,
                                bool need_w) {
  LayerLayout L = {};
  auto take = [](size_t& end, size_t bytes) {
    const size_t at = end;
    end += align256(bytes);
    return at;
  };
  auto values = [](int64_t r, int64_t c) { return size_t(r) * q_pad(c); };
  auto scales = [](int64_t r, int64_t c) { return size_t(q_pad(c) / QB) * q_scale_rows(r); };
  if (need_w) {
    L.xt = take(L.kept, values(k, m));
    L.xt_scales = take(L.kept, scales(k, m));
  }
  if (need_x) L.wt = take(L.kept, values(k, n));
  L.w_scales = take(L.kept, size_t(q_pad(n) / QB) * (q_pad(k) / QB));
  // What `kept` holds is told by its size: no two choices of gradients have the same.
  if (need_w && !need_x && L.w_scales == align256(values(k, n))) take(L.kept, 1);
  L.q = take(L.forward, values(m, k));
  L.q_scales = take(L.forward, scales(m, k));
  L.w = take(L.forward, values(n, k));
  L.forward_product = take(L.forward, block_matmul_plan(m, n, k, y_f32).bytes);
  if (need_x) {
    L.g = take(L.backward, values(m, n));
    L.g_scales = take(L.backward, scales(m, n));
  }
  if (need_w) {
    L.gt = take(L.backward, values(n, m));
    L.gt_scales = take(L.backward, scales(n, m));
  }
  size_t product = 0;   // the two products follow each other
  if (need_x) product = block_matmul_plan(m, k, n, dx_f32).bytes;
  if (need_w) {
    const size_t b = block_matmul_plan(w_t ? k : n, w_t ? n : k, m, dw_f32).bytes;
    if (b > product) product = b;
  }
  L.backward_product = take(L.backward, product);
  return L;
}

static malt_status_t check_layer(int64_t m, int64_t n, int64_t k) {
  size_t v, s;
  MALT_TRY(malt_block_size(m, k, &v, &s));
  MALT_TRY(malt_block_size(n, k, &v, &s));
  if (m > kMaxMatrix / n || m > kMaxMatrix / k || n > kMaxMatrix / k)
    return fail(MALT_ERR_SHAPE, "a layer of %lld x %lld on %lld rows", (long long)n, (long long)k, (long long)m);
  if (size_t(q_pad(k) / QB) * q_scale_rows(m) > 0xffffffffull || size_t(q_pad(n) / QB) * q_scale_rows(m) > 0xffffffffull ||
      size_t(q_pad(m) / QB) * q_scale_rows(n) > 0xffffffffull || size_t(q_pad(m) / QB) * q_scale_rows(k) > 0xffffffffull)
    return fail(MALT_ERR_SHAPE, "an operand's scales exceed 4 GiB");
  return MALT_OK;
}

malt_status_t malt_block_layer_size(int64_t m, int64_t n, int64_t k, int32_t w_transposed, malt_dtype_t y_type,
                                    malt_dtype_t dx_type, malt_dtype_t dw_type, int32_t need_dx, int32_t need_dw,
                                    size_t* kept_bytes, size_t* forward_bytes, size_t* backward_bytes) {
  if (!kept_bytes || !forward_bytes || !backward_bytes) return fail(MALT_ERR_INVALID_ARG, "output pointer is NULL");
  if (!op_dtype_ok(y_type) || !op_dtype_ok(dx_type) || !op_dtype_ok(dw_type)) return fail(MALT_ERR_INVALID_ARG, "unknown element type");
  if (w_transposed != 0 && w_transposed != 1) return fail(MALT_ERR_INVALID_ARG, "w_transposed must be 0 or 1");
  MALT_TRY(check_layer(m, n, k));
  const LayerLayout L = layer_layout(m, n, k, w_transposed != 0, y_type == MALT_FLOAT32, dx_type == MALT_FLOAT32,
                                     dw_type == MALT_FLOAT32, need_dx != 0, need_dw != 0);
  *kept_bytes = L.kept;
  *forward_bytes = L.forward;
  *backward_bytes = L.backward;
  return MALT_OK;
}

malt_status_t malt_block_layer_forward(const void* x, malt_dtype_t x_type, int64_t m, int64_t k, int64_t ldx,
                                       const void* w, malt_dtype_t w_type, int64_t n, int64_t ldw, int32_t w_transposed,
                                       void* y, malt_dtype_t y_type, int64_t ldy, int32_t need_dx, int32_t need_dw,
                                       void* kept, size_t kept_bytes, void* workspace, size_t workspace_bytes,
                                       void* stream) {
  if (w_transposed != 0 && w_transposed != 1) return fail(MALT_ERR_INVALID_ARG, "w_transposed must be 0 or 1");
  MALT_TRY(check_layer(m, n, k));
  const bool wt = w_transposed != 0;
  const Mat xm = {"x", x, x_type, m, k, ldx}, wm = {"w", w, w_type, wt ? k : n, wt ? n : k, ldw}, ym = {"y", y, y_type, m, n, ldy};
  MALT_TRY(check_mat(xm));
  MALT_TRY(check_mat(wm));
  MALT_TRY(check_mat(ym));
  const LayerLayout L = layer_layout(m, n, k, wt, y_type == MALT_FLOAT32, false, false, need_dx != 0, need_dw != 0);
  MALT_TRY(check_workspace(kept, kept_bytes, L.kept));
  MALT_TRY(check_workspace(workspace, workspace_bytes, L.forward));
  struct Buf { const void* p; size_t n; };
  const Buf b[] = {{x, xm.bytes()}, {w, wm.bytes()}, {y, ym.bytes()}, {kept, L.kept}, {workspace, L.forward}};
  for (int i = 2; i < 5; ++i)
    for (int j = 0; j < i; ++j)
      if (op_overlap(b[i].p, b[i].n, b[j].p, b[j].n)) return fail(MALT_ERR_ALIAS, "two of the layer's buffers overlap");
  uint8_t *const kb = static_cast<uint8_t*>(kept), *const ws = static_cast<uint8_t*>(workspace);
  QuantArgs qx = {}, qw = {};
  qx.x = x;
  qx.rows = m;
  qx.cols = k;
  qx.ld = ldx;
  qx.values = ws + L.q;
  qx.scales = ws + L.q_scales;
  qx.t_values = need_dw ? kb + L.xt : nullptr;
  qx.t_scales = need_dw ? kb + L.xt_scales : nullptr;
  qw.x = w;
  qw.rows = wm.rows;
  qw.cols = wm.cols;
  qw.ld = ldw;
  // The forward product takes the weight as n rows, the input gradient as k.
  uint8_t* const by_k = need_dx ? kb + L.wt : nullptr;
  qw.values = wt ? by_k : ws + L.w;
  qw.t_values = wt ? ws + L.w : by_k;
  qw.block_scales = kb + L.w_scales;
  const hipError_t e = launch_block_quant_pair(qx, x_type == MALT_FLOAT32, qw, w_type == MALT_FLOAT32, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, "launching the 8-bit conversion");
  return malt_block_matmul(m, n, k, ws + L.q, ws + L.q_scales, ws + L.w, kb + L.w_scales, 1, wt ? 1 : q_pad(k) / QB,
                           wt ? q_pad(n) / QB : 1, y, y_type, ldy, 0, ws + L.forward_product, L.forward - L.forward_product, stream);
}

malt_status_t malt_block_layer_backward(const void* dy, malt_dtype_t dy_type, int64_t m, int64_t n, int64_t lddy,
                                        int64_t k, int32_t w_transposed, const void* kept, size_t kept_bytes, void* dx,
                                        malt_dtype_t dx_type, int64_t lddx, void* dw, malt_dtype_t dw_type, int64_t lddw,
                                        int32_t accumulate, void* workspace, size_t workspace_bytes, void* stream) {
  if (w_transposed != 0 && w_transposed != 1) return fail(MALT_ERR_INVALID_ARG, "w_transposed must be 0 or 1");
  MALT_TRY(check_layer(m, n, k));
  const bool wt = w_transposed != 0;
  if (!dx && !dw) return fail(MALT_ERR_INVALID_ARG, "neither dx nor dw is wanted");
  if (accumulate != 0 && accumulate != 1) return fail(MALT_ERR_INVALID_ARG, "accumulate must be 0 or 1");
  const Mat g = {"dy", dy, dy_type, m, n, lddy}, xm = {"dx", dx, dx_type, m, k, lddx}, wm = {"dw", dw, dw_type, wt ? k : n, wt ? n : k, lddw};
  MALT_TRY(check_mat(g));
  if (dx) MALT_TRY(check_mat(xm));
  if (dw) MALT_TRY(check_mat(wm));
  const LayerLayout L = layer_layout(m, n, k, wt, false, dx_type == MALT_FLOAT32, dw_type == MALT_FLOAT32, dx != nullptr,
                                     dw != nullptr);
  MALT_TRY(check_workspace(kept, kept_bytes, L.kept));
  MALT_TRY(check_workspace(workspace, workspace_bytes, L.backward));
  struct Buf { const void* p; size_t n; };
  const Buf b[] = {{dy, g.bytes()}, {kept, L.kept}, {dx, dx ? xm.bytes() : 0}, {dw, dw ? wm.bytes() : 0}, {workspace, L.backward}};
  for (int i = 2; i < 5; ++i)
    for (int j = 0; j < i; ++j)
      if (op_overlap(b[i].p, b[i].n, b[j].p, b[j].n)) return fail(MALT_ERR_ALIAS, "two of the layer's buffers overlap");
  if (kept_bytes != L.kept)
    return fail(MALT_ERR_INVALID_ARG, "%zu kept bytes where these gradients need %zu: the forward call kept for others", kept_bytes, L.kept);
  const uint8_t* const kb = static_cast<const uint8_t*>(kept);
  uint8_t* const ws = static_cast<uint8_t*>(workspace);
  QuantArgs q = {};
  q.x = dy;
  q.rows = m;
  q.cols = n;
  q.ld = lddy;
  if (dx) {
    q.values = ws + L.g;
    q.scales = ws + L.g_scales;
  }
  if (dw) {
    q.t_values = ws + L.gt;
    q.t_scales = ws + L.gt_scales;
  }
  const hipError_t e = launch_block_quant(q, dy_type == MALT_FLOAT32, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, "launching the 8-bit conversion");
  const size_t product = L.backward - L.backward_product;
  if (dx)
    MALT_TRY(malt_block_matmul(m, k, n, ws + L.g, ws + L.g_scales, kb + L.wt, kb + L.w_scales, 1, wt ? q_pad(n) / QB : 1,
                               wt ? 1 : q_pad(k) / QB, dx, dx_type, lddx, 0, ws + L.backward_product, product, stream));
  const uint8_t *const gt = ws + L.gt, *const gs = ws + L.gt_scales, *const xt = kb + L.xt, *const xs = kb + L.xt_scales;
  if (dw)
    MALT_TRY(malt_block_matmul(wm.rows, wm.cols, m, wt ? xt : gt, wt ? xs : gs, wt ? gt : xt, wt ? gs : xs, 0, 0, 0, dw, dw_type,
                               lddw, accumulate, ws + L.backward_product, product, stream));
  return MALT_OK;
}

}  // extern "C"
