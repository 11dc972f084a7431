// C ABI of the single operators (include/asteroid_ops.h): argument checks, then the launches of ops.h.
#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <string>

#include "ops.h"

namespace ast {
void set_last_error(const std::string& msg);  // api.cpp
}

namespace {

ast_status fail(const char* what, const char* why, ast_status code = AST_EINVAL) {
  ast::set_last_error(std::string(what) + ": " + why);
  return code;
}

ast_status launched(const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? AST_OK : fail(what, hipGetErrorString(e), AST_EHIP);
}

hipStream_t stream_of(void* s) { return static_cast<hipStream_t>(s); }
bool dtype_ok(int32_t d) { return d == AST_F32 || d == AST_BF16_F32ACC; }
size_t esize(int32_t d) { return d == AST_F32 ? 4 : 2; }
bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

constexpr int64_t kMostRows = ((int64_t)1 << 31) - 1;  // tokens and rows are counted in 32 bits
constexpr int64_t kMostWidth = (int64_t)1 << 20;

const char* embedding_sizes(int64_t tokens, int64_t rows, int64_t width) {
  if (tokens < 0 || tokens > kMostRows) return "tokens must lie in [0, 2^31)";
  if (rows < 1 || rows > kMostRows - 1) return "rows must lie in [1, 2^31 - 2]";
  if (width < 1 || width > kMostWidth) return "width must lie in [1, 2^20]";
  return nullptr;
}

const char* stash_sizes(int64_t rows, int64_t cols) {
  if (rows < 0 || rows > kMostRows) return "rows must lie in [0, 2^31)";
  if (cols < 1 || cols > kMostWidth) return "the row length must lie in [1, 2^20]";
  if (rows * ast::stash8_pitch(cols) >= (int64_t)1 << 40) return "the matrix must stay below 2^40 values";
  return nullptr;
}

const char* wgrad_sizes(int64_t rows, int64_t in, int64_t out) {
  if (const char* e = stash_sizes(rows, in)) return e;
  if (out < 1 || out > kMostWidth) return "out must lie in [1, 2^20]";
  if (in * out > (int64_t)1 << 36) return "in * out must not exceed 2^36";
  return nullptr;
}

const char* qk_cfg(const ast_qk_cfg* c) {
  if (!c) return "cfg is NULL";
  if (!dtype_ok(c->dtype)) return "unknown dtype";
  if (c->tokens < 0 || c->tokens > kMostRows) return "tokens must lie in [0, 2^31)";
  if (c->head_dim < 1 || c->head_dim > 256) return "head_dim must lie in [1, 256]";
  if (c->rotary < 0 || c->rotary > c->head_dim || c->rotary % 2) return "rotary must be even and lie in [0, head_dim]";
  if (!(c->eps > 0.f) || !std::isfinite(c->eps)) return "eps must be positive";
  if (!(c->theta > 0.0) || !std::isfinite(c->theta)) return "theta must be positive";
  if (c->positions_dev ? !aligned(c->positions_dev, 4) : c->period < 1) return "positions_dev must be 4-byte aligned, or period >= 1";
  return nullptr;
}

const char* heads_ok(const ast_qk_cfg& c, const ast_heads* h, int32_t heads) {
  if (!h) return "a head tensor is NULL";
  if (h->heads < 1 || h->heads > 65535) return "heads must lie in [1, 65535]";
  if (h->heads != heads) return "the numbers of heads differ between inputs and outputs";
  if (h->token_stride < 0 || h->token_stride > kMostRows || h->head_stride < 0 || h->head_stride > (int64_t)1 << 40)
    return "strides must lie in [0, 2^31) (tokens) and [0, 2^40] (heads)";
  if (c.tokens > 0 && (!h->dev || !aligned(h->dev, esize(c.dtype)))) return "head tensors must be non-NULL and aligned to their element size";
  return nullptr;
}
// a tensor that is written: its heads may not lie on top of each other
const char* heads_apart(const ast_qk_cfg& c, const ast_heads& h) {
  const int64_t d = c.head_dim, H = h.heads;
  const bool head_inner = (H == 1 || h.head_stride >= d) && (c.tokens <= 1 || h.token_stride >= (H - 1) * h.head_stride + d);
  const bool token_inner = (c.tokens <= 1 || h.token_stride >= d) && (H == 1 || h.head_stride >= (c.tokens - 1) * h.token_stride + d);
  return head_inner || token_inner ? nullptr : "the heads of an output overlap";
}

// The memory of a tensor: rows of `wide` bytes, `step` bytes from one to the next, all of them in [lo, hi).  (Products of the sizes and
// strides that the calls take do not fit 64 bits: they are formed in 128, and hi ends with the address space.)
typedef unsigned __int128 Wide;
struct Area {
  uint64_t lo = 0, hi = 0;  // (equal: nothing, a tensor that is not there or has no rows)
  uint64_t rows = 0, step = 0, wide = 0;
  Area() {}
  Area(const void* p, int64_t rows_, int64_t step_, int64_t wide_) {
    if (!p || rows_ <= 0 || wide_ <= 0) return;
    lo = reinterpret_cast<uintptr_t>(p);
    rows = (uint64_t)rows_, step = (uint64_t)step_, wide = (uint64_t)wide_;
    hi = (uint64_t)std::min(lo + (Wide)(rows - 1) * step + wide, (Wide)UINT64_MAX);
    if (step <= wide) wide = hi - lo, rows = 1;  // (no gaps)
  }
};
Area block_of(const void* p, size_t bytes) { return Area(p, 1, (int64_t)bytes, (int64_t)bytes); }
// A byte belongs to both, whose ranges lie on each other.  Exact, except that rows with gaps and different steps count as all that lies
// between their first and last.
bool rows_meet(const Area& a, const Area& b) {
  if (a.rows == 1 && b.rows == 1) return true;
  if (a.rows == 1 || b.rows == 1) {
    const Area &one = a.rows == 1 ? a : b, &many = a.rows == 1 ? b : a;
    const uint64_t row = std::min((one.hi - 1 - many.lo) / many.step, many.rows - 1);  // the last that begins in front of its end
    return many.lo + (Wide)row * many.step + many.wide > one.lo;
  }
  if (a.step != b.step) return true;
  const Area &p = a.lo <= b.lo ? a : b, &q = a.lo <= b.lo ? b : a;  // q's first row: behind p's row k, by r bytes
  const uint64_t k = (q.lo - p.lo) / p.step, r = (q.lo - p.lo) % p.step;
  return (k < p.rows && r < p.wide) || (k + 1 < p.rows && p.step - r < q.wide);
}
bool meet(const Area& a, const Area& b) { return a.lo < b.hi && b.lo < a.hi && rows_meet(a, b); }
// the same rows at the same place
bool same(const Area& a, const Area& b) {
  return a.lo == b.lo && a.hi == b.hi && a.rows == b.rows && (a.rows == 1 || (a.step == b.step && a.wide == b.wide));
}
struct Some {  // (a list of areas holds no copies)
  const Area* area;
  Some(const Area& a) : area(&a) {}
};
typedef std::initializer_list<Some> Areas;
bool any_meet(Areas outputs) {
  for (auto a = outputs.begin(); a != outputs.end(); ++a)
    for (auto b = outputs.begin(); b != a; ++b)
      if (meet(*a->area, *b->area)) return true;
  return false;
}
// ... one of each; in_place: not counting an output that is the input
bool any_meet(Areas outputs, Areas inputs, bool in_place = false) {
  for (const Some& a : outputs)
    for (const Some& b : inputs)
      if (meet(*a.area, *b.area) && !(in_place && same(*a.area, *b.area))) return true;
  return false;
}
const char* const kOnInput = "an output and an input overlap, and are not the same rows where that is allowed";
const char* const kOnWorkspace = "the workspace overlaps a tensor";

const char* norm_cfg(const ast_norm_cfg* c) {
  if (!c) return "cfg is NULL";
  if (!dtype_ok(c->dtype) || !dtype_ok(c->sum_dtype)) return "unknown dtype";
  if (c->sum_dtype != c->dtype && c->sum_dtype != AST_F32) return "sum_dtype must be dtype or AST_F32";
  if (c->rows < 0 || c->rows > kMostRows) return "rows must lie in [0, 2^31)";
  if (c->width < 1 || c->width > 16384) return "width must lie in [1, 16384]";
  if (!(c->eps >= 0x1p-126f) || !std::isfinite(c->eps)) return "eps must be positive, and no subnormal number";
  return nullptr;
}

size_t norm_bytes(const ast_norm_cfg& c, int32_t dtype) { return (size_t)c.rows * (size_t)c.width * esize(dtype); }

const char* recurrence_cfg(const ast_recurrence_cfg* c) {
  if (!c) return "cfg is NULL";
  if (!dtype_ok(c->dtype)) return "unknown dtype";
  if (c->tokens < 0 || c->tokens > kMostRows) return "tokens must lie in [0, 2^31)";
  if (c->channels < 1 || c->channels > kMostWidth) return "channels must lie in [1, 2^20]";
  // (a launch has fewer than 2^32 threads)
  if ((c->tokens + 511) / 512 * 512 * ((c->channels + 63) / 64 * 64) > (int64_t)1 << 34) return "tokens * channels must not exceed 2^34";
  if (c->offsets_dev) {
    if (!aligned(c->offsets_dev, 4)) return "offsets_dev must be 4-byte aligned";
    if (c->sequences < 0 || c->sequences > kMostRows - 1) return "sequences must lie in [0, 2^31 - 2]";
  } else if (c->period < 1 || c->period > kMostRows) {
    return "offsets_dev, or a period in [1, 2^31), must be given";
  }
  return nullptr;
}

const char* rows_ok(const ast_recurrence_cfg& c, const ast_rows* r, bool out) {
  if (!r) return "a tensor is NULL";
  if (r->stride < 0 || r->stride > (int64_t)1 << 40) return "strides must lie in [0, 2^40]";
  if (c.tokens > 0 && (!r->dev || !aligned(r->dev, esize(c.dtype)))) return "tensors must be non-NULL and aligned to their element size";
  if (out && c.tokens > 1 && r->stride < c.channels) return "the rows of an output overlap";
  return nullptr;
}
Area rows_of(const ast_recurrence_cfg& c, const ast_rows* r) {
  const int64_t e = (int64_t)esize(c.dtype);
  return r ? Area(r->dev, c.tokens, r->stride * e, c.channels * e) : Area();
}
Area states_of(const ast_recurrence_cfg& c, const float* p) {
  const int64_t n = c.offsets_dev ? c.sequences : (c.tokens + c.period - 1) / c.period;
  return Area(p, n, c.channels * 4, c.channels * 4);
}
Area saved_of(const ast_recurrence_cfg& c, const float* p) {
  return Area(p, (c.tokens + AST_RECURRENCE_CHUNK - 1) / AST_RECURRENCE_CHUNK, c.channels * 4, c.channels * 4);
}
Area offsets_of(const ast_recurrence_cfg& c) { return Area(c.offsets_dev, c.sequences + 1, 4, 4); }

const char* distill_cfg(const ast_distill_cfg* c) {
  if (!c) return "cfg is NULL";
  if (!dtype_ok(c->dtype) || !dtype_ok(c->teacher_dtype)) return "unknown dtype";
  if (c->rows < 0 || c->rows > kMostRows) return "rows must lie in [0, 2^31)";
  if (c->vocab < 1 || c->vocab > (int64_t)1 << 30) return "vocab must lie in [1, 2^30]";
  if (c->logits_stride < c->vocab || c->logits_stride > (int64_t)1 << 31) return "logits_stride must lie in [vocab, 2^31]";
  if (c->entries < 1 || c->entries > 1024) return "entries must lie in [1, 1024]";
  if (!(c->temperature >= 0x1p-30f && c->temperature <= 0x1p30f)) return "temperature must lie in [2^-30, 2^30]";  // (T^2 and log2(e) / T)
  if (!(c->label_weight >= 0.f && c->label_weight <= 1.f)) return "label_weight must lie in [0, 1]";
  if (!c->labels_dev && c->label_weight != 0.f) return "a label_weight needs labels";
  if (!aligned(c->labels_dev, 4)) return "labels_dev must be 4-byte aligned";
  return nullptr;
}
const char* distill_inputs(const ast_distill_cfg& c, const void* z, const int32_t* ids, const void* t) {
  if (!z || !ids || !t) return "NULL argument";
  if (!aligned(z, esize(c.dtype)) || !aligned(ids, 4) || !aligned(t, esize(c.teacher_dtype))) return "buffers must be aligned to their element size";
  return nullptr;
}
Area vocab_rows(const ast_distill_cfg& c, const void* p, int64_t stride) {
  const int64_t e = (int64_t)esize(c.dtype);
  return Area(p, c.rows, stride * e, c.vocab * e);
}
Area entries_of(const ast_distill_cfg& c, const void* p, size_t e) {
  const int64_t wide = c.entries * (int64_t)e;
  return Area(p, c.rows, wide, wide);
}
Area a_row(const ast_distill_cfg& c, const void* p, int64_t values = 1) { return Area(p, c.rows, 4 * values, 4 * values); }
const char* distill_gradient(const ast_distill_cfg& c, const float* dloss, const void* z, const int32_t* ids, const void* t, const void* dz,
                             int64_t stride) {
  if (!dloss || !dz) return "NULL argument";
  if (!aligned(dloss, 4) || !aligned(dz, esize(c.dtype))) return "buffers must be aligned to their element size";
  if (stride < c.vocab || stride > (int64_t)1 << 31) return "dlogits_stride must lie in [vocab, 2^31]";
  if (z == dz && stride != c.logits_stride) return "a gradient in place of the logits needs their stride";
  const Area g = vocab_rows(c, dz, stride);
  const Area id = entries_of(c, ids, 4), top = entries_of(c, t, esize(c.teacher_dtype));
  if (any_meet({g}, {vocab_rows(c, z, c.logits_stride)}, true) || any_meet({g}, {id, top, a_row(c, dloss), a_row(c, c.labels_dev)})) return kOnInput;
  return nullptr;
}

}  // namespace

extern "C" {

ast_status asteroid_embedding_forward(const int32_t* ids_dev, int64_t tokens, const void* table_dev, int32_t table_dtype,
                                      int64_t rows, int64_t width, float scale, void* y_dev, int32_t y_dtype, void* hip_stream) {
  const char* const fn = "embedding_forward";
  if (!dtype_ok(table_dtype) || !dtype_ok(y_dtype)) return fail(fn, "unknown dtype");
  if (const char* e = embedding_sizes(tokens, rows, width)) return fail(fn, e);
  if (!std::isfinite(scale)) return fail(fn, "scale must be finite");
  if (tokens == 0) return AST_OK;
  if (!ids_dev || !table_dev || !y_dev) return fail(fn, "NULL argument");
  if (!aligned(ids_dev, 4) || !aligned(table_dev, esize(table_dtype)) || !aligned(y_dev, esize(y_dtype)))
    return fail(fn, "buffers must be aligned to their element size");
  ast::embedding_fwd(stream_of(hip_stream), ids_dev, tokens, table_dev, table_dtype != AST_F32, rows, width, scale, y_dev,
                     y_dtype != AST_F32);
  return launched(fn);
}

ast_status asteroid_embedding_backward_workspace(int64_t tokens, int64_t rows, int64_t width, size_t* bytes) {
  const char* const fn = "embedding_backward_workspace";
  if (!bytes) return fail(fn, "NULL argument");
  if (const char* e = embedding_sizes(tokens, rows, width)) return fail(fn, e);
  *bytes = ast::embedding_bwd_ws_bytes(tokens, rows, width);
  return AST_OK;
}

ast_status asteroid_embedding_backward(const int32_t* ids_dev, int64_t tokens, const void* dy_dev, int32_t dy_dtype, int64_t rows,
                                       int64_t width, float scale, int32_t accumulate, float* dtable_dev, void* workspace_dev,
                                       size_t workspace_bytes, void* hip_stream) {
  const char* const fn = "embedding_backward";
  if (!dtype_ok(dy_dtype)) return fail(fn, "unknown dtype");
  if (const char* e = embedding_sizes(tokens, rows, width)) return fail(fn, e);
  if (!std::isfinite(scale)) return fail(fn, "scale must be finite");
  if (!dtable_dev || !aligned(dtable_dev, 4)) return fail(fn, "dtable_dev must be non-NULL and 4-byte aligned");
  if (tokens > 0) {
    if (!ids_dev || !dy_dev) return fail(fn, "NULL argument");
    if (!aligned(ids_dev, 4) || !aligned(dy_dev, esize(dy_dtype))) return fail(fn, "buffers must be aligned to their element size");
  }
  const size_t need = ast::embedding_bwd_ws_bytes(tokens, rows, width);
  if (need && (!workspace_dev || workspace_bytes < need || !aligned(workspace_dev, 16)))
    return fail(fn, "the workspace is missing, too small or not 16-byte aligned");
  ast::embedding_bwd(stream_of(hip_stream), ids_dev, tokens, dy_dev, dy_dtype != AST_F32, rows, width, scale, accumulate != 0,
                     dtable_dev, workspace_dev);
  return launched(fn);
}

ast_status asteroid_qk_norm_rope_forward(const ast_qk_cfg* cfg, const ast_heads* q, const ast_heads* k, const float* q_gain_dev,
                                         const float* k_gain_dev, const ast_heads* yq, const ast_heads* yk, void* hip_stream) {
  const char* const fn = "qk_norm_rope_forward";
  if (const char* e = qk_cfg(cfg)) return fail(fn, e);
  const ast_heads* const all[4] = {q, yq, k, yk};
  for (int i = 0; i < 4; ++i)
    if (const char* e = heads_ok(*cfg, all[i], (i < 2 ? q : k) ? (i < 2 ? q : k)->heads : 0)) return fail(fn, e);
  for (const ast_heads* h : {yq, yk})
    if (const char* e = heads_apart(*cfg, *h)) return fail(fn, e);
  if (cfg->tokens == 0) return AST_OK;
  if (!q_gain_dev || !k_gain_dev || !aligned(q_gain_dev, 4) || !aligned(k_gain_dev, 4))
    return fail(fn, "gains must be non-NULL and 4-byte aligned");
  if (yq->dev == yk->dev) return fail(fn, "yq and yk are one tensor");
  ast::qk_norm_rope_fwd(stream_of(hip_stream), *cfg, *q, *k, q_gain_dev, k_gain_dev, *yq, *yk);
  return launched(fn);
}

ast_status asteroid_qk_norm_rope_backward_workspace(const ast_qk_cfg* cfg, int32_t q_heads, int32_t k_heads, size_t* bytes) {
  const char* const fn = "qk_norm_rope_backward_workspace";
  if (!bytes) return fail(fn, "NULL argument");
  if (const char* e = qk_cfg(cfg)) return fail(fn, e);
  if (q_heads < 1 || q_heads > 65535 || k_heads < 1 || k_heads > 65535) return fail(fn, "heads must lie in [1, 65535]");
  *bytes = ast::qk_norm_rope_bwd_ws_bytes(cfg->tokens, cfg->head_dim);
  return AST_OK;
}

ast_status asteroid_qk_norm_rope_backward(const ast_qk_cfg* cfg, const ast_heads* dyq, const ast_heads* dyk, const ast_heads* q,
                                          const ast_heads* k, const float* q_gain_dev, const float* k_gain_dev, const ast_heads* dq,
                                          const ast_heads* dk, float* dq_gain_dev, float* dk_gain_dev, int32_t accumulate,
                                          void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
  const char* const fn = "qk_norm_rope_backward";
  if (const char* e = qk_cfg(cfg)) return fail(fn, e);
  const ast_heads* const all[6] = {q, dyq, dq, k, dyk, dk};
  for (int i = 0; i < 6; ++i)
    if (const char* e = heads_ok(*cfg, all[i], (i < 3 ? q : k) ? (i < 3 ? q : k)->heads : 0)) return fail(fn, e);
  for (const ast_heads* h : {dq, dk})
    if (const char* e = heads_apart(*cfg, *h)) return fail(fn, e);
  for (const float* p : {q_gain_dev, k_gain_dev, (const float*)dq_gain_dev, (const float*)dk_gain_dev})
    if (!p || !aligned(p, 4)) return fail(fn, "gains and their gradients must be non-NULL and 4-byte aligned");
  const size_t need = ast::qk_norm_rope_bwd_ws_bytes(cfg->tokens, cfg->head_dim);
  if (need && (!workspace_dev || workspace_bytes < need || !aligned(workspace_dev, 16)))
    return fail(fn, "the workspace is missing, too small or not 16-byte aligned");
  if (dq_gain_dev < dk_gain_dev + cfg->head_dim && dk_gain_dev < dq_gain_dev + cfg->head_dim)
    return fail(fn, "the gains' gradients overlap");
  if (cfg->tokens > 0 && dq->dev == dk->dev) return fail(fn, "dq and dk are one tensor");
  ast::qk_norm_rope_bwd(stream_of(hip_stream), *cfg, *dyq, *dyk, *q, *k, q_gain_dev, k_gain_dev, *dq, *dk, dq_gain_dev, dk_gain_dev,
                        accumulate != 0, workspace_dev);
  return launched(fn);
}

ast_status asteroid_rms_norm_forward(const ast_norm_cfg* cfg, const void* x_dev, const void* residual_dev, const float* gain_dev,
                                     void* y_dev, void* sum_dev, void* stash_dev, void* hip_stream) {
  const char* const fn = "rms_norm_forward";
  if (const char* e = norm_cfg(cfg)) return fail(fn, e);
  if (!residual_dev != !sum_dev) return fail(fn, "the residual and the sum go together");
  if (!residual_dev && cfg->sum_dtype != cfg->dtype && cfg->rows > 0) return fail(fn, "without a residual the sum is x: sum_dtype must be dtype");
  if (cfg->rows == 0) return AST_OK;
  if (!x_dev || !gain_dev || !y_dev) return fail(fn, "NULL argument");
  if (!aligned(x_dev, esize(cfg->dtype)) || !aligned(y_dev, esize(cfg->dtype)) || !aligned(residual_dev, esize(cfg->sum_dtype)) ||
      !aligned(sum_dev, esize(cfg->sum_dtype)) || !aligned(gain_dev, 4) || !aligned(stash_dev, 16))
    return fail(fn, "buffers must be aligned to their element size, the stash to 16 bytes");
  const Area x = block_of(x_dev, norm_bytes(*cfg, cfg->dtype)), r = block_of(residual_dev, norm_bytes(*cfg, cfg->sum_dtype));
  const Area y = block_of(y_dev, norm_bytes(*cfg, cfg->dtype)), sum = block_of(sum_dev, norm_bytes(*cfg, cfg->sum_dtype));
  const Area kept = block_of(stash_dev, ast::stash8_bytes(cfg->rows, cfg->width)), gain = block_of(gain_dev, 4 * (size_t)cfg->width);
  if (any_meet({y, sum, kept})) return fail(fn, "outputs overlap");
  // (rows of another type lie elsewhere: a block's would be another block's)
  if (any_meet({y, sum}, {x, r}, true) || any_meet({kept}, {x, r}) || any_meet({y, sum, kept}, {gain})) return fail(fn, kOnInput);
  ast::rms_norm_fwd(stream_of(hip_stream), *cfg, x_dev, residual_dev, gain_dev, y_dev, sum_dev, stash_dev);
  return launched(fn);
}

ast_status asteroid_rms_norm_backward_workspace(const ast_norm_cfg* cfg, size_t* bytes) {
  const char* const fn = "rms_norm_backward_workspace";
  if (!bytes) return fail(fn, "NULL argument");
  if (const char* e = norm_cfg(cfg)) return fail(fn, e);
  *bytes = ast::rms_norm_bwd_ws_bytes(cfg->rows, cfg->width);
  return AST_OK;
}

ast_status asteroid_rms_norm_backward(const ast_norm_cfg* cfg, const void* dy_dev, const void* sum_dev, const float* gain_dev,
                                      const void* dsum_dev, void* dx_dev, void* ds_dev, float* dgain_dev, int32_t accumulate,
                                      void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
  const char* const fn = "rms_norm_backward";
  if (const char* e = norm_cfg(cfg)) return fail(fn, e);
  if (!gain_dev || !dgain_dev || !aligned(gain_dev, 4) || !aligned(dgain_dev, 4))
    return fail(fn, "the gain and its gradient must be non-NULL and 4-byte aligned");
  if (cfg->rows > 0) {
    if (!dy_dev || !sum_dev) return fail(fn, "NULL argument");
    if (!dx_dev && !ds_dev) return fail(fn, "dx_dev or ds_dev must be given");
    if (!aligned(dy_dev, esize(cfg->dtype)) || !aligned(dx_dev, esize(cfg->dtype)) || !aligned(sum_dev, esize(cfg->sum_dtype)) ||
        !aligned(dsum_dev, esize(cfg->sum_dtype)) || !aligned(ds_dev, esize(cfg->sum_dtype)))
      return fail(fn, "buffers must be aligned to their element size");
  }
  const Area dy = block_of(dy_dev, norm_bytes(*cfg, cfg->dtype)), sum = block_of(sum_dev, norm_bytes(*cfg, cfg->sum_dtype));
  const Area dsum = block_of(dsum_dev, norm_bytes(*cfg, cfg->sum_dtype)), gain = block_of(gain_dev, 4 * (size_t)cfg->width);
  const Area dx = block_of(dx_dev, norm_bytes(*cfg, cfg->dtype)), ds = block_of(ds_dev, norm_bytes(*cfg, cfg->sum_dtype));
  const Area dgain = block_of(dgain_dev, 4 * (size_t)cfg->width);
  if (any_meet({dx, ds, dgain})) return fail(fn, "outputs overlap");
  if (any_meet({dx, ds}, {dy, sum, dsum}, true) || any_meet({dx, ds}, {gain}) || any_meet({dgain}, {gain}, true) ||
      any_meet({dgain}, {dy, sum, dsum}))
    return fail(fn, kOnInput);
  const size_t need = ast::rms_norm_bwd_ws_bytes(cfg->rows, cfg->width);
  if (need && (!workspace_dev || workspace_bytes < need || !aligned(workspace_dev, 16)))
    return fail(fn, "the workspace is missing, too small or not 16-byte aligned");
  if (any_meet({block_of(workspace_dev, need)}, {dx, ds, dgain, dy, sum, dsum, gain})) return fail(fn, kOnWorkspace);
  ast::rms_norm_bwd(stream_of(hip_stream), *cfg, dy_dev, sum_dev, gain_dev, dsum_dev, dx_dev, ds_dev, dgain_dev, accumulate != 0,
                    workspace_dev);
  return launched(fn);
}

ast_status asteroid_recurrence_workspace(const ast_recurrence_cfg* cfg, size_t* bytes) {
  const char* const fn = "recurrence_workspace";
  if (!bytes) return fail(fn, "NULL argument");
  if (const char* e = recurrence_cfg(cfg)) return fail(fn, e);
  *bytes = ast::recurrence_ws_bytes(*cfg);
  return AST_OK;
}

ast_status asteroid_recurrence_forward(const ast_recurrence_cfg* cfg, const ast_rows* f, const ast_rows* z, const ast_rows* o,
                                       const float* state_dev, void* y_dev, float* final_dev, float* saved_dev,
                                       void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
  const char* const fn = "recurrence_forward";
  if (const char* e = recurrence_cfg(cfg)) return fail(fn, e);
  for (const ast_rows* r : {f, z, o ? o : z})
    if (const char* e = rows_ok(*cfg, r, false)) return fail(fn, e);
  if (!aligned(state_dev, 4) || !aligned(final_dev, 4) || !aligned(saved_dev, 4)) return fail(fn, "states must be 4-byte aligned");
  if (cfg->tokens > 0 && (!y_dev || !aligned(y_dev, esize(cfg->dtype)))) return fail(fn, "y_dev must be non-NULL and aligned to its element size");
  const ast_rows dense = {y_dev, cfg->channels};
  const Area y = rows_of(*cfg, &dense), fin = states_of(*cfg, final_dev), kept = saved_of(*cfg, saved_dev);
  if (any_meet({y, fin, kept})) return fail(fn, "outputs overlap");
  const Area xf = rows_of(*cfg, f), xz = rows_of(*cfg, z), xo = rows_of(*cfg, o), xs = states_of(*cfg, state_dev), off = offsets_of(*cfg);
  if (any_meet({y}, {xf, xz, xo}, true) || any_meet({y}, {xs, off}) || any_meet({fin}, {xs}, true) || any_meet({fin}, {xf, xz, xo, off}) ||
      any_meet({kept}, {xf, xz, xo, xs, off}))
    return fail(fn, kOnInput);
  const size_t need = ast::recurrence_ws_bytes(*cfg);
  if (need && (!workspace_dev || workspace_bytes < need || !aligned(workspace_dev, 16)))
    return fail(fn, "the workspace is missing, too small or not 16-byte aligned");
  if (any_meet({block_of(workspace_dev, need)}, {y, fin, kept, xf, xz, xo, xs, off})) return fail(fn, kOnWorkspace);
  ast::recurrence_fwd(stream_of(hip_stream), *cfg, *f, *z, o, state_dev, y_dev, final_dev, saved_dev, workspace_dev);
  return launched(fn);
}

ast_status asteroid_recurrence_backward(const ast_recurrence_cfg* cfg, const ast_rows* dy, const ast_rows* f, const ast_rows* z,
                                        const ast_rows* o, const float* state_dev, const float* saved_dev,
                                        const float* dfinal_dev, const ast_rows* df, const ast_rows* dz, const ast_rows* dgo,
                                        float* dstate_dev, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
  const char* const fn = "recurrence_backward";
  if (const char* e = recurrence_cfg(cfg)) return fail(fn, e);
  if (!o != !dgo) return fail(fn, "o and its gradient go together");
  for (const ast_rows* r : {dy, f, z, o ? o : z})
    if (const char* e = rows_ok(*cfg, r, false)) return fail(fn, e);
  for (const ast_rows* r : {df, dz, dgo ? dgo : dz})
    if (const char* e = rows_ok(*cfg, r, true)) return fail(fn, e);
  const Area gf = rows_of(*cfg, df), gz = rows_of(*cfg, dz), go = rows_of(*cfg, dgo), gs = states_of(*cfg, dstate_dev);
  if (any_meet({gf, gz, go, gs})) return fail(fn, "outputs overlap");
  const Area ydy = rows_of(*cfg, dy), xf = rows_of(*cfg, f), xz = rows_of(*cfg, z), xo = rows_of(*cfg, o), off = offsets_of(*cfg);
  const Area xs = states_of(*cfg, state_dev), xd = states_of(*cfg, dfinal_dev), kept = saved_of(*cfg, saved_dev);
  if (any_meet({gf, gz, go}, {ydy, xf, xz, xo}, true) || any_meet({gf, gz, go}, {xs, xd, kept, off}) || any_meet({gs}, {xs, xd}, true) ||
      any_meet({gs}, {ydy, xf, xz, xo, kept, off}))
    return fail(fn, kOnInput);
  if (cfg->tokens > 0 && !saved_dev) return fail(fn, "saved_dev is NULL");
  if (!aligned(state_dev, 4) || !aligned(saved_dev, 4) || !aligned(dfinal_dev, 4) || !aligned(dstate_dev, 4))
    return fail(fn, "states must be 4-byte aligned");
  const size_t need = ast::recurrence_ws_bytes(*cfg);
  if (need && (!workspace_dev || workspace_bytes < need || !aligned(workspace_dev, 16)))
    return fail(fn, "the workspace is missing, too small or not 16-byte aligned");
  if (any_meet({block_of(workspace_dev, need)}, {gf, gz, go, gs, ydy, xf, xz, xo, xs, xd, kept, off})) return fail(fn, kOnWorkspace);
  ast::recurrence_bwd(stream_of(hip_stream), *cfg, *dy, *f, *z, o, state_dev, saved_dev, dfinal_dev, *df, *dz, dgo, dstate_dev,
                      workspace_dev);
  return launched(fn);
}

ast_status asteroid_distill_forward(const ast_distill_cfg* cfg, const void* logits_dev, const int32_t* ids_dev, const void* teacher_dev,
                                    float* loss_dev, float* stats_dev, void* hip_stream) {
  const char* const fn = "distill_forward";
  if (const char* e = distill_cfg(cfg)) return fail(fn, e);
  if (cfg->rows == 0) return AST_OK;
  if (const char* e = distill_inputs(*cfg, logits_dev, ids_dev, teacher_dev)) return fail(fn, e);
  if (!loss_dev || !stats_dev || !aligned(loss_dev, 4) || !aligned(stats_dev, 4)) return fail(fn, "loss_dev and stats_dev must be non-NULL and 4-byte aligned");
  const Area loss = a_row(*cfg, loss_dev), stats = a_row(*cfg, stats_dev, 3);
  if (any_meet({loss, stats})) return fail(fn, "outputs overlap");
  if (any_meet({loss, stats}, {vocab_rows(*cfg, logits_dev, cfg->logits_stride), entries_of(*cfg, ids_dev, 4),
                               entries_of(*cfg, teacher_dev, esize(cfg->teacher_dtype)), a_row(*cfg, cfg->labels_dev)}))
    return fail(fn, kOnInput);
  ast::distill_fwd(stream_of(hip_stream), *cfg, logits_dev, ids_dev, teacher_dev, loss_dev, stats_dev);
  return launched(fn);
}

ast_status asteroid_distill_backward(const ast_distill_cfg* cfg, const float* dloss_dev, const void* logits_dev,
                                     const int32_t* ids_dev, const void* teacher_dev, const float* stats_dev, void* dlogits_dev,
                                     int64_t dlogits_stride, void* hip_stream) {
  const char* const fn = "distill_backward";
  if (const char* e = distill_cfg(cfg)) return fail(fn, e);
  if (cfg->rows == 0) return AST_OK;
  if (const char* e = distill_inputs(*cfg, logits_dev, ids_dev, teacher_dev)) return fail(fn, e);
  if (const char* e = distill_gradient(*cfg, dloss_dev, logits_dev, ids_dev, teacher_dev, dlogits_dev, dlogits_stride)) return fail(fn, e);
  if (!stats_dev || !aligned(stats_dev, 4)) return fail(fn, "stats_dev must be non-NULL and 4-byte aligned");
  if (any_meet({vocab_rows(*cfg, dlogits_dev, dlogits_stride)}, {a_row(*cfg, stats_dev, 3)})) return fail(fn, kOnInput);
  ast::distill_bwd(stream_of(hip_stream), *cfg, dloss_dev, logits_dev, ids_dev, teacher_dev, stats_dev, dlogits_dev, dlogits_stride);
  return launched(fn);
}

ast_status asteroid_distill_step_workspace(const ast_distill_cfg* cfg, size_t* bytes) {
  const char* const fn = "distill_step_workspace";
  if (!bytes) return fail(fn, "NULL argument");
  if (const char* e = distill_cfg(cfg)) return fail(fn, e);
  *bytes = ast::distill_step_ws_bytes(*cfg);
  return AST_OK;
}

ast_status asteroid_distill_step(const ast_distill_cfg* cfg, const float* dloss_dev, const void* logits_dev, const int32_t* ids_dev,
                                 const void* teacher_dev, float* loss_dev, void* dlogits_dev, int64_t dlogits_stride, void* workspace_dev,
                                 size_t workspace_bytes, void* hip_stream) {
  const char* const fn = "distill_step";
  if (const char* e = distill_cfg(cfg)) return fail(fn, e);
  if (cfg->rows == 0) return AST_OK;
  if (const char* e = distill_inputs(*cfg, logits_dev, ids_dev, teacher_dev)) return fail(fn, e);
  if (const char* e = distill_gradient(*cfg, dloss_dev, logits_dev, ids_dev, teacher_dev, dlogits_dev, dlogits_stride)) return fail(fn, e);
  if (!loss_dev || !aligned(loss_dev, 4)) return fail(fn, "loss_dev must be non-NULL and 4-byte aligned");
  const Area loss = a_row(*cfg, loss_dev), g = vocab_rows(*cfg, dlogits_dev, dlogits_stride), z = vocab_rows(*cfg, logits_dev, cfg->logits_stride);
  if (any_meet({loss, g})) return fail(fn, "outputs overlap");
  // (dloss too: of a row in slices one writes the loss while others may still have to read dloss)
  const Area id = entries_of(*cfg, ids_dev, 4), top = entries_of(*cfg, teacher_dev, esize(cfg->teacher_dtype));
  const Area w = a_row(*cfg, dloss_dev), lab = a_row(*cfg, cfg->labels_dev);
  if (any_meet({loss}, {z, id, top, w, lab})) return fail(fn, kOnInput);
  const size_t need = ast::distill_step_ws_bytes(*cfg);
  if (need && (!workspace_dev || workspace_bytes < need || !aligned(workspace_dev, 16)))
    return fail(fn, "the workspace is missing, too small or not 16-byte aligned");
  if (any_meet({block_of(workspace_dev, need)}, {loss, g, z, id, top, w, lab})) return fail(fn, kOnWorkspace);
  ast::distill_step(stream_of(hip_stream), *cfg, dloss_dev, logits_dev, ids_dev, teacher_dev, loss_dev, dlogits_dev, dlogits_stride,
                    workspace_dev);
  return launched(fn);
}

ast_status asteroid_stash8_bytes(int64_t rows, int64_t cols, size_t* bytes) {
  const char* const fn = "stash8_bytes";
  if (!bytes) return fail(fn, "NULL argument");
  if (const char* e = stash_sizes(rows, cols)) return fail(fn, e);
  *bytes = ast::stash8_bytes(rows, cols);
  return AST_OK;
}

ast_status asteroid_stash8_pack(const void* x_dev, int32_t x_dtype, int64_t rows, int64_t cols, void* stash_dev, void* hip_stream) {
  const char* const fn = "stash8_pack";
  if (!dtype_ok(x_dtype)) return fail(fn, "unknown dtype");
  if (const char* e = stash_sizes(rows, cols)) return fail(fn, e);
  if (rows == 0) return AST_OK;
  if (!x_dev || !stash_dev) return fail(fn, "NULL argument");
  if (!aligned(x_dev, esize(x_dtype)) || !aligned(stash_dev, 16)) return fail(fn, "x_dev must be aligned to its element size, the stash to 16 bytes");
  ast::stash8_pack(stream_of(hip_stream), x_dev, x_dtype != AST_F32, rows, cols, stash_dev);
  return launched(fn);
}

ast_status asteroid_stash8_unpack(const void* stash_dev, int64_t rows, int64_t cols, void* x_dev, int32_t x_dtype, void* hip_stream) {
  const char* const fn = "stash8_unpack";
  if (!dtype_ok(x_dtype)) return fail(fn, "unknown dtype");
  if (const char* e = stash_sizes(rows, cols)) return fail(fn, e);
  if (rows == 0) return AST_OK;
  if (!x_dev || !stash_dev) return fail(fn, "NULL argument");
  if (!aligned(x_dev, esize(x_dtype)) || !aligned(stash_dev, 16)) return fail(fn, "x_dev must be aligned to its element size, the stash to 16 bytes");
  ast::stash8_unpack(stream_of(hip_stream), stash_dev, rows, cols, x_dev, x_dtype != AST_F32);
  return launched(fn);
}

ast_status asteroid_linear_wgrad_stash8_workspace(int64_t rows, int64_t in, int64_t out, size_t* bytes) {
  const char* const fn = "linear_wgrad_stash8_workspace";
  if (!bytes) return fail(fn, "NULL argument");
  if (const char* e = wgrad_sizes(rows, in, out)) return fail(fn, e);
  *bytes = ast::linear_wgrad_stash8_ws_bytes(rows, in, out);
  return AST_OK;
}

ast_status asteroid_linear_wgrad_stash8(const void* dy_dev, const void* stash_dev, int64_t rows, int64_t in, int64_t out,
                                        float* dw_dev, float* db_dev, int32_t accumulate, void* workspace_dev,
                                        size_t workspace_bytes, void* hip_stream) {
  const char* const fn = "linear_wgrad_stash8";
  if (const char* e = wgrad_sizes(rows, in, out)) return fail(fn, e);
  if (!dw_dev || !aligned(dw_dev, 4) || !aligned(db_dev, 4)) return fail(fn, "dw_dev must be non-NULL, dw_dev and db_dev 4-byte aligned");
  if (rows > 0) {
    if (!dy_dev || !stash_dev) return fail(fn, "NULL argument");
    if (!aligned(dy_dev, 2) || !aligned(stash_dev, 16)) return fail(fn, "dy_dev must be 2-byte aligned, the stash 16-byte aligned");
  }
  const size_t need = ast::linear_wgrad_stash8_ws_bytes(rows, in, out);
  if (need && (!workspace_dev || workspace_bytes < need || !aligned(workspace_dev, 16)))
    return fail(fn, "the workspace is missing, too small or not 16-byte aligned");
  if (db_dev && db_dev < dw_dev + in * out && dw_dev < db_dev + out) return fail(fn, "dw_dev and db_dev overlap");
  ast::linear_wgrad_stash8(stream_of(hip_stream), dy_dev, stash_dev, rows, in, out, dw_dev, db_dev, accumulate != 0, workspace_dev);
  return launched(fn);
}

ast_status asteroid_gelu_backward_stash8(const void* dy_dev, int32_t dtype, const void* stash_dev, int64_t rows, int64_t cols,
                                         void* dz_dev, void* hip_stream) {
  const char* const fn = "gelu_backward_stash8";
  if (!dtype_ok(dtype)) return fail(fn, "unknown dtype");
  if (const char* e = stash_sizes(rows, cols)) return fail(fn, e);
  if (rows == 0) return AST_OK;
  if (!dy_dev || !stash_dev || !dz_dev) return fail(fn, "NULL argument");
  if (!aligned(dy_dev, esize(dtype)) || !aligned(dz_dev, esize(dtype)) || !aligned(stash_dev, 16))
    return fail(fn, "dy_dev and dz_dev must be aligned to their element size, the stash to 16 bytes");
  ast::gelu_bwd_stash8(stream_of(hip_stream), dy_dev, dtype != AST_F32, stash_dev, rows, cols, dz_dev);
  return launched(fn);
}

}  // extern "C"
