// C ABI of the single operators (include/asteroid_ops.h): argument checks, then the launches of ops.h.
#include <cmath>
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
