// The single operators of language-model stages: launches behind include/asteroid_ops.h and the stage executor.
// Arguments have been checked; everything is enqueued on `st`.
#pragma once
#include <hip/hip_runtime.h>
#include <limits.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/asteroid_ops.h"

namespace ast {

// ---- token embedding (op_embedding.hip)
void embedding_fwd(hipStream_t st, const int32_t* ids, int64_t tokens, const void* table, bool table_bf16, int64_t rows,
                   int64_t width, float scale, void* y, bool y_bf16);
size_t embedding_bwd_ws_bytes(int64_t tokens, int64_t rows, int64_t width);
void embedding_bwd(hipStream_t st, const int32_t* ids, int64_t tokens, const void* dy, bool dy_bf16, int64_t rows,
                   int64_t width, float scale, bool accumulate, float* dtable, void* ws);

// ---- norm and rotation of queries and keys (op_qk_norm_rope.hip)
void qk_norm_rope_fwd(hipStream_t st, const ast_qk_cfg& c, const ast_heads& q, const ast_heads& k, const float* gq,
                      const float* gk, const ast_heads& yq, const ast_heads& yk);
size_t qk_norm_rope_bwd_ws_bytes(int64_t tokens, int head_dim);
void qk_norm_rope_bwd(hipStream_t st, const ast_qk_cfg& c, const ast_heads& dyq, const ast_heads& dyk, const ast_heads& q,
                      const ast_heads& k, const float* gq, const float* gk, const ast_heads& dq, const ast_heads& dk,
                      float* dgq, float* dgk, bool accumulate, void* ws);

// ---- RMS norm with the residual's addition (op_rms_norm.hip)
void rms_norm_fwd(hipStream_t st, const ast_norm_cfg& c, const void* x, const void* residual, const float* gain, void* y,
                  void* sum, void* stash);
size_t rms_norm_bwd_ws_bytes(int64_t rows, int64_t width);
void rms_norm_bwd(hipStream_t st, const ast_norm_cfg& c, const void* dy, const void* sum, const float* gain, const void* dsum,
                  void* dx, void* ds, float* dgain, bool accumulate, void* ws);

// ---- gated linear recurrence (op_recurrence.hip)
size_t recurrence_ws_bytes(const ast_recurrence_cfg& c);
void recurrence_fwd(hipStream_t st, const ast_recurrence_cfg& c, const ast_rows& f, const ast_rows& z, const ast_rows* o,
                    const float* state, void* y, float* final, float* saved, void* ws);
void recurrence_bwd(hipStream_t st, const ast_recurrence_cfg& c, const ast_rows& dy, const ast_rows& f, const ast_rows& z,
                    const ast_rows* o, const float* state, const float* saved, const float* dfinal, const ast_rows& df,
                    const ast_rows& dz, const ast_rows* dgo, float* dstate, void* ws);

// ---- distillation from a teacher's top logits (op_distill.hip)
size_t distill_step_ws_bytes(const ast_distill_cfg& c);
void distill_fwd(hipStream_t st, const ast_distill_cfg& c, const void* z, const int32_t* ids, const void* t, float* loss, float* stats);
void distill_bwd(hipStream_t st, const ast_distill_cfg& c, const float* dloss, const void* z, const int32_t* ids, const void* t,
                 const float* stats, void* dz, int64_t dz_stride);
void distill_step(hipStream_t st, const ast_distill_cfg& c, const float* dloss, const void* z, const int32_t* ids, const void* t,
                  float* loss, void* dz, int64_t dz_stride, void* ws);

// ---- activations kept in 8 bits (op_stash8.hip, op_stash8_wgrad.hip)
constexpr int kStash8Block = 32;  // values that share a scale
inline int64_t stash8_pitch(int64_t cols) { return (cols + kStash8Block - 1) / kStash8Block * kStash8Block; }
inline size_t stash8_bytes(int64_t rows, int64_t cols) {
  return ((size_t)rows * (size_t)(stash8_pitch(cols) / kStash8Block) * (kStash8Block + 1) + 15) / 16 * 16;
}
inline const uint8_t* stash8_scales(const void* stash, int64_t rows, int64_t cols) {
  return static_cast<const uint8_t*>(stash) + rows * stash8_pitch(cols);
}
void stash8_pack(hipStream_t st, const void* x, bool bf16, int64_t rows, int64_t cols, void* stash);
void stash8_unpack(hipStream_t st, const void* stash, int64_t rows, int64_t cols, void* x, bool bf16);
void gelu_bwd_stash8(hipStream_t st, const void* dy, bool bf16, const void* stash, int64_t rows, int64_t cols, void* dz);
// most: an upper bound on the shares of the rows, for callers whose workspace is limited (one share takes none)
size_t linear_wgrad_stash8_ws_bytes(int64_t rows, int64_t in, int64_t out, int most = INT_MAX);
// Several such gradients, each added to dw and db, in one launch: dy 16-byte aligned with out a multiple of 8, nothing in shares (no
// workspace).  A stage builds the tables once: `task` is host memory of stash8_group_task_bytes(), blocks_dev holds pairs
// (product, block of it) of uint32_t.
size_t stash8_group_task_bytes();
int stash8_group_blocks(int64_t in, int64_t out);
void stash8_group_task(void* task, const void* dy, const void* stash, int64_t rows, int64_t in, int64_t out, float* dw, float* db);
void linear_wgrad_stash8_group(hipStream_t st, const void* tasks_dev, const void* blocks_dev, int blocks);
void linear_wgrad_stash8(hipStream_t st, const void* dy, const void* stash, int64_t rows, int64_t in, int64_t out, float* dw,
                         float* db, bool accumulate, void* ws, int most = INT_MAX);

}  // namespace ast
