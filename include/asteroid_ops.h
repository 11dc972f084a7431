/*
 * asteroid_ops.h -- C ABI of the single operators of language-model stages (MI355X).
 *
 * A stage (asteroid.h) runs whole layers; the calls below are the operators that the stages of a
 * language model are made of beside those layers, for callers that drive them one by one:
 *
 *   embedding      rows of a token table, scaled; its gradient, summed in the order of the tokens
 *   qk_norm_rope   RMS norm of every query and key head with a gain, then the rotation by the
 *                  token's position, in one pass; and its gradient
 *   stash8         activations that are kept in 8 bits between the forward and the backward pass of a
 *                  micro-batch (the ACT term of Eq. (3)), and what the backward pass makes of them:
 *                  the weight gradient of a dense layer, the gradient through GELU
 *
 * Conventions: `*_dev` is DEVICE memory of the caller on the device that is current and owns
 * `hip_stream` (a hipStream_t; NULL = the default stream).  Every call enqueues kernels on that stream
 * and nothing else: no allocation, no memset, no host synchronisation, nothing kept between calls, so a
 * call may be recorded into a HIP graph.  `workspace_dev` is the call's alone until the stream has
 * passed it: calls that may overlap in time (two streams, two graphs replayed side by side) take one
 * each.  Its contents before the call do not matter.  Outputs may not overlap each other, nor inputs or
 * the workspace except where a call allows it.
 * Element types are AST_F32 and AST_BF16_F32ACC (bf16) of ast_dtype; sums, norms and angles are formed
 * in 32 bits or more and every result is rounded once.  Results do not depend on the order in which
 * blocks run: equal calls give equal bits.
 * Pointers are aligned to their element size (AST_EINVAL otherwise); 16-byte aligned ones are read and
 * written faster.  Workspaces and stash buffers are 16-byte aligned.
 * Every function returns an ast_status; asteroid_last_error() gives the message of a failure.
 */
#ifndef ASTEROID_OPS_H
#define ASTEROID_OPS_H

#include <stddef.h>
#include <stdint.h>

#include "asteroid.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------ token embedding
 *   y[t][:] = scale * table[ids[t]][:]          0 where ids[t] lies outside [0, rows) (padding)
 * ids_dev int32[tokens], table_dev [rows][width], y_dev [tokens][width].
 * tokens >= 0 (0: nothing is done), rows in [1, 2^31 - 2], tokens < 2^31, width in [1, 2^20], scale finite. */
ast_status asteroid_embedding_forward(const int32_t* ids_dev, int64_t tokens, const void* table_dev,
                                      int32_t table_dtype, int64_t rows, int64_t width, float scale,
                                      void* y_dev, int32_t y_dtype, void* hip_stream);

/*   dtable[v][:] = scale * sum over t with ids[t] == v of dy[t][:]      (accumulate == 0: every row is written)
 *   dtable[v][:] += ...                                                 (accumulate != 0: rows without a token stay)
 * dy_dev [tokens][width], dtable_dev fp32 [rows][width].  Tokens outside [0, rows) add nothing.  The
 * tokens are sorted (stably) by id, so one writer adds a row's tokens in order, however often an id
 * occurs.  The workspace size is a function of tokens, rows and width alone. */
ast_status asteroid_embedding_backward_workspace(int64_t tokens, int64_t rows, int64_t width, size_t* bytes);
ast_status asteroid_embedding_backward(const int32_t* ids_dev, int64_t tokens, const void* dy_dev,
                                       int32_t dy_dtype, int64_t rows, int64_t width, float scale,
                                       int32_t accumulate, float* dtable_dev, void* workspace_dev,
                                       size_t workspace_bytes, void* hip_stream);

/* ------------------------------------------------------------------ norm and rotation of queries and keys
 * For every token t and head, with x its head_dim values:
 *   n = x / sqrt(mean(x^2) + eps),  u_i = gain_i * n_i,  y = u rotated by the token's position p:
 *   the first `rotary` values form rotary / 2 pairs; pair i turns by the angle p * theta^(-2 i / rotary):
 *     (y_a, y_b) = (u_a cos - u_b sin, u_a sin + u_b cos)
 *   a, b = i, i + rotary / 2 (interleaved == 0) or 2 i, 2 i + 1 (interleaved != 0); the values from
 *   `rotary` on are not rotated.  Angles are formed in 64 bits.
 * A set of heads is one tensor [tokens][heads][head_dim] with unit stride inside a head and any strides
 * (in elements, tokens < 2^31, heads <= 2^40; those of an output leave no two heads on top of each other): queries and keys may lie inside one packed projection.
 * positions_dev int32[tokens], or NULL: token t stands at t modulo `period` (>= 1; sequences of that
 * length one after the other).  Gains are fp32[head_dim].  Query and key heads may differ in number.
 * head_dim in [1, 256], rotary even in [0, head_dim], eps > 0, theta > 0, tokens < 2^31, heads in [1, 65535].
 * y may be x itself (same pointer and strides). */
typedef struct {
  const void* dev;      /* first value of the first token's first head */
  int64_t token_stride; /* elements */
  int64_t head_stride;  /* elements */
  int32_t heads;
} ast_heads;

typedef struct {
  int64_t tokens;
  int32_t dtype;       /* ast_dtype of every head tensor of the call */
  int32_t head_dim;
  int32_t rotary;
  int32_t interleaved;
  float eps;
  double theta;
  const int32_t* positions_dev; /* or NULL */
  int32_t period;               /* used where positions_dev is NULL */
} ast_qk_cfg;

ast_status asteroid_qk_norm_rope_forward(const ast_qk_cfg* cfg, const ast_heads* q, const ast_heads* k,
                                         const float* q_gain_dev, const float* k_gain_dev, const ast_heads* yq,
                                         const ast_heads* yk, void* hip_stream);

/* Gradients: dq, dk of the inputs (the norms are formed again from q and k), and of the gains, fp32[head_dim],
 * written (accumulate == 0) or added to.  dq may be dyq itself and dk dyk (same pointer and strides). */
ast_status asteroid_qk_norm_rope_backward_workspace(const ast_qk_cfg* cfg, int32_t q_heads, int32_t k_heads,
                                                    size_t* bytes);
ast_status asteroid_qk_norm_rope_backward(const ast_qk_cfg* cfg, const ast_heads* dyq, const ast_heads* dyk,
                                          const ast_heads* q, const ast_heads* k, const float* q_gain_dev,
                                          const float* k_gain_dev, const ast_heads* dq, const ast_heads* dk,
                                          float* dq_gain_dev, float* dk_gain_dev, int32_t accumulate,
                                          void* workspace_dev, size_t workspace_bytes, void* hip_stream);

/* ------------------------------------------------------------------ activations kept in 8 bits
 * A matrix x [rows][cols] is kept in blocks of 32 consecutive values of a row (the last block of a row is
 * filled up with zeros).  With e the least integer in [-126, 121] for which 127 * 2^e >= max |x| of a block:
 *   q = round-to-nearest-even(x / 2^e)  (one signed byte a value),   restored: x' = q * 2^e
 * so |x' - x| <= 2^e / 2, a restored value is exact in bf16 (and fp32), and packing a restored matrix
 * gives the same values again.  (127 * 2^121, 0.8 % below the largest fp32 value, is the largest that is
 * kept: values beyond it are restored as it.)  A block that holds an infinity or a NaN is restored as NaN.
 * Layout of the buffer (asteroid_stash8_bytes, 16-byte aligned): rows * P bytes of q, P = cols rounded up
 * to 32, then rows * P / 32 bytes e + 127 (255: a block that is not finite).  rows < 2^31, rows * P < 2^40,
 * cols in [1, 2^20]. */
ast_status asteroid_stash8_bytes(int64_t rows, int64_t cols, size_t* bytes);
ast_status asteroid_stash8_pack(const void* x_dev, int32_t x_dtype, int64_t rows, int64_t cols, void* stash_dev,
                                void* hip_stream);
ast_status asteroid_stash8_unpack(const void* stash_dev, int64_t rows, int64_t cols, void* x_dev, int32_t x_dtype,
                                  void* hip_stream);

/* Weight and bias gradient of a dense layer y = x W^T + b whose input x [rows][in] was kept:
 *   dw[out][in] (+)= sum_r dy[r][out] * x'[r][in],   db[out] (+)= sum_r dy[r][out]
 * dy_dev bf16 [rows][out]; dw_dev, db_dev fp32 (db_dev may be NULL); accumulate == 0: written, else added to.
 * in, out in [1, 2^20].  rows == 0 is a sum of nothing. */
ast_status asteroid_linear_wgrad_stash8_workspace(int64_t rows, int64_t in, int64_t out, size_t* bytes);
ast_status asteroid_linear_wgrad_stash8(const void* dy_dev, const void* stash_dev, int64_t rows, int64_t in,
                                        int64_t out, float* dw_dev, float* db_dev, int32_t accumulate,
                                        void* workspace_dev, size_t workspace_bytes, void* hip_stream);

/* Gradient through y = GELU(z) (the exact erf form) whose pre-activation z [rows][cols] was kept:
 *   dz = dy * (Phi(z') + z' phi(z'))          dz_dev may be dy_dev. */
ast_status asteroid_gelu_backward_stash8(const void* dy_dev, int32_t dtype, const void* stash_dev, int64_t rows,
                                         int64_t cols, void* dz_dev, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* ASTEROID_OPS_H */
