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
 *   rms_norm       RMS norm between two blocks with the residual's addition, also with the result in
 *                  8 bits for the weight gradient of the layer behind it; and its gradient
 *   recurrence     a gated linear recurrence over the tokens of sequences, with states in and out; and
 *                  its gradient
 *   distill        the loss of the last stage: the divergence from a teacher's top logits, mixed with
 *                  the cross entropy of labels; and its gradient
 *
 * Conventions: `*_dev` is DEVICE memory of the caller on the device that is current and owns
 * `hip_stream` (a hipStream_t; NULL = the default stream).  Every call enqueues kernels on that stream
 * and nothing else: no allocation, no memset, no host synchronisation, nothing kept between calls, so a
 * call may be recorded into a HIP graph.  `workspace_dev` is the call's alone until the stream has
 * passed it: calls that may overlap in time (two streams, two graphs replayed side by side) take one
 * each.  Its contents before the call do not matter.  Outputs may not overlap each other, nor inputs or
 * the workspace except where a call allows it; rms_norm, recurrence and distill refuse it (rows
 * that lie between those of another tensor, as parts of one packed tensor do, are taken where the strides are equal).
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

/* ------------------------------------------------------------------ RMS norm with the residual's addition
 *   s = x + residual, rounded to sum_dtype;   y = s / sqrt(mean(s^2) + eps) * gain      (of every row)
 * x_dev, y_dev [rows][width] of dtype; residual_dev, sum_dev [rows][width] of sum_dtype, which is dtype or AST_F32 (an fp32
 * residual stream between bf16 layers); gain_dev fp32[width].  The norm is that of s as it is written.
 * residual_dev == NULL: s is x, sum_dtype == dtype, nothing is written to sum_dev (NULL).
 * stash_dev (NULL: none) receives y, as it is written, in 8 bits: the bytes of asteroid_stash8_pack(y_dev).  (s is the same with and
 * without it; y too, bit for bit, where width is a multiple of 8, otherwise the squares may be added up in another order.)
 * rows < 2^31, width in [1, 16384], eps >= 2^-126; squares are added up in fp32 (a row whose sum that does not hold: y is 0).
 * sum_dev may be residual_dev, y_dev may be x_dev, and where the types are the same sum_dev may be x_dev and y_dev residual_dev. */
typedef struct {
  int64_t rows;
  int64_t width;
  int32_t dtype;     /* of x, y, dy, dx */
  int32_t sum_dtype; /* of the residual, the sum and their gradients */
  float eps;
} ast_norm_cfg;

ast_status asteroid_rms_norm_forward(const ast_norm_cfg* cfg, const void* x_dev, const void* residual_dev, const float* gain_dev,
                                     void* y_dev, void* sum_dev, void* stash_dev, void* hip_stream);

/* Gradients, from the sum s (x, where nothing was added):
 *   ds = dsum + rho (dy gain - n mean(dy gain n)),  n = s rho,  rho = 1 / sqrt(mean(s^2) + eps);   dgain (+)= sum over the rows of dy n
 * dsum_dev (NULL: none): the gradient that reaches the sum from further on, of sum_dtype.  ds is the gradient of x and of
 * the residual: dx_dev receives it in dtype, ds_dev in sum_dtype; either may be NULL, not both.  dgain_dev fp32[width], written
 * (accumulate == 0) or added to; it may be gain_dev.  dx_dev may be dy_dev, ds_dev may be dsum_dev or sum_dev; where the types are the
 * same either output may be any of the three inputs. */
ast_status asteroid_rms_norm_backward_workspace(const ast_norm_cfg* cfg, size_t* bytes);
ast_status asteroid_rms_norm_backward(const ast_norm_cfg* cfg, const void* dy_dev, const void* sum_dev, const float* gain_dev,
                                      const void* dsum_dev, void* dx_dev, void* ds_dev, float* dgain_dev, int32_t accumulate,
                                      void* workspace_dev, size_t workspace_bytes, void* hip_stream);

/* ------------------------------------------------------------------ gated linear recurrence
 * For every channel of a sequence, from its state h on:
 *   a_t = sigmoid(f_t),   h_t = a_t h_{t-1} + (1 - a_t) z_t,   y_t = h_t * o_t sigmoid(o_t)      (o == NULL: y_t = h_t)
 * Sequences lie one behind the other in `tokens` rows: sequence s has the tokens [offsets[s], offsets[s + 1])
 * (offsets_dev int32[sequences + 1], not decreasing, within [0, tokens]; a length may be zero), or, with
 * offsets_dev == NULL, `period` tokens (the last one what is left: sequences = tokens / period rounded up).  Rows that belong to
 * no sequence are not read into any result and not written.  (Offsets that decrease or lie outside give results
 * without meaning, but no access outside the tensors.)
 * f, z, o: rows of `channels` values of dtype with any stride (elements, >= 0): parts of one packed projection.
 * y_dev: [tokens][channels], dense; it may be f, z or o where that is dense too.
 * state_dev fp32 [sequences][channels]: the state in front of every sequence, NULL: 0.  final_dev, the same shape, or NULL:
 * receives the state behind every sequence (of one without tokens: its state); it may be state_dev.  States are
 * fp32 throughout, and nothing of a sequence, infinities and NaN included, reaches another.
 * saved_dev (NULL: no backward pass follows): fp32 [tokens / AST_RECURRENCE_CHUNK rounded up][channels], for the backward
 * pass: the state in front of every AST_RECURRENCE_CHUNK-th token.
 * tokens < 2^31, channels in [1, 2^20], tokens (rounded up to 512) * channels (rounded up to 64) <= 2^34, sequences in
 * [0, 2^31 - 2], period in [1, 2^31). */
#define AST_RECURRENCE_CHUNK 64

typedef struct {
  const void* dev; /* first value of the first row */
  int64_t stride;  /* elements from row to row */
} ast_rows;

typedef struct {
  int64_t tokens;
  int64_t channels;
  int32_t dtype; /* of f, z, o, y and their gradients */
  const int32_t* offsets_dev; /* or NULL */
  int64_t sequences;          /* used where offsets_dev is given */
  int64_t period;             /* used where offsets_dev is NULL */
} ast_recurrence_cfg;

/* (the size looks at whether offsets_dev is given, not at what it holds; it may be 0) */
ast_status asteroid_recurrence_workspace(const ast_recurrence_cfg* cfg, size_t* bytes);
ast_status asteroid_recurrence_forward(const ast_recurrence_cfg* cfg, const ast_rows* f, const ast_rows* z, const ast_rows* o,
                                       const float* state_dev, void* y_dev, float* final_dev, float* saved_dev,
                                       void* workspace_dev, size_t workspace_bytes, void* hip_stream);

/* Gradients of all inputs from dy, dfinal_dev (NULL: none; fp32 [sequences][channels]), and saved_dev of the
 * forward pass of the same inputs.  df, dz, dgo (NULL iff o is) are rows of any stride >= channels, and may be the
 * tensors of f, z, o (same pointer and stride), or dy; they may not overlap each other.  dstate_dev (or NULL): fp32
 * [sequences][channels], the gradient of state_dev (of a sequence without tokens: its dfinal, or 0); it may be dfinal_dev or
 * state_dev. */
ast_status asteroid_recurrence_backward(const ast_recurrence_cfg* cfg, const ast_rows* dy, const ast_rows* f, const ast_rows* z,
                                        const ast_rows* o, const float* state_dev, const float* saved_dev,
                                        const float* dfinal_dev, const ast_rows* df, const ast_rows* dz, const ast_rows* dgo,
                                        float* dstate_dev, void* workspace_dev, size_t workspace_bytes, void* hip_stream);

/* ------------------------------------------------------------------ distillation from a teacher's top logits
 * Of every row z [vocab] of the student's logits, with the teacher's logits t_k at the places id_k (k < entries), temperature T
 * and label weight l:
 *   p = softmax of t / T over the row's valid entries,  q = softmax(z / T),  q1 = softmax(z)
 *   loss = (1 - l) T^2 sum_k p_k (log p_k - log q[id_k])  -  l log q1[label]
 * An entry is valid if its id lies in [0, vocab) and its logit is not -inf (others are padding); an id that stands several times
 * counts with the sum of its p.  A row without a valid entry has no first term, a row whose label lies outside [0, vocab) no
 * second one.  labels_dev int32[rows], or NULL: l is 0.
 * logits: [rows][vocab] in rows of logits_stride >= vocab elements; ids_dev int32[rows][entries], teacher_dev
 * [rows][entries]; loss_dev fp32[rows].  rows < 2^31, vocab in [1, 2^30], entries in [1, 1024], T in [2^-30, 2^30],
 * l in [0, 1].
 * stats_dev fp32[rows][3], for the backward pass: max z, sum exp((z - max) / T), sum exp(z - max) (0 without labels or with l == 0). */
typedef struct {
  int64_t rows;
  int64_t vocab;
  int64_t logits_stride;
  int32_t dtype; /* of the logits and their gradient */
  int32_t entries;
  int32_t teacher_dtype;
  float temperature;
  float label_weight;
  const int32_t* labels_dev; /* or NULL */
} ast_distill_cfg;

ast_status asteroid_distill_forward(const ast_distill_cfg* cfg, const void* logits_dev, const int32_t* ids_dev, const void* teacher_dev,
                                    float* loss_dev, float* stats_dev, void* hip_stream);

/* dlogits = dloss[row] * d loss / d z, in rows of dlogits_stride >= vocab elements; dlogits_dev may be logits_dev (with the
 * same stride).  A row whose dloss is 0 (a token that does not count) gets zeros, whatever its logits are. */
ast_status asteroid_distill_backward(const ast_distill_cfg* cfg, const float* dloss_dev, const void* logits_dev,
                                     const int32_t* ids_dev, const void* teacher_dev, const float* stats_dev, void* dlogits_dev,
                                     int64_t dlogits_stride, void* hip_stream);

/* Both at once, where dloss is known beforehand (1 / tokens, a mask): the logits are read from memory once.  The workspace may
 * be of 0 bytes (it serves few long rows). */
ast_status asteroid_distill_step_workspace(const ast_distill_cfg* cfg, size_t* bytes);
ast_status asteroid_distill_step(const ast_distill_cfg* cfg, const float* dloss_dev, const void* logits_dev, const int32_t* ids_dev,
                                 const void* teacher_dev, float* loss_dev, void* dlogits_dev, int64_t dlogits_stride,
                                 void* workspace_dev, size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* ASTEROID_OPS_H */
