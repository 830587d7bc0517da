/*
 * dycl_tokens.h - operators of networks that decide for every token: the
 * layers of a block whose each row (a token) picks k of E expert
 * sub-networks.  A logic node selects per input which sub-DNN runs next
 * (Sec. 5.3); here the selection is k of E instead of one of two, the
 * partition of the rows is by expert, and the experts' layers run on all
 * of them at once.  Around them: the norms before and after a block with
 * its gate and residual scale, and a dense layer with its epilogue.
 *
 * Tensors are row-major matrices of bf16 (uint16_t bits) or float32 with a
 * row pitch `ld*` in elements (at least the row length; rows need not be
 * packed).  All pointers but those of the size functions' are device
 * pointers, caller-owned, aligned to their element; where a call is faster
 * on 16-byte aligned rows it finds that out by itself.  Work is queued on
 * `hip_stream` (a hipStream_t, NULL = default stream); no call allocates,
 * copies to the host or waits, so all may be captured into a HIP graph.
 * Outputs and workspaces must not overlap inputs or one another, except
 * where said.  Errors are dycl_status codes with dycl_last_error()
 * (dycl.h); validation happens before any launch.  Results do not depend on
 * the order in which workgroups run, and a row's results are the same bits
 * whatever the number and the values of the rows beside it: the number of
 * rows selects a kernel, never the order of a sum.
 */
#ifndef DYCL_TOKENS_H_
#define DYCL_TOKENS_H_

#include <stddef.h>
#include <stdint.h>

#include "dycl.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of the tensors that may have either. */
typedef enum { DYCL_BF16 = 0, DYCL_F32 = 1 } dycl_type;

/*
 * The norm after a block, its gate, the residual sum and the norm before
 * the next block, in one pass over the rows:
 *   z = post(y) * act(gate) * channel_scale * row_gate
 *   h = residual_scale * x + z
 *   u = pre(h)
 * with post and pre one of
 *   DYCL_NORM_NONE   v
 *   DYCL_NORM_RMS    v / sqrt(mean(v^2) + eps) * weight + bias
 *   DYCL_NORM_LAYER  (v - mean(v)) / sqrt(mean((v - mean(v))^2) + eps) * weight + bias
 * over each row of d values.  Statistics and sums are float32; u comes
 * from the sum before h is rounded.
 *   x              [n][d] x_type, the residual stream.
 *   y              [n][d] y_type, the block's output, or NULL: z = 0 (then
 *                  post must be NONE and the gates NULL).
 *   gate           [n][d] y_type or NULL; gate_act 0 none, 1 sigmoid, 2 SiLU.
 *   row_gate       [n] float32 or NULL.  Where it is 0 the block was skipped
 *                  for that row: z = 0 whatever y and gate hold there (they
 *                  are not read).
 *   channel_scale  [d] float32 or NULL.
 *   post_weight, post_bias, pre_weight, pre_bias  [d] float32 or NULL (1, 0).
 *   h              [n][d] x_type, or NULL: not written.  May be x itself
 *                  (the same pointer and pitch) or y.
 *   u              [n][d] u_type, or NULL (then pre must be NONE).  May not
 *                  be x, y or gate.
 * 1 <= d <= 32768, n >= 0 (0 does nothing), eps >= 0.
 */
typedef enum { DYCL_NORM_NONE = 0, DYCL_NORM_RMS = 1, DYCL_NORM_LAYER = 2 } dycl_norm_kind;
int dycl_op_norm(const void* x, int x_type, int64_t ldx, const void* y, int y_type, int64_t ldy, const void* gate,
                 int64_t ldg, int gate_act, const float* row_gate, const float* channel_scale, float residual_scale,
                 int post, const float* post_weight, const float* post_bias, int pre, const float* pre_weight,
                 const float* pre_bias, float eps, int64_t n, int d, void* h, int64_t ldh, void* u, int u_type,
                 int64_t ldu, void* hip_stream);

/*
 * The choice of experts for every row, and the partition of the (row,
 * expert) pairs by expert.
 *   p = softmax(logits row) (score 0) or sigmoid(logits) (score 1), float32
 *   v = p + bias
 * An expert is closed to a row where its logit is -infinity or NaN, to all
 * rows where its bias is, and all are closed where mask[row] == 0; a logit of +infinity counts as the largest
 * finite value.  With groups > 1 the experts are `groups` runs of
 * experts / groups; a group's score is the sum of its two largest v of open
 * experts (its one v if one is open), and only the top_groups best groups
 * stay.  The k best open experts by v are chosen, best first; among equal
 * values the lowest index wins, for groups too.  Their weights are p,
 * divided by their sum if renormalise != 0 (0 if that is 0), times scale.
 *   logits   [n][experts] logits_type, pitch ldl.
 *   bias     [experts] float32 or NULL.
 *   mask     [n] uint8 or NULL.
 *   ids      [n][k] int32: the experts, -1 where fewer than k are open.
 *   weights  [n][k] float32: their weights, 0 where the id is -1.
 *   offsets  [experts + 1] int32: expert e's pairs are positions offsets[e]
 *            to offsets[e + 1] - 1; offsets[experts] counts all pairs.
 *   order    [n * k] int32: the pair (row * k + place among its choices) at
 *            each position, rows in order within an expert; -1 past the end.
 *   slots    [n][k] int32: each pair's position, -1 where the id is -1.
 *            offsets, order and slots are given together, or all NULL.
 *   workspace  dycl_op_route_workspace(n, experts, k) bytes, 8-byte aligned
 *            (may be NULL when that is 0); only the partition needs it.
 * 1 <= experts <= 1024, 1 <= k <= min(experts, 32), 1 <= groups <= 64
 * dividing experts, 1 <= top_groups <= groups, n >= 0, n * k < 2^31.
 * n == 0 writes offsets (zeros) only.
 */
size_t dycl_op_route_workspace(int64_t n, int experts, int k);
int dycl_op_route(const void* logits, int logits_type, int64_t ldl, const float* bias, const uint8_t* mask, int64_t n,
                  int experts, int groups, int top_groups, int k, int score, int renormalise, float scale, int32_t* ids,
                  float* weights, int32_t* offsets, int32_t* order, int32_t* slots, void* workspace,
                  size_t workspace_bytes, void* hip_stream);

/*
 * Weights of the products below, laid out for the matrix cores: `experts`
 * layers of n outputs on k inputs, w [experts][n][k] bf16 (contiguous), and
 * with a gate a second such tensor.  Zero-padded to 32 outputs and 64
 * inputs.  dycl_op_linear_packed_bytes returns 0 for sizes out of range
 * (1 <= n, k <= 2^20, 1 <= experts <= 1024); packed is 16-byte aligned.
 */
size_t dycl_op_linear_packed_bytes(int experts, int n, int k, int gated);
int dycl_op_linear_pack(const uint16_t* w, const uint16_t* gate, int experts, int n, int k, uint16_t* packed,
                        size_t packed_bytes, void* hip_stream);

/*
 * One layer on m rows of x:
 *   y = act(x W^T + bias) + residual                              (plain)
 *   y = (x W^T + bias) * act(x G^T + gate_bias) + residual        (gated)
 * bf16 inputs, float32 sums and epilogue, one rounding to y_type.
 *   x         [m][k] bf16, pitch ldx.
 *   packed    one layer (experts 1) from dycl_op_linear_pack.
 *   bias, gate_bias  [n] float32 or NULL (gate_bias only if gated).
 *   act       0 none, 1 ReLU, 2 exact GELU, 3 SiLU; of NaN each is NaN.
 *   residual  [m][n] bf16, pitch ldr, or NULL.
 *   y         [m][n] y_type, pitch ldy; may be the residual itself if bf16.
 *   workspace dycl_op_linear_workspace(x, ldx, m, k, n, gated) bytes, 16-byte aligned:
 *             0 (NULL) where x is 16-byte aligned and k and ldx are
 *             multiples of 8, room for aligned rows otherwise.
 * m >= 0 (0 does nothing).  A launch holds fewer than 2^23 - 1 tiles: as many
 * or more of the largest (256 rows x 256 outputs, 128 gated) return
 * DYCL_E_INVALID, here and below.
 *
 * dycl_op_linear_tile tells which kernel a product takes: tile receives the
 * rows and outputs of its tiles and how many of them a CU takes together.
 * experts 0: dycl_op_linear on `rows` rows.  experts > 0: a product of
 * dycl_op_experts over `rows` pairs (n outputs on k inputs each).  For
 * profiles and tests; results do not depend on it.
 */
int dycl_op_linear_tile(int64_t rows, int n, int k, int gated, int experts, int32_t tile[3]);
size_t dycl_op_linear_workspace(const uint16_t* x, int64_t ldx, int64_t m, int k, int n, int gated);
int dycl_op_linear(const uint16_t* x, int64_t ldx, int64_t m, int k, const uint16_t* packed, int n, int gated,
                   const float* bias, const float* gate_bias, int act, const uint16_t* residual, int64_t ldr, void* y,
                   int y_type, int64_t ldy, void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * The chosen experts' two layers on every row, weighted and summed:
 *   out[t] = residual[t] + sum over j with slots[t][j] >= 0 of
 *            weights[t][j] * (W2_e f_e(x[t]) + bias2_e),   e the pair's expert
 *   f_e(v) = act(W_e v + bias_e)  or  (W_e v + bias_e) * act(G_e v + gate_bias_e)
 * bf16 in and out; sums, epilogues, each expert's results and their weighted
 * sum are float32.  f_e is rounded to bf16, the second product's input: the
 * one rounding in between.
 *   x         [n][d] bf16, pitch ldx.
 *   packed1   experts layers of f outputs on d inputs (gated or not),
 *   packed2   experts layers of d outputs on f inputs (not gated), both
 *             from dycl_op_linear_pack.
 *   bias1, gate_bias1 [experts][f], bias2 [experts][d] float32 or NULL.
 *   weights, offsets, order, slots  as dycl_op_route writes them for n rows
 *             of k choices (indices are not checked on the device).
 *   residual  [n][d] bf16, pitch ldr, or NULL.
 *   out       [n][d] bf16, pitch ldo; may be the residual itself.
 *   workspace dycl_op_experts_workspace(x, ldx, n, experts, k, d, f) bytes,
 *             16-byte aligned.
 * n >= 0 (0 does nothing), n * k < 2^31.
 */
size_t dycl_op_experts_workspace(const uint16_t* x, int64_t ldx, int64_t n, int experts, int k, int d, int f);
int dycl_op_experts(const uint16_t* x, int64_t ldx, int64_t n, int d, int f, int experts, int k,
                    const uint16_t* packed1, int gated, const float* bias1, const float* gate_bias1, int act,
                    const uint16_t* packed2, const float* bias2, const float* weights, const int32_t* offsets,
                    const int32_t* order, const int32_t* slots, const uint16_t* residual, int64_t ldr, uint16_t* out,
                    int64_t ldo, void* workspace, size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* DYCL_TOKENS_H_ */
