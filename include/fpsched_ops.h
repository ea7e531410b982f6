/*
 * fpsched_ops.h -- C ABI of the operators that the items of a language model's pipeline stages run.
 *
 * A schedule orders items (F, B, W, R); what an item costs on this card is what the profiler of the
 * paper's Section 3 measures, and what an item runs is what Section 4 maps an instruction to.  These
 * are the operators of the stages of a language model, each with its backward pass split the way the
 * items are split (CompInputGrad and CompWeightGrad, Table 1):
 *   first stage    embedding lookup                          F, W
 *   inner stages   gated linear recurrence (mixes tokens)    F, B
 *                  gated feed-forward block (mixes channels) F, B, W
 *   last stage     log probabilities of given tokens         F, B
 * An R item is the F item run again: F keeps nothing that it does not compute from its inputs, and
 * gives the same bits for the same inputs.
 *
 * As in fpsched.h: plain pointers and sizes, 0 or a negative FPSCHED_E* code, no exception and no
 * abort.  All tensors are DEVICE memory of GPU device_id and belong to the caller, workspaces
 * included; a call allocates nothing, keeps nothing, and only enqueues kernels on hip_stream (a
 * hipStream_t, NULL = default stream), so it can be captured into a graph and replayed.  Two calls
 * may share a workspace, or a tensor that one of them writes, only if they run one after the other.
 * Workspaces are 16-byte aligned, tensors to their elements.  A size of 0 rows is no error: nothing is read, and what is
 * written of a gradient over no rows is zero.  Sums, states and softmax statistics are held in 32
 * bits; an output of a 16-bit type is rounded once, to nearest even, and nothing on the way to it is rounded to fewer than 32
 * bits but for what the feed-forward block says below.  Results are the same bits
 * from call to call (no atomic decides an order of additions).
 */
#ifndef FPSCHED_OPS_H
#define FPSCHED_OPS_H

#include "fpsched.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Types of tensor elements. */
enum { FPSCHED_BF16 = 0, FPSCHED_F16 = 1, FPSCHED_F32 = 2 };

/* ---- embedding lookup --------------------------------------------------------------------------
 * out[t][:] = scale * table[tokens[t]][:].  A token outside 0 .. n_rows - 1 (-1 for padding) gives
 * zeros, and no row of the table is read for it.  table: [n_rows][width], rows table_stride elements
 * apart (>= width); out: [n_tokens][width], rows out_stride apart, of the same type; tokens int32 or,
 * with tokens64, int64.  width <= 2^20, n_tokens < 2^31. */
int fpsched_op_embedding(int device_id, int type, const void *table, int64_t table_stride, int64_t n_rows,
                         int64_t width, const void *tokens, int tokens64, int64_t n_tokens, float scale,
                         void *out, int64_t out_stride, void *hip_stream);

/* The gradient of the table: out[v][:] = scale * sum of grad[t][:] over the t with tokens[t] == v, in
 * ascending t within blocks of 16 sorted occurrences and then over the blocks, in an order that the
 * tokens alone decide.  All n_rows rows are
 * written, with zeros where no token is; with accumulate (out_type FPSCHED_F32 only) the sums are added
 * to what out holds, and rows without a token are left as they are.  grad: [n_tokens][width] of `type`,
 * rows grad_stride apart; out: [n_rows][width] of `type` or FPSCHED_F32, rows out_stride apart.
 * width <= 2^20, n_tokens < 2^30, n_rows < 2^31. */
size_t fpsched_op_embedding_grad_workspace_bytes(int64_t n_rows, int64_t width, int64_t n_tokens);
int fpsched_op_embedding_grad(int device_id, int type, const void *grad, int64_t grad_stride, int64_t n_rows,
                              int64_t width, const void *tokens, int tokens64, int64_t n_tokens, float scale,
                              int out_type, void *out, int64_t out_stride, int accumulate,
                              void *d_workspace, size_t workspace_bytes, void *hip_stream);

/* ---- gated linear recurrence --------------------------------------------------------------------
 * Per sequence and channel, with a = sigmoid(gate):  h[t] = a[t] h[t-1] + (1 - a[t]) value[t], from
 * h[-1] = state (zero if NULL).  out[t] = h[t]; final_state = h at the sequence's end (float; may be
 * the same memory as state).  lengths (int32 [n_batch], NULL: all n_steps; clamped to 0 .. n_steps):
 * what is behind a sequence's end does not count, out is zero and the state stands still.  gate, value, out:
 * [n_batch][n_steps][width] of `type`, channels adjacent, steps and sequences `strides` elements apart
 * (HOST: batch and step stride of gate, of value, of out; <= 2^31, and of an output no two elements in one place); state, final_state: float [n_batch][width].
 * kept (NULL, or float [n_batch][ceil(n_steps / FPSCHED_RECURRENCE_BLOCK)][width]): the state in front
 * of every block of steps, from which the backward pass starts.  One step (n_steps = 1) is the form for
 * serving.  n_batch < 2^16, n_steps < 2^31, width <= 2^24. */
#define FPSCHED_RECURRENCE_BLOCK 64
size_t fpsched_op_recurrence_workspace_bytes(int64_t n_batch, int64_t n_steps, int64_t width);
int fpsched_op_recurrence(int device_id, int type, int64_t n_batch, int64_t n_steps, int64_t width,
                          const void *gate, const void *value, const int64_t *strides /* HOST [6] */,
                          const float *state, const int32_t *lengths, void *out, float *final_state,
                          float *kept, void *d_workspace, size_t workspace_bytes, void *hip_stream);

/* Its backward pass: with d[t] = grad[t] + a[t+1] d[t+1] (behind the last step grad_state, or zero if
 * NULL):  d_value[t] = (1 - a[t]) d[t],  d_gate[t] = d[t] (h[t-1] - value[t]) a[t] (1 - a[t]),
 * d_state = a[0] d[0] (float [n_batch][width], NULL: not wanted).  Behind a sequence's end the gradients
 * are zero.  kept: what the forward pass wrote.  strides: of grad, gate, value, d_gate, d_value. */
int fpsched_op_recurrence_grad(int device_id, int type, int64_t n_batch, int64_t n_steps, int64_t width,
                               const void *grad, const void *gate, const void *value,
                               const int64_t *strides /* HOST [10] */, const float *kept,
                               const float *grad_state, const int32_t *lengths, void *d_gate, void *d_value,
                               float *d_state, void *d_workspace, size_t workspace_bytes, void *hip_stream);

/* ---- gated feed-forward block -------------------------------------------------------------------
 * [g u] = x w_in^T,  hidden = act(g) u,  out = hidden w_out^T.  x, out: [n_tokens][width], rows x_stride
 * and out_stride apart; w_in: [2 hidden_width][width], the gate's rows first; w_out: [width][hidden_width];
 * hidden: [n_tokens][hidden_width], free again when the call's work is done; kept: NULL, or
 * FPSCHED_FFN_KEPT_BYTES of g and u in 24 bits for the backward pass.  Types FPSCHED_BF16 and FPSCHED_F16, the
 * same for all; weights and hidden contiguous.  width, hidden_width and the strides are multiples of 8,
 * the tensors 16-byte aligned (FPSCHED_EINVAL): rows are moved 16 bytes at a time; width and strides <= 2^21,
 * hidden_width <= 2^20, n_tokens < 2^31.  act is computed in 32
 * bits from unrounded g and u; hidden is rounded to `type`, as the matrix cores take it, for the second product, which is as much
 * of an error again as rounding out is (as are d_pre and hidden for the gradients).  FPSCHED_EUNSUPPORTED where a product has 2^23
 * tiles of 128 x 128 or more. */
enum { FPSCHED_SILU = 0, FPSCHED_GELU = 1 /* with tanh */, FPSCHED_RELU = 2 };
#define FPSCHED_FFN_KEPT_BYTES(n_tokens, hidden_width) ((size_t)6 * (n_tokens) * (hidden_width))
size_t fpsched_op_ffn_workspace_bytes(int64_t n_tokens, int64_t width, int64_t hidden_width);
int fpsched_op_ffn(int device_id, int type, int act, int64_t n_tokens, int64_t width, int64_t hidden_width,
                   const void *x, int64_t x_stride, const void *w_in, const void *w_out, void *kept,
                   void *hidden, void *out, int64_t out_stride, void *d_workspace, size_t workspace_bytes,
                   void *hip_stream);

/* The B item: d_hidden = grad w_out, d_pre = [d_hidden u act'(g), d_hidden act(g)] (rounded to `type`),
 * d_x = d_pre w_in.  kept: what the F item wrote; on return it holds d_pre, [n_tokens][2 hidden_width] of
 * `type`, and behind it hidden again, [n_tokens][hidden_width], for the W item.  So it serves one B item. */
int fpsched_op_ffn_input_grad(int device_id, int type, int act, int64_t n_tokens, int64_t width,
                              int64_t hidden_width, const void *grad, int64_t grad_stride, const void *w_in,
                              const void *w_out, void *kept, void *d_x, int64_t d_x_stride,
                              void *d_workspace, size_t workspace_bytes, void *hip_stream);

/* The W item: d_w_in = d_pre^T x, d_w_out = grad^T hidden, of `type` or FPSCHED_F32; with accumulate
 * (FPSCHED_F32 only) added to what is there.  kept: as the B item left it. */
int fpsched_op_ffn_weight_grad(int device_id, int type, int64_t n_tokens, int64_t width, int64_t hidden_width,
                               const void *x, int64_t x_stride, const void *grad, int64_t grad_stride,
                               const void *kept, int out_type, void *d_w_in, void *d_w_out, int accumulate,
                               void *d_workspace, size_t workspace_bytes, void *hip_stream);

/* ---- log probabilities of given tokens ------------------------------------------------------------
 * Per row of logits ([n_rows][vocab], rows logits_stride apart), with p = softmax:
 *   logprob = log p[token], entropy = -sum p log p, and the n_alternatives (0 .. 32) largest logits by
 *   (logit descending, id ascending): ids int32 [n_rows][n_alternatives] and their log probabilities.
 * lse: float [n_rows][2], the logarithm of the sum of exponentials in two parts, the largest logit and the
 * rest, for the backward pass.  A logit of minus infinity is masked: probability 0, and no alternative (id
 * -1, log probability minus infinity).  A row with nothing else: logprob minus infinity, entropy 0,
 * lse (0, minus infinity).  A token outside 0 .. vocab - 1 (-1 for padding): logprob 0.  A row that holds
 * NaN or plus infinity, padding or not: NaN throughout (of lse, the rest), ids -1.  vocab >= 1, n_rows < 2^31, vocab < 2^31. */
size_t fpsched_op_logprobs_workspace_bytes(int64_t n_rows, int64_t vocab, int n_alternatives);
int fpsched_op_logprobs(int device_id, int type, int64_t n_rows, int64_t vocab, const void *logits,
                        int64_t logits_stride, const void *tokens, int tokens64, int n_alternatives,
                        float *logprob, float *entropy, float *lse, int32_t *ids, float *alternatives,
                        void *d_workspace, size_t workspace_bytes, void *hip_stream);

/* The gradient of the logits for the gradients of logprob and of entropy (either may be NULL: zero):
 *   out[i] = grad_logprob ([i = token] - p[i]) - grad_entropy p[i] (log p[i] + entropy).
 * A row without a valid token takes no grad_logprob; a row with every logit masked gets zeros.  A p below
 * 2^-126 counts as 0.  out has the logits' type and may be the same memory (with the same stride). */
int fpsched_op_logprobs_grad(int device_id, int type, int64_t n_rows, int64_t vocab, const void *logits,
                             int64_t logits_stride, const void *tokens, int tokens64, const float *lse,
                             const float *entropy, const float *grad_logprob, const float *grad_entropy,
                             void *out, int64_t out_stride, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* FPSCHED_OPS_H */
