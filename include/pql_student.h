/*
 * libpql, operators of a student policy: what a policy needs that sees less than the PQL policy it learns
 * from.  It carries a memory along each episode (the gated delta rule: stepped one token at a time by the
 * Actor for every environment, trained over windows or long sequences by the learner) and is trained on its
 * teacher's largest logits (selection, loss, gradient).
 *
 * The conventions of pql.h hold (return values, caller-owned memory, streams, threads, error text of the
 * context); a context created for the student's calls alone may have any valid configuration, of which these
 * calls read nothing.  Differences:
 *   Types       Token tensors and logits are fp32 or bfloat16 (PQL_F32 / PQL_BF16), everything else is what
 *               its parameter says.  All sums, states, decays and softmax statistics are held in fp32 or more.
 *   Strides     Token tensors are described by pql_seq: element (b, t, h, d) lies at
 *               data[b * stride_b + t * stride_t + h * stride_h + d], strides counted in elements, the last
 *               dimension contiguous.  Packed projections and transposed layouts therefore need no copy.
 *               data must be aligned to its element; rows that all start on 16-byte boundaries load faster.
 *               Inputs may repeat elements (a stride of 0); each repetition has its own element in the gradient.
 *   Graphs      Every call only enqueues kernels and may be captured.
 *   Aliasing    Outputs must not overlap inputs except where a call says so.
 */
#ifndef PQL_STUDENT_H
#define PQL_STUDENT_H

#include "pql.h"

#ifdef __cplusplus
extern "C" {
#endif

#define PQL_F32  0
#define PQL_BF16 1

/* ---- the gated delta rule ----------------------------------------------------------------- */

/* [device] token tensor, see "Strides". */
typedef struct { void* data; int64_t stride_b, stride_t, stride_h; } pql_seq;

#define PQL_DELTA_MAX_DIM_K 128
#define PQL_DELTA_MAX_DIM_V 256

/* batch sequences of at most `steps` tokens; heads_v value heads, of which heads_v / heads_k consecutive ones
 * share one query / key head (heads_v a multiple of heads_k); dim_k 1..PQL_DELTA_MAX_DIM_K, dim_v
 * 1..PQL_DELTA_MAX_DIM_V; dtype of q, k, v, the output and their gradients; scale multiplies the output. */
typedef struct {
    int32_t batch, steps, heads_k, heads_v, dim_k, dim_v, dtype;
    float   scale;
} pql_delta_shape;

/* q, k: heads_k heads of dim_k; v: heads_v heads of dim_v; log_decay, beta: fp32, heads_v heads of ONE element
 * (stride_h = 1 when dense); lengths[batch] (int32, or NULL: all `steps`): tokens of each sequence that count,
 * clamped to [0, steps]; what lies behind them is not read; state: fp32 [batch][heads_v][dim_k][dim_v]
 * contiguous, 16-byte aligned, or NULL (zeros).
 * log_decay <= 0; -inf, and any other value whose exponential is 0 in fp32 (below about -104, the type's lowest among
 * them), forgets the whole state before the token (the first token of an episode).  Nothing is normalised here: with
 * keys of unit length and beta in [0, 2] the state stays bounded.
 * Values that are not finite reach what the recurrence takes them to: later tokens of their own episode, nothing
 * before them and nothing from the next token that forgets the state on, in either form.  Gradients of other episodes
 * are what they would be without them; within the episode they need not be finite.  Sequences with such values are worked
 * through token by token in every form, which takes longer (about 1.5 us a token). */
typedef struct {
    pql_seq q, k, v, log_decay, beta;
    const int32_t* lengths;
    const float* state;
} pql_delta_input;

/* Gradients with the layouts of the tensors they belong to (dtype tokens, fp32 log_decay, beta and state);
 * all but state required, state may be NULL.  Elements behind a sequence's length are written as zeros. */
typedef struct {
    pql_seq q, k, v, log_decay, beta;
    float* state;
} pql_delta_grad;

/* One or a few tokens in the recurrent form (an Actor step: steps = 1):
 *     S~ = exp(log_decay_t) S_{t-1},  u_t = beta_t (v_t - S~^T k_t),  S_t = S~ + k_t u_t^T,
 *     out_t = scale S_t^T q_t
 * with S_0 = input.state; the last state of each sequence goes to state_out (may be input.state itself).
 * Sequences of length 0 keep their state; outputs behind a length are zeros.  Time grows with steps:
 * pql_delta_forward is the faster call from about 12 tokens on (1024 or 16384 states of 64 x 64, fp32).
 * Errors: PQL_ERR_NULL, PQL_ERR_INVALID_ARG, PQL_ERR_ALIGNMENT. */
int32_t pql_delta_step(pql_ctx* ctx, const pql_delta_shape* shape, const pql_delta_input* input,
                       float* state_out, pql_seq out, void* stream);

/* The same results over whole sequences, by chunks of tokens as matrix products.  state_out may be NULL or
 * input.state itself.  saved: NULL, or [device] pql_delta_saved_bytes(shape) bytes that pql_delta_backward
 * reads; workspace: [device] pql_delta_workspace_bytes(shape, 0) bytes; both 256-byte aligned. */
int64_t pql_delta_saved_bytes(const pql_delta_shape* shape);
int64_t pql_delta_workspace_bytes(const pql_delta_shape* shape, int32_t backward);
int32_t pql_delta_forward(pql_ctx* ctx, const pql_delta_shape* shape, const pql_delta_input* input, pql_seq out,
                          float* state_out, void* saved, void* workspace, void* stream);

/* Gradient of a loss whose gradients with respect to the outputs are out_grad (dtype) and, for the last
 * states, state_out_grad (fp32, laid out as the state; NULL: zeros).  input and saved: as given to and left by
 * pql_delta_forward of the same shape; input.state must still hold what the call read (do not let state_out
 * overwrite it).  The gradient of a log_decay that forgets the state is 0.  Key heads shared by several value
 * heads receive the sum over them, always added in the same order.  workspace: pql_delta_workspace_bytes(shape, 1)
 * bytes. */
int32_t pql_delta_backward(pql_ctx* ctx, const pql_delta_shape* shape, const pql_delta_input* input, const void* saved,
                           pql_seq out_grad, const float* state_out_grad, const pql_delta_grad* grads,
                           void* workspace, void* stream);

/* ---- a teacher's largest logits, and distillation from them -------------------------------- */

#define PQL_MAX_TOP 256

/* [device] rows of `vocab` logits, row n at data + n * stride elements (stride >= vocab), dtype as above. */
typedef struct { void* data; int64_t rows, stride; int32_t vocab, dtype; } pql_logits;

/* [device] lists of `top` entries a row, dense: index[rows][top], value[rows][top] (the teacher's logits; any
 * constant may be added to a row), top in 1..min(PQL_MAX_TOP, vocab).  An index outside [0, vocab) or a value of
 * -inf is no entry; an index that occurs twice counts with both values. */
typedef struct { const int32_t* index; const float* value; int32_t top; } pql_teacher;

/* The `top` (1..min(PQL_MAX_TOP, vocab)) largest logits of every row in descending order, equal ones by
 * ascending index: index_out[rows][top], value_out[rows][top].  -inf (a masked answer) and NaN are never
 * selected: places they would take get index -1 and value -inf.  workspace: [device]
 * pql_top_logits_workspace_bytes bytes, 256-byte aligned (may be NULL when that is 0). */
int64_t pql_top_logits_workspace_bytes(const pql_logits* logits, int32_t top);
int32_t pql_top_logits(pql_ctx* ctx, pql_logits logits, int32_t top, int32_t* index_out, float* value_out,
                       void* workspace, void* stream);

/* With q = softmax(z_n / t) over the row's logits and p = softmax(value / t) over its valid entries,
 *     loss_out[n] = w_n t^2 sum_k p_k (log p_k - log q_{index_k}),    lse_out[n] = log sum_j exp(z_nj / t),
 * t = temperature > 0, w = row_weight ([device] float[rows], NULL: ones).  With grad.data set (same rows,
 * vocab and dtype, a stride of its own; may be the logits themselves), the gradient of sum_n loss_out[n],
 *     grad_nj = w_n t (q_j - sum_{k: index_k = j} p_k),
 * is written in the same pass.  Nothing is used of rows with w_n = 0 or without a valid entry,
 * whatever they hold: loss, lse and gradient 0.  A listed answer that the student has at -inf gives loss +inf; a row of nothing but -inf has
 * lse -inf, q = 0.  workspace as above, pql_distill_workspace_bytes. */
int64_t pql_distill_workspace_bytes(const pql_logits* logits);
int32_t pql_distill_loss(pql_ctx* ctx, pql_logits logits, pql_teacher teacher, float temperature,
                         const float* row_weight, float* loss_out, float* lse_out, pql_logits grad, void* workspace,
                         void* stream);

/* The gradient alone, for a loss sum_n loss_grad[n] L_n with L_n the loss above at w_n = 1, from the lse_out of
 * that call: grad_nj = loss_grad[n] t (q_j - ...).  Nothing is used of rows with loss_grad[n] = 0 or without a
 * valid entry, which get zeros; rows of weight 0 in that call have no log-sum-exp, and must have loss_grad[n] = 0
 * here.  The rounding of lse_out costs q 2e-7 |lse|; rows with |lse| > 32 are therefore read once more for the
 * maximum and sum of their own.  grad may be the logits themselves. */
int32_t pql_distill_backward(pql_ctx* ctx, pql_logits logits, pql_teacher teacher, float temperature, const float* lse,
                             const float* loss_grad, pql_logits grad, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* PQL_STUDENT_H */
