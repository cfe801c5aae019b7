/*
 * libpql, operators around a student's memory (pql_student.h): the lookup of its tokens' embeddings, the norms
 * before and after a block with the block's gate and residual sum, and the gated feed-forward block; each with its
 * gradient.
 *
 * The conventions of pql.h and pql_student.h hold (return values, caller-owned memory, streams, threads, graphs,
 * error text of the context; PQL_F32 and PQL_BF16; sums, statistics and products held in fp32 or more).  Differences:
 *   Rows        Token tensors are batch * steps rows of contiguous elements, described by pql_rows: row n (= sequence *
 *               steps + step) starts at data + n * stride elements, stride >= its columns.  data must be aligned to its
 *               element; rows that all start on 16-byte boundaries load faster.  Rows may repeat (a stride of 0) where
 *               they are read; gradients and outputs have rows of their own.
 *   Lengths     lengths[batch] ([device] int32, or NULL: all `steps`): tokens of each sequence that count, clamped to
 *               [0, steps].  What lies behind them is not read, outputs and gradients there are written as zeros, and
 *               it has no part in the gradients of weights.
 *   Matrices    Weights are matrices of rows [out][in] (y_o = sum_i W_oi x_i) of the tokens' type, with a stride of their
 *               own; their gradients have that form and type, and are written, not added to.
 *   Order       Every sum is taken in one order: equal calls give equal bits.
 *   Aliasing    Outputs must not overlap inputs or each other except where a call says so.
 */
#ifndef PQL_BLOCK_H
#define PQL_BLOCK_H

#include "pql_student.h"

#ifdef __cplusplus
extern "C" {
#endif

/* [device] rows of a matrix, see "Rows". */
typedef struct { void* data; int64_t stride; } pql_rows;

/* ---- embeddings ------------------------------------------------------------------------------- */

/* batch * steps rows of `per_row` tokens each (at least 1; a token for every action dimension, say), whose embeddings
 * are added; vocab and dim at least 1; dtype of the table, the output and their gradients.  batch * steps * per_row
 * must stay below 2^31. */
typedef struct {
    int32_t batch, steps, per_row, vocab, dim, dtype;
    float   scale;
} pql_embed_shape;

/* out_n = scale * sum_j table[tokens[n][j]].  tokens: [device] int32 [batch * steps][per_row], dense; a token outside
 * [0, vocab) adds nothing.  table: vocab rows of dim.
 * Errors: PQL_ERR_NULL, PQL_ERR_INVALID_ARG, PQL_ERR_ALIGNMENT (of these and all calls below). */
int32_t pql_embed_forward(pql_ctx* ctx, const pql_embed_shape* shape, const int32_t* tokens, const int32_t* lengths,
                          const pql_rows* table, const pql_rows* out, void* stream);

/* table_grad_v = scale * sum over (n, j) with tokens[n][j] = v of out_grad_n, in ascending order of (n, j); every row
 * of table_grad is written.  workspace: [device] pql_embed_workspace_bytes(shape) bytes, 256-byte aligned. */
int64_t pql_embed_workspace_bytes(const pql_embed_shape* shape);
int32_t pql_embed_backward(pql_ctx* ctx, const pql_embed_shape* shape, const int32_t* tokens, const int32_t* lengths,
                           const pql_rows* out_grad, const pql_rows* table_grad, void* workspace, void* stream);

/* ---- norms, gate and residual sum around a block ------------------------------------------------ */

#define PQL_ACT_NONE    0              /* x (a gated feed-forward block without an activation is bilinear) */
#define PQL_ACT_SIGMOID 1              /* 1 / (1 + exp(-x)) */
#define PQL_ACT_SILU    2              /* x / (1 + exp(-x)) */
#define PQL_ACT_GELU    3              /* x (1 + erf(x / sqrt 2)) / 2 */
#define PQL_ACT_RELU    4              /* max(x, 0), derivative 0 at 0 */

#define PQL_RESIDUAL_MAX_DIM    8192
#define PQL_RESIDUAL_MAX_GROUPS 256

/* Rows of dim elements in `groups` equal parts (the heads of a memory; groups divides dim).  Where there are several, each
 * counts as a power of two of elements, at least 8, and together they must not exceed PQL_RESIDUAL_MAX_DIM.  gate_cols: columns of the
 * gate: 0 (no gate), groups (one value for each part) or dim; gate_act: PQL_ACT_*.  eps_post, eps_pre: 0 for no norm
 * in that place, or what is added to the mean square. */
typedef struct {
    int32_t batch, steps, dim, groups, dtype, gate_cols, gate_act;
    float   eps_post, eps_pre, scale_x, scale_y;
} pql_residual_shape;

/* x: the residual stream (data NULL: zeros); y: the block's output (data NULL: zeros; then no gate); gate;
 * post, pre: [device] fp32 [dim] weights after and before a block, or NULL: ones. */
typedef struct {
    pql_rows x, y, gate;
    const float *post, *pre;
    const int32_t* lengths;
} pql_residual_input;

/* Gradients with the layouts of what they belong to; any may be NULL (data or pointer) and is then not computed. */
typedef struct {
    pql_rows x, y, gate;
    float *post, *pre;
} pql_residual_grad;

/* With N(z) = z / sqrt(mean(z^2) + eps), the mean taken over each part of the row for y and over the row for sum (in fp32: of
 * values whose squares sum beyond its range, 1e19 and more, N is 0),
 *     sum_n = scale_x x_n + scale_y act(gate_n) post N(y_n),        next_n = pre N(sum_n)
 * where what is left out (a norm of eps 0, a gate, a weight) is the factor 1 or the identity.  sum may be x or y itself,
 * next may be y; either may have data NULL, not both.  next follows from the sum before that is rounded to dtype. */
int32_t pql_residual_forward(pql_ctx* ctx, const pql_residual_shape* shape, const pql_residual_input* input,
                             const pql_rows* sum, const pql_rows* next, void* stream);

/* Gradient of a loss whose gradients with respect to the outputs are sum_grad and next_grad (data NULL: zeros, not
 * both).  input: as given to pql_residual_forward; it must still hold what that call read.  grads->x may be sum_grad,
 * grads->y next_grad.  workspace: [device] pql_residual_workspace_bytes(shape) bytes, 256-byte aligned, or NULL where
 * neither post nor pre has a gradient. */
int64_t pql_residual_workspace_bytes(const pql_residual_shape* shape);
int32_t pql_residual_backward(pql_ctx* ctx, const pql_residual_shape* shape, const pql_residual_input* input,
                              const pql_rows* sum_grad, const pql_rows* next_grad, const pql_residual_grad* grads,
                              void* workspace, void* stream);

/* ---- the gated feed-forward block ---------------------------------------------------------------- */

#define PQL_FFN_MAX_DIM 65536

/* calls to ask a workspace's size for */
#define PQL_FFN_FORWARD        0
#define PQL_FFN_BACKWARD       1       /* with saved */
#define PQL_FFN_BACKWARD_ALONE 2       /* without */

/* batch * steps rows (below 2^30) of dim elements, `hidden` elements between the projections (both 1..PQL_FFN_MAX_DIM);
 * dtype of tokens, weights and their gradients; act: PQL_ACT_*. */
typedef struct { int32_t batch, steps, dim, hidden, dtype, act; } pql_ffn_shape;

/* x: rows of dim; gate, up: hidden rows of dim; down: dim rows of hidden. */
typedef struct {
    pql_rows x, gate, up, down;
    const int32_t* lengths;
} pql_ffn_input;

/* Gradients; any may have data NULL and is then not computed. */
typedef struct { pql_rows x, gate, up, down; } pql_ffn_grad;

/*     a = gate x_n,  b = up x_n,  m = act(a) b (element by element),  out_n = down m.
 * saved: NULL, or [device] pql_ffn_saved_bytes(shape) bytes that keep a and b (fp32) and m for pql_ffn_backward.
 * workspace: [device] pql_ffn_workspace_bytes(shape, PQL_FFN_FORWARD) bytes; both 256-byte aligned.  bf16: m is rounded to
 * bf16 once as an operand of the second product, or, in a call of few rows without saved, kept in 16 bits; a and b are in
 * fp32.  fp32: products of 24-bit operands, sums in fp32.  Infinite values
 * and sums that overflow give what fp32 arithmetic gives, in both types and in calls of any number of rows (values within a
 * hundredth of the largest number may become infinite). */
int64_t pql_ffn_saved_bytes(const pql_ffn_shape* shape);
int64_t pql_ffn_workspace_bytes(const pql_ffn_shape* shape, int32_t call);
int32_t pql_ffn_forward(pql_ctx* ctx, const pql_ffn_shape* shape, const pql_ffn_input* input, const pql_rows* out,
                        void* saved, void* workspace, void* stream);

/* Gradient of a loss whose gradient with respect to out is out_grad.  saved: as left by pql_ffn_forward of the same
 * shape and input (lengths among it), or NULL: a, b and m are worked out again.  bf16: m and the gradients of a and b are
 * rounded to bf16 once as operands of the products that follow.  workspace: pql_ffn_workspace_bytes(shape,
 * PQL_FFN_BACKWARD or, without saved, PQL_FFN_BACKWARD_ALONE) bytes. */
int32_t pql_ffn_backward(pql_ctx* ctx, const pql_ffn_shape* shape, const pql_ffn_input* input, const void* saved,
                         const pql_rows* out_grad, const pql_ffn_grad* grads, void* workspace, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* PQL_BLOCK_H */
