// Internal declarations of the student's operators (include/pql_student.h): element types and argument blocks.
#pragma once

#include "pql_internal.h"
#include "pql_student.h"

namespace pql {

using bf16_t = __bf16;
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(bf16_t x) { return (float)x; }
template <typename E> __device__ __forceinline__ E from_float(float x) { return (E)x; }      // bf16: to nearest even

// Which rows a launch of the gradient by itself takes: all, or by whether their log-sum-exp is too large to take q from it.
enum PartRows : int { ROWS_ALL = 0, ROWS_NEAR = 1, ROWS_FAR = 2 };

struct DistillArgs {
    const void* z;
    int64_t rows, stride, grad_stride;
    int vocab, top, pieces, piece;      // pieces of `piece` logits a row
    float temp, inv_temp;
    const int* index; const float* value;
    const float* weight;                // per row, NULL: ones
    const float* lse;                   // backward only
    float *loss_out, *lse_out;
    void* grad;
    float* part;                        // [rows][pieces][2]: maximum (-inf: nothing finite) and sum of each piece
    float* part_z;                      // [rows][top]: logits of the listed answers
    int part_rows;                      // PartRows
};

struct TopArgs {
    const void* z;
    int64_t rows, stride;
    int vocab, top, pieces, piece;
    int* index_out; float* value_out;
    int* part_index; float* part_value; // [rows][pieces][top]
};

// f(row, column) for rows from .. to - 1 and the first n of COLS columns, by the 64 lanes of one wavefront.  Rows are counted as
// they are: rows times columns may pass 32 bits.
template <int COLS, typename F> __host__ __device__ inline void each_of_rows(int lane, int64_t from, int64_t to, int n, F&& f) {
    if (lane % COLS >= n) return;
    for (int64_t row = from + lane / COLS; row < to; row += 64 / COLS) f(row, lane % COLS);
}

struct DeltaSeq { void* p; int64_t b, t, h; };
struct DeltaArgs {
    int batch, steps, heads_k, heads_v, group, dim_k, dim_v;
    int chunks, dvp;                    // chunks of a full sequence; dim_v padded for the arrays below
    int bh0;                            // first (sequence, head) of this launch
    int narrow;                         // scans take 16 columns a workgroup
    int heads_wg;                       // value heads per workgroup of the gradient's parallel part
    float scale;
    DeltaSeq q, k, v, g, beta, out;
    const int* lengths;
    const float* state;
    float* state_out;
    // per (sequence, head, chunk), fp32: T and P in operand order, gates; K^T and, for narrow scans, K and Q per key head, of the tokens' type.  What only
    // the gradient reads may be NULL: T^T, P^T, Q^T, R [64][dvp], S [dim_k padded][dvp] (before the chunk)
    void *T, *P, *TT, *PT, *KT, *QT, *KO, *QO;
    float *G, *R, *S;
    // gradient: dX, dY [64][dvp], dS [dim_k padded][dvp] (after the chunk); dq, dk per value head where those are shared
    DeltaSeq out_grad, dq, dk, dv, dg, dbeta;
    const float* state_grad;
    float* dstate;
    float *dX, *dY, *dS, *part_q, *part_k;
};

}  // namespace pql
