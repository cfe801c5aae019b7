// Internal declarations of the gated feed-forward block (include/pql_block.h): its argument blocks and the launches of
// its two families of kernels, products of row tiles (pql_ffn.hip) and of few rows (pql_ffn_rows.hip).
#pragma once

#include "pql_block_internal.h"

namespace pql {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

// Results of matrix instructions must not be read for some cycles; behind branches the compiler's own waits have been found to
// miss a short side, so they are waited for here before a branch can lie between.
__device__ __forceinline__ void settle_products() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 15\n\ts_nop 3");
    __builtin_amdgcn_sched_barrier(0);
}

// x = h + m + l, exactly from 2^-110 on (below, terms fall under the smallest normal number, 2^-126): the nearest bf16 (8 bits), the
// next 8 bits of the rest, and what is left.  Values that are not finite are their first term alone.
struct Terms { float t[3]; };
__device__ __forceinline__ Terms three_terms(float x) {
    Terms s;
    s.t[0] = (float)(bf16_t)x;
    float r = x - s.t[0];
    if (!(fabsf(s.t[0]) < __builtin_inff())) {                  // too large for a bf16, infinite or NaN
        s.t[0] = __uint_as_float(__float_as_uint(x) & 0xffff0000u);
        if (x != x) s.t[0] = x;
        r = fabsf(x) < __builtin_inff() ? x - s.t[0] : 0.f;
    }
    s.t[1] = __uint_as_float(__float_as_uint(r) & 0xffff0000u);
    s.t[2] = r - s.t[1];
    return s;
}

// Calls of at most so many rows take the kernels for few rows, which read the rows again for each 16 outputs; the tiles' kernels read
// them once, but split rows and 32-bit weights into terms and join sums.  By the elements of a projection; whole: the tiles' kernels can
// read 32-bit weights as they are.  us a call, rows / tiles.  1024 and 4096 (4 Mi), 64 rows: fp32 37 / 60, bf16 22 / 31.  1408 and 5632, 64
// rows: 95 / 78 and 50 / 37, 32 rows: 54 / 76 and 29 / 36.  2048 and 8192, 32 rows: 82 / 112 and 43 / 48; with planes of fp32 weights 64 rows 136 /
// 195.  4096 and 16384 (64 Mi): fp32 32 rows 311 / 332, bf16 16 rows 117 / 128, 24 rows 142 / 121.
constexpr int FFN_FEW_ROWS = 64;
inline int ffn_few_rows(int32_t dtype, int64_t elements, bool whole) {
    if (elements <= 4 << 20 || (dtype == PQL_F32 && !whole)) return FFN_FEW_ROWS;
    return dtype == PQL_F32 || elements <= 32 << 20 ? 32 : 16;
}

struct FfnRowsArgs {
    Live live;
    int rows, dim, hidden, act;
    const void *x, *gate, *up, *down;
    int64_t x_stride, gate_stride, up_stride, down_stride;
    void* m; int64_t m_stride, m_plane;         // [rows][m_stride] of the tokens' type; bf16: two planes of terms
    void* out; int64_t out_stride;
};
hipError_t ffn_rows_launch(const FfnRowsArgs& a, int32_t dtype, hipStream_t st);

}  // namespace pql
