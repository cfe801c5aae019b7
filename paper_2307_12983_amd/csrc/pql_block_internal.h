// Internal declarations of the operators around a student's memory (include/pql_block.h).
#pragma once

#include "pql_block.h"
#include "pql_student_internal.h"

namespace pql {

constexpr int ROW_ALIGN = 16;               // bytes of the widest load or store

inline int elem_size(int32_t dtype) { return dtype == PQL_F32 ? 4 : 2; }
inline size_t to256(size_t x) { return (x + 255) / 256 * 256; }
inline bool off_by(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) != 0; }
// Rows that all start on 16-byte boundaries.
inline bool rows_aligned(const pql_rows& r, int32_t dtype) {
    return !off_by(r.data, ROW_ALIGN) && r.stride * elem_size(dtype) % ROW_ALIGN == 0;
}
// Rows that may be written: each has a place of its own (one row needs none).
inline bool own_rows(const pql_rows& r, int64_t rows, int64_t cols) { return rows <= 1 || r.stride >= cols; }
inline bool read_rows(const pql_rows& r) { return r.stride >= 0; }

// Which rows count: row = sequence * steps + step.
struct Live {
    const int* lengths;
    unsigned steps;
    __device__ __forceinline__ bool operator()(unsigned row) const {
        if (!lengths) return true;
        const unsigned b = row / steps;
        return (int)(row - b * steps) < lengths[b];
    }
};

// ---- 16 bytes of elements as floats ----------------------------------------------------------------
template <typename E> constexpr int VEC_OF = ROW_ALIGN / (int)sizeof(E);
__device__ __forceinline__ void widen(uint4 g, float* x, float) {
    x[0] = __uint_as_float(g.x); x[1] = __uint_as_float(g.y); x[2] = __uint_as_float(g.z); x[3] = __uint_as_float(g.w);
}
__device__ __forceinline__ void widen(uint4 g, float* x, bf16_t) {
    const unsigned u[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(u[i] << 16); x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
}
__device__ __forceinline__ uint4 narrow(const float* x, float) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
}
typedef __bf16 block_bf16x2 __attribute__((ext_vector_type(2)));
typedef float block_floatx2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ unsigned narrow2(float a, float b) {      // to nearest even, both in one register
    return __builtin_bit_cast(unsigned, __builtin_convertvector((block_floatx2{a, b}), block_bf16x2));
}
__device__ __forceinline__ uint4 narrow(const float* x, bf16_t) {
    return make_uint4(narrow2(x[0], x[1]), narrow2(x[2], x[3]), narrow2(x[4], x[5]), narrow2(x[6], x[7]));
}

// ---- activations -----------------------------------------------------------------------------------
// exp(x): 2^t by the one instruction, t = x log2 e rounded, times what the rounding has left out, to first order: below 3 u
// everywhere but for results that are no normal numbers.  Arguments are brought to where t is finite; NaN stays.
__device__ __forceinline__ float exp_near(float x) {
    x = x > 128.f ? 128.f : x < -128.f ? -128.f : x;
    const float t = x * 1.44269504f, r = fmaf(x, 1.44269504f, -t) + x * 1.92596299e-8f;
    return __builtin_amdgcn_exp2f(t) * fmaf(r, 0.693147181f, 1.f);
}
// s = 1 / (1 + exp(-x)) and 1 - s, neither from the other: both keep all their bits where they are small.
struct Sigmoid { float s, rest; };
__device__ __forceinline__ Sigmoid sigmoid(float x) {
    const float e = exp_near(-fabsf(x)), large = __builtin_amdgcn_rcpf(1.f + e), small = e * large;
    return x < 0.f ? Sigmoid{small, large} : Sigmoid{large, small};
}
// Half of erfc(-x / sqrt 2), the normal distribution's share below x.  fp32: by the library's erfc.  bf16: exp(-z^2) times a polynomial in
// t = 1 / (1 + 0.33 z), z = |x| / sqrt 2, fitted to exp(z^2) erfc(z) / 2 on [0, 10] for the least largest relative error (9.4e-8, 4.5e-7 in
// fp32 arithmetic), so that small results keep their bits.  A quarter of the time: a step of 16384 rows took 131 us for its projections with
// erfc.
__device__ __forceinline__ float share_below(float x, float) { return 0.5f * erfcf(-0.70710678f * x); }
__device__ __forceinline__ float share_below(float x, bf16_t) {
    const float t = __builtin_amdgcn_rcpf(fmaf(0.233345238f, fabsf(x), 1.f));
    const float half[8] = {0.093178895f, 0.091478075f, 0.10061129f, 0.023612525f, 0.204245715f, -0.17557006f, 0.23011568f, -0.06767213f};
    float p = half[7];
#pragma unroll
    for (int i = 6; i >= 0; --i) p = fmaf(t, p, half[i]);
    const float tail = t * p * __builtin_amdgcn_exp2f(-0.72134752f * x * x);
    return x > 0.f ? 1.f - tail : tail;
}
// f(x) and f'(x).  Factors that vanish do so before they meet a large x, so that finite x give finite results.  E: the type of what
// is worked out from them.
struct Act { float f, d; };
template <int ACT, typename E> __device__ __forceinline__ Act activate(float x) {
    if constexpr (ACT == PQL_ACT_SIGMOID) {
        const Sigmoid g = sigmoid(x);
        return {g.s, g.s * g.rest};
    } else if constexpr (ACT == PQL_ACT_SILU) {
        const Sigmoid g = sigmoid(x);
        return {x * g.s, g.s * (1.f + x * g.rest)};
    } else if constexpr (ACT == PQL_ACT_GELU) {
        const float h = share_below(x, E{});
        return {x * h, h + x * (0.39894228f * __builtin_amdgcn_exp2f(-0.72134752f * x * x))};
    } else if constexpr (ACT == PQL_ACT_RELU) {
        return {x > 0.f ? x : (x != x ? x : 0.f), x > 0.f ? 1.f : 0.f};
    } else {
        return {x, 1.f};
    }
}
// The same for N values at a time, by the activation's number.
template <typename E, int N> __device__ __forceinline__ void activate_all(int act, const float (&x)[N], float (&f)[N], float (&d)[N]) {
#define PQL_ACTIVATE(A) case A: _Pragma("unroll") for (int i = 0; i < N; ++i) { const Act y = activate<A, E>(x[i]); f[i] = y.f; d[i] = y.d; } break;
    switch (act) {
        PQL_ACTIVATE(PQL_ACT_SIGMOID)
        PQL_ACTIVATE(PQL_ACT_SILU)
        PQL_ACTIVATE(PQL_ACT_GELU)
        PQL_ACTIVATE(PQL_ACT_RELU)
        PQL_ACTIVATE(PQL_ACT_NONE)
    }
#undef PQL_ACTIVATE
}

}  // namespace pql
