// The gated delta rule (include/pql_student.h): a state S [dim_k][dim_v] per sequence and value head,
//     S~ = exp(g_t) S,  r_t = v_t - S~^T k_t,  S = S~ + k_t (beta_t r_t)^T,  o_t = scale S^T q_t.
//
// One token or a few: delta_step_kernel keeps the state in registers and reads and writes it once; bound by that.
// (All times below: fp32 "windows" = 512 sequences of up to 32 tokens, 4 heads of 64 x 64, forward and gradient; bf16
// "sequences" = 4 of 2048 tokens, 16 value heads of 128 x 128 on 8 key heads, forward and gradient; "long" = one of 16384, forward.)
//
// Sequences go by chunks of 32 or 64 tokens.  With S0 the state before the chunk, G_i the sums of g in it, gam_i = e^{G_i},
// Gam_ij = e^{G_i - G_j} (0 where a reset lies between: a g for which e^g is 0 in fp32), e_i = e^{G_last - G_i}, all tokens of a chunk follow from
//     N_ij = Gam_ij k_i.k_j (i > j),  T = (I + N diag(beta))^-1,  X = V - gam o (K S0),  R = T X,  Y = beta o R,
//     P_ij = Gam_ij q_i.k_j (i >= j),  O = scale (gam o (Q S0) + P Y),  S1 = e^{G_last} S0 + K^T (e o Y),
// R being the errors r_t.  delta_prepare_kernel finds T and P of all chunks at once; delta_scan_kernel goes through the
// chunks of one sequence, head and block of columns of the state (columns never mix).
// Gradient, with dO scaled: delta_back_scan_kernel goes through the chunks in reverse,
//     dY = P^T dO + e o (K dS1),  dX = T^T (beta o dY) = dV,  dS0 = e^{G_last} dS1 - K^T (gam o dX) + Q^T (gam o dO),
// and delta_back_kernel takes all chunks at once for the rest,
//     E = Gam o (dO Y^T) (i >= j),  F = -Gam o (dX R^T) (i > j),
//     dQ = gam o (dO S0^T) + E K,
//     dK = -gam o (dX S0^T) + (F diag(beta)) K + e o (Y dS1^T) + beta o (F^T K) + E^T Q,
//     dbeta_j = dY_j.R_j + k_j.(F^T K)_j,
//     dG_i = q_i.dQ_i + k_i.(first two terms of dK_i) - k_i.(last three),
//     dG_last += sum_j k_j.(e o (Y dS1^T))_j + e^{G_last} <dS1, S0>,  dg_t = sum of dG_i from t to its segment's end.
//
// Arithmetic: products on the matrix cores with 32-bit results.  fp32 tokens: v_mfma_f32_16x16x4_f32.  bf16 tokens:
// q, k and dO are exact operands; what has been computed (S, X, Y, T, P, ...) is split into three bf16 terms, which
// together hold the 24 bits of an fp32 value, so that rounding to bf16 happens at the outputs only and the fp32 outputs
// (states, gradients of gates) are as exact as with fp32 products.
#include "pql_student_internal.h"

namespace pql {
namespace {

constexpr int MAXC = 64;                    // most tokens per chunk (C below: 64 or 32)

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

// ---- operands of 16x16x32 products -----------------------------------------------------------
// Lane l holds row (A) or column (B) l % 16, elements 8 (l / 16) .. + 7 of the contraction; results: column l % 16,
// rows 4 (l / 16) .. + 3.
struct F1 { bf16x8 h; };                    // exact bf16
struct F3 { bf16x8 h, m, l; };              // an fp32 value as three bf16 terms
struct FF { float v[8]; };
__device__ __forceinline__ floatx4 mm(bf16x8 a, bf16x8 b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ void mma(floatx4& c, const F1& a, const F1& b) { c = mm(a.h, b.h, c); }
__device__ __forceinline__ void mma(floatx4& c, const F1& a, const F3& b) { c = mm(a.h, b.l, c); c = mm(a.h, b.m, c); c = mm(a.h, b.h, c); }
__device__ __forceinline__ void mma(floatx4& c, const F3& a, const F1& b) { c = mm(a.l, b.h, c); c = mm(a.m, b.h, c); c = mm(a.h, b.h, c); }
// terms below 2^-24 of the product are left out
__device__ __forceinline__ void mma(floatx4& c, const F3& a, const F3& b) {
    c = mm(a.l, b.h, c); c = mm(a.h, b.l, c); c = mm(a.m, b.m, c);
    c = mm(a.m, b.h, c); c = mm(a.h, b.m, c); c = mm(a.h, b.h, c);
}
__device__ __forceinline__ void mma(floatx4& c, const FF& a, const FF& b) {
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[j], b.v[j], c, 0, 0, 0);
}
// x = h + m + l exactly: the nearest bf16 (8 bits), the next 8 bits of the rest, and what is left.  Two values at a time,
// each term of both in one register.
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
struct Split2 { unsigned h, m, l; };
__device__ __forceinline__ Split2 split2(float x, float y) {
    Split2 s;
    s.h = __builtin_bit_cast(unsigned, __builtin_convertvector((floatx2{x, y}), bf16x2));
    const float rx = x - __uint_as_float(s.h << 16), ry = y - __uint_as_float(s.h & 0xffff0000u);
    const unsigned mx = __float_as_uint(rx), my = __float_as_uint(ry);
    s.m = __builtin_amdgcn_perm(my, mx, 0x07060302);
    const float lx = rx - __uint_as_float(mx & 0xffff0000u), ly = ry - __uint_as_float(my & 0xffff0000u);
    s.l = __builtin_amdgcn_perm(__float_as_uint(ly), __float_as_uint(lx), 0x07060302);
    return s;
}
typedef unsigned uintx2 __attribute__((ext_vector_type(2)));
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));
// A sum of products on a chain that others wait for: independent accumulators by the size of the terms, joined at the end.
struct Acc {
    floatx4 a[3] = {};
    __device__ __forceinline__ void add(const F1& x, const F3& y) { a[2] = mm(x.h, y.l, a[2]); a[1] = mm(x.h, y.m, a[1]); a[0] = mm(x.h, y.h, a[0]); }
    __device__ __forceinline__ void add(const F3& x, const F1& y) { a[2] = mm(x.l, y.h, a[2]); a[1] = mm(x.m, y.h, a[1]); a[0] = mm(x.h, y.h, a[0]); }
    __device__ __forceinline__ void add(const F3& x, const F3& y) {
        a[2] = mm(x.l, y.h, a[2]); a[1] = mm(x.m, y.h, a[1]); a[0] = mm(x.h, y.h, a[0]);
        a[2] = mm(x.h, y.l, a[2]); a[1] = mm(x.h, y.m, a[1]); a[2] = mm(x.m, y.m, a[2]);
    }
    __device__ __forceinline__ void add(const FF& x, const FF& y) {
#pragma unroll
        for (int j = 0; j < 8; ++j) a[j & 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(x.v[j], y.v[j], a[j & 1], 0, 0, 0);
    }
    __device__ __forceinline__ floatx4 sum() const { return a[2] + a[1] + a[0]; }
};

// Results of matrix instructions must not be read for some cycles.  The compiler sees to that, but not on every path where
// branches lie between (a short side of a branch is missed when a long one has been looked at first; a result was read too
// early that way): behind products in branches all results are waited for, and nothing is moved across.
__device__ __forceinline__ void settle() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 15\n\ts_nop 3");
    __builtin_amdgcn_sched_barrier(0);
}

struct ModeB {                              // bf16 tokens
    using E = bf16_t; using X = F1; using Y = F3;
    static constexpr int PLANES = 3, PAD = 8;
    static __device__ __forceinline__ Y computed(const float* x) {
        uintx4 h, m, l;
#pragma unroll
        for (int j = 0; j < 4; ++j) { const Split2 s = split2(x[2 * j], x[2 * j + 1]); h[j] = s.h; m[j] = s.m; l[j] = s.l; }
        return F3{__builtin_bit_cast(bf16x8, h), __builtin_bit_cast(bf16x8, m), __builtin_bit_cast(bf16x8, l)};
    }
    static __device__ __forceinline__ X exact(const float* x) {
        F1 f;
#pragma unroll
        for (int j = 0; j < 8; ++j) f.h[j] = (__bf16)x[j];
        return f;
    }
};
struct ModeF {                              // fp32 tokens
    using E = float; using X = FF; using Y = FF;
    static constexpr int PLANES = 1, PAD = 4;
    static __device__ __forceinline__ Y computed(const float* x) {
        FF f;
#pragma unroll
        for (int j = 0; j < 8; ++j) f.v[j] = x[j];
        return f;
    }
    static __device__ __forceinline__ X exact(const float* x) { return computed(x); }
};

// A matrix in LDS, [rows][cols], contraction along the columns, rows padded by 16 bytes.  Computed values take
// M::PLANES planes, exact ones a single one.
template <typename M, int ROWS, int COLS, bool EXACT> struct Tile {
    using E = typename M::E;
    static constexpr int LD = COLS + M::PAD, PLANES = EXACT ? 1 : M::PLANES;
    static constexpr int BYTES = ROWS * LD * PLANES * (int)sizeof(E);
    E* p;
    __device__ __forceinline__ explicit Tile(void* q) : p((E*)q) {}
    __device__ __forceinline__ void put4(int row, int k, floatx4 x) const {
        E* o = p + row * LD + k;
        if constexpr (sizeof(E) == 4) {
            *(floatx4*)o = x;
        } else if constexpr (EXACT) {
            bf16x4 h;
#pragma unroll
            for (int i = 0; i < 4; ++i) h[i] = (__bf16)x[i];
            *(bf16x4*)o = h;
        } else {
            const Split2 s = split2(x[0], x[1]), t = split2(x[2], x[3]);
            *(uintx2*)o = uintx2{s.h, t.h}; *(uintx2*)(o + ROWS * LD) = uintx2{s.m, t.m}; *(uintx2*)(o + 2 * ROWS * LD) = uintx2{s.l, t.l};
        }
    }
    __device__ __forceinline__ void put8(int row, int k, const float* x) const {
        E* o = p + row * LD + k;
        const auto f = M::computed(x);
        if constexpr (PLANES == 3) {
            *(bf16x8*)o = f.h; *(bf16x8*)(o + ROWS * LD) = f.m; *(bf16x8*)(o + 2 * ROWS * LD) = f.l;
        } else {
            *(floatx4*)o = floatx4{f.v[0], f.v[1], f.v[2], f.v[3]};
            *(floatx4*)(o + 4) = floatx4{f.v[4], f.v[5], f.v[6], f.v[7]};
        }
    }
    __device__ __forceinline__ void put1(int row, int k, float x) const {
        E* o = p + row * LD + k;
        if constexpr (PLANES == 3) {
            const Split2 s = split2(x, 0.f);
            *(unsigned short*)o = (unsigned short)s.h; *(unsigned short*)(o + ROWS * LD) = (unsigned short)s.m; *(unsigned short*)(o + 2 * ROWS * LD) = (unsigned short)s.l;
        } else {
            o[0] = (E)x;
        }
    }
    // the operands of N 16-row tiles (rows row + 16 n) over K steps of 32, all requested at once
    template <int K, int N, typename F> __device__ __forceinline__ void frags(int row, int k, F (&f)[K][N]) const {
#pragma unroll
        for (int d = 0; d < K; ++d)
#pragma unroll
            for (int n = 0; n < N; ++n) f[d][n] = frag(row + 16 * n, k + 32 * d);
    }
    __device__ __forceinline__ auto frag(int row, int k) const {
        const E* o = p + row * LD + k;
        if constexpr (sizeof(E) == 4) {
            FF f;
            const floatx4 a = *(const floatx4*)o, b = *(const floatx4*)(o + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) { f.v[i] = a[i]; f.v[4 + i] = b[i]; }
            return f;
        } else if constexpr (EXACT) {
            return F1{*(const bf16x8*)o};
        } else {
            return F3{*(const bf16x8*)o, *(const bf16x8*)(o + ROWS * LD), *(const bf16x8*)(o + 2 * ROWS * LD)};
        }
    }
};

// ---- tokens in memory -----------------------------------------------------------------------
// Eight consecutive elements d .. d + 7 of one token row; zeros from dim on and where the token does not count.
template <typename E, bool AL>
__device__ __forceinline__ void load8(const E* row, int d, int dim, bool ok, float* x) {
    if (AL) {                               // 16-byte aligned rows of a multiple of 16 bytes
        if constexpr (sizeof(E) == 4) {
            floatx4 a = {}, b = {};
            if (ok && d < dim) a = *(const floatx4*)(row + d);
            if (ok && d + 4 < dim) b = *(const floatx4*)(row + d + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) { x[i] = a[i]; x[4 + i] = b[i]; }
        } else {
            bf16x8 a = {};
            if (ok && d < dim) a = *(const bf16x8*)(row + d);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = (float)a[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = ok && d + i < dim ? to_float(row[d + i]) : 0.f;
    }
}
// Eight consecutive fp32 values of a padded array of the library's own.
__device__ __forceinline__ void load8(const float* p, float* x) {
    const floatx4 a = *(const floatx4*)p, b = *(const floatx4*)(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[i] = a[i]; x[4 + i] = b[i]; }
}
// The chunk's tokens transposed: tile[d][token], d < D.  Values that are not finite are left out: these are operands in which all
// tokens of a chunk meet, with a factor of 0 where they must not.  Such a token's own results still show it, through its row operands.
template <typename M, int C, int D, bool AL, typename T>
__device__ __forceinline__ void stage_transposed(const T& tile, const typename M::E* base, int64_t stride_t, int len, int dim, int d0 = 0) {
    for (int u = threadIdx.x; u < D / 8 * (C / 4); u += 4 * C) {
        const int t = u % (C / 4) * 4, d = u / (C / 4) * 8;
        float x[4][8];
#pragma unroll
        for (int i = 0; i < 4; ++i) load8<typename M::E, AL>(base + (t + i) * stride_t, d0 + d, dim, t + i < len, x[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            floatx4 y;
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = __builtin_isfinite(x[i][j]) ? x[i][j] : 0.f;
            tile.put4(d + j, t, y);
        }
    }
}

// ---- gates of a chunk -------------------------------------------------------------------------
struct Gates {
    double sum[MAXC];                       // G_i, counted from the last reset on; double, so that differences of long sums stay exact
    int part[MAXC];                         // resets up to and including the token
    float beta[MAXC], gam[MAXC], end[MAXC];
    float last;                             // e^{G_last}, 0 after a reset in the chunk
};
// By the first wavefront, from the token values that it has requested before; a barrier follows.  Every g for which e^g is 0 in
// fp32, as the recurrent form has it, is a reset, and sums begin anew behind it: kept in the sum, a g of -1e12 would cost all
// that follow the bits of their differences, and one that is not a number would reach beyond the reset.
struct GateValues {
    float g = 0.f, beta = 0.f;
    __device__ __forceinline__ void load(const float* g_, int64_t g_stride, const float* beta_, int64_t b_stride, int len) {
        const int i = threadIdx.x;
        if (i >= min(len, 64)) return;
        g = g_[i * g_stride];
        beta = beta_[i * b_stride];
    }
};
__device__ __forceinline__ void gates_of(Gates& s, const GateValues& v) {
    const int i = threadIdx.x;
    if (i >= 64) return;
    const bool reset = expf(v.g) == 0.f;
    const unsigned long long resets = __ballot(reset), before = resets & (~0ull >> (63 - i));
    const int start = before ? 63 - __clzll(before) : 0;        // the last reset's place
    double sum = reset ? 0.f : v.g;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) { const double o = __shfl_up(sum, d); if (i - d >= start) sum += o; }
    const int part = __popcll(before), all = __popcll(resets);
    const double total = __shfl(sum, 63);
    s.sum[i] = sum;
    s.part[i] = part;
    s.beta[i] = v.beta;
    s.gam[i] = part == 0 ? expf((float)sum) : 0.f;
    s.end[i] = part == all ? expf((float)(total - sum)) : 0.f;
    if (i == 63) s.last = all == 0 ? expf((float)total) : 0.f;
}
// f x, and 0 for f = 0 whatever x is: behind a reset nothing is left of a state that is not finite.
__device__ __forceinline__ float damp(float f, float x) { return f == 0.f ? 0.f : f * x; }
// 0 as long as all it is given is finite, and not a number from then on.
__device__ __forceinline__ float watch(float odd, floatx4 x) {
#pragma unroll
    for (int r = 0; r < 4; ++r) odd = fmaf(x[r], 0.f, odd);
    return odd;
}
__device__ __forceinline__ float decay(const Gates& s, int i, int j) {
    return s.part[i] == s.part[j] ? expf((float)(s.sum[i] - s.sum[j])) : 0.f;
}

struct Where {                              // one sequence and head
    int b, h, hk, len, bh;
};
__device__ __forceinline__ Where where_of(const DeltaArgs& a, int bh) {
    Where w;
    w.bh = bh + a.bh0; w.b = w.bh / a.heads_v; w.h = w.bh - w.b * a.heads_v; w.hk = w.h / a.group;
    w.len = a.lengths ? min(max(a.lengths[w.b], 0), a.steps) : a.steps;
    return w;
}
// Workgroup `id` of a scan over n (sequence, head) pairs with `blocks` column blocks each.  Workgroups go round the eight XCDs
// in turn; the blocks of one pair, which read the same q, k, T, P and K^T, are given to one XCD so that its L2 serves all but
// the first (1 x 16384 tokens, 16 heads of 128 x 128, bf16: 529 us, in the order of ids 580).
__device__ __forceinline__ void place_of(int id, int n, int blocks, int& bh, int& block) {
    const int whole = n & ~7;
    if (id < whole * blocks) {
        const int slot = id >> 3;
        bh = slot / blocks * 8 + (id & 7);
        block = slot % blocks;
    } else {
        bh = whole + (id - whole * blocks) / blocks;
        block = (id - whole * blocks) % blocks;
    }
}
template <typename E> __device__ __forceinline__ const E* at(const DeltaSeq& s, int b, int64_t t, int h) {
    return (const E*)s.p + b * s.b + t * s.t + h * s.h;
}
template <typename E> __device__ __forceinline__ E* at_out(const DeltaSeq& s, int b, int64_t t, int h) {
    return (E*)s.p + b * s.b + t * s.t + h * s.h;
}

// =============================================================================================
// One token or a few.  A workgroup holds up to 4 LX columns of one state in registers: lanes along the columns (four
// each), 256 / LX groups of rows.  With z = S~^T k and w = S~^T q found together, u = beta (v - z) and
// o = scale (w + (q.k) u) need one reduction per token instead of two.  One token of 16384 environments, 4 heads of 64 x 64,
// bf16: 361 us, 6.0 TB/s of states read and written to another buffer, in place 385 us (a large copy reaches 5.0 TB/s); fp32 393 and 398 us; of
// 64 environments, 2 heads of 32 x 32: 4 us, a launch.
// =============================================================================================
template <typename E, int LX, bool VEC>
__global__ __launch_bounds__(256) void delta_step_kernel(DeltaArgs a) {
    constexpr int RY = 256 / LX, NR = PQL_DELTA_MAX_DIM_K / RY;
    __shared__ float s_k[2][PQL_DELTA_MAX_DIM_K], s_q[2][PQL_DELTA_MAX_DIM_K];
    __shared__ float s_red[2][4][LX * 8];
    const Where w = where_of(a, blockIdx.x);
    const int t = threadIdx.x, lx = t % LX, ry = t / LX, c0 = blockIdx.y * LX * 4;
    const int dk = a.dim_k, dv = a.dim_v;
    const int64_t base = (int64_t)w.bh * dk * dv;
    float s[NR][4];
    auto col = [&](int j) { return c0 + (VEC ? lx * 4 + j : lx + LX * j); };
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        const int r = ry + RY * i;
#pragma unroll
        for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
        if (a.state && r < dk) {
            const float* p = a.state + base + (int64_t)r * dv;
            if (VEC) {
                if (col(0) < dv) {
                    const floatx4 x = *(const floatx4*)(p + col(0));
#pragma unroll
                    for (int j = 0; j < 4; ++j) s[i][j] = x[j];
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) if (col(j) < dv) s[i][j] = p[col(j)];
            }
        }
    }
    for (int n = 0; n < a.steps; ++n) {
        const int slot = n & 1;
        E* out = at_out<E>(a.out, w.b, n, w.h);
        if (n >= w.len) {
            if (ry == 0)
                for (int j = 0; j < 4; ++j) if (col(j) < dv) out[col(j)] = from_float<E>(0.f);
            continue;
        }
        if (t < PQL_DELTA_MAX_DIM_K) s_k[slot][t] = t < dk ? to_float(at<E>(a.k, w.b, n, w.hk)[t]) : 0.f;
        else s_q[slot][t - PQL_DELTA_MAX_DIM_K] = t - PQL_DELTA_MAX_DIM_K < dk ? to_float(at<E>(a.q, w.b, n, w.hk)[t - PQL_DELTA_MAX_DIM_K]) : 0.f;
        const float alpha = expf(*at<float>(a.g, w.b, n, w.h)), beta = *at<float>(a.beta, w.b, n, w.h);
        float v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = col(j) < dv ? to_float(at<E>(a.v, w.b, n, w.h)[col(j)]) : 0.f;
        __syncthreads();
        float z[8] = {}, qk = 0.f;
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const int r = ry + RY * i;
            const float k = s_k[slot][r], q = s_q[slot][r];
            qk += q * k;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[i][j] = damp(alpha, s[i][j]);
                z[j] += s[i][j] * k;
                z[4 + j] += s[i][j] * q;
            }
        }
        // the lanes of a wavefront that hold the same columns, then the four wavefronts
#pragma unroll
        for (int d = LX; d < 64; d *= 2) {
            qk += __shfl_xor(qk, d);
#pragma unroll
            for (int j = 0; j < 8; ++j) z[j] += __shfl_xor(z[j], d);
        }
        __shared__ float s_qk[2][4];
        if ((t & 63) < LX) {
#pragma unroll
            for (int j = 0; j < 8; ++j) s_red[slot][t >> 6][j * LX + lx] = z[j];
            if (lx == 0) s_qk[slot][t >> 6] = qk;
        }
        __syncthreads();
        qk = s_qk[slot][0] + s_qk[slot][1] + s_qk[slot][2] + s_qk[slot][3];
        float u[4], o[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float zz = 0.f, zq = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) { zz += s_red[slot][i][j * LX + lx]; zq += s_red[slot][i][(4 + j) * LX + lx]; }
            u[j] = beta * (v[j] - zz);
            o[j] = a.scale * (zq + qk * u[j]);
        }
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const float k = s_k[slot][ry + RY * i];
#pragma unroll
            for (int j = 0; j < 4; ++j) s[i][j] += k * u[j];
        }
        if (ry == 0) {
#pragma unroll
            for (int j = 0; j < 4; ++j) if (col(j) < dv) out[col(j)] = from_float<E>(o[j]);
        }
    }
    if (a.state_out == a.state && w.len == 0) return;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        const int r = ry + RY * i;
        if (r >= dk) continue;
        float* p = a.state_out + base + (int64_t)r * dv;
        if (VEC) {
            if (col(0) < dv) *(floatx4*)(p + col(0)) = floatx4{s[i][0], s[i][1], s[i][2], s[i][3]};
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) if (col(j) < dv) p[col(j)] = s[i][j];
        }
    }
}

// =============================================================================================
// Chunks: T and P of every chunk.
// =============================================================================================
// t = (I + m)^-1 of a strictly lower triangular m.  Blocks of 16: those on the diagonal by substitution (stable whatever the
// keys; a series of powers is not), one wavefront each; then T_ij = -T_ii sum_{j <= k < i} m_ik T_kj downwards, one block
// column per wavefront.  With the contraction index 4 (l / 16) + s in step s, a result is the next product's right operand
// as it lies in the registers, so a column needs nothing from LDS but m and the diagonal.  Blocks (0, 1) and (2, 3), which
// operands of 32 columns cover, are zeroed; others above the diagonal are not written.
template <int C> struct Matrix { static constexpr int LD = C + 4; float v[C][LD]; };
template <int C> __device__ __forceinline__ void invert(const Matrix<C>& m, Matrix<C>& t) {
    constexpr int NW = C / 16;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, c = l & 15, q = l >> 4;
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        float y = i == c ? 1.f : 0.f;
#pragma unroll
        for (int k = 0; k < i; k += 4) {
            const floatx4 r = *(const floatx4*)&m.v[16 * w + i][16 * w + k];
#pragma unroll
            for (int j = 0; j < 4; ++j) if (k + j < i) y -= r[j] * x[k + j];
        }
        x[i] = y;
    }
    floatx4 col[NW];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const float d = q == 0 ? x[r] : q == 1 ? x[4 + r] : q == 2 ? x[8 + r] : x[12 + r];
#pragma unroll
        for (int k = 0; k < NW; ++k) col[k][r] = d;        // only [w] is read
        t.v[16 * w + 4 * q + r][16 * w + c] = d;
        if (w & 1) t.v[16 * (w - 1) + 4 * q + r][16 * w + c] = 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int i = 1; i < NW; ++i) {
        if (i <= w) continue;
        floatx4 acc = {0.f, 0.f, 0.f, 0.f}, o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < i; ++k) {
            if (k < w) continue;
            const floatx4 r = *(const floatx4*)&m.v[16 * i + c][16 * k + 4 * q];
#pragma unroll
            for (int s = 0; s < 4; ++s) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(r[s], col[k][s], acc, 0, 0, 0);
        }
        settle();
        const floatx4 r = *(const floatx4*)&t.v[16 * i + c][16 * i + 4 * q];
#pragma unroll
        for (int s = 0; s < 4; ++s) o = __builtin_amdgcn_mfma_f32_16x16x4f32(r[s], acc[s], o, 0, 0, 0);
        settle();
        col[i] = -o;
#pragma unroll
        for (int s = 0; s < 4; ++s) t.v[16 * i + 4 * q + s][16 * w + c] = -o[s];
    }
    __syncthreads();
}

// ---- what the prepare kernel leaves for the others, all in operand order --------------------------------------------
// T and P (rows of A operands) and, for the gradient, their transposes: the 16 x 32 blocks that are not all zero (six of
// 64 tokens, two of 32), [block][term][lane][8], computed values split already.  Rows 16 w .. of T and P need the
// contraction blocks 0 .. w / 2, those of the transposes w / 2 .. C / 32 - 1.
template <int C> constexpr int BLOCKS = C == 64 ? 6 : 2;
template <typename M> constexpr int BLOCK = 64 * 8 * M::PLANES;          // elements of a block
template <typename M, int C> constexpr int TRI = BLOCKS<C> * BLOCK<M>;
template <int C> __device__ __forceinline__ constexpr int tri_block(int w, int ks) { return C == 32 || w < 2 ? w : 2 * w - 2 + ks; }        // 64: 0 1 2 3 4 5
template <int C> __device__ __forceinline__ constexpr int tri_block_t(int w, int ks) { return C == 32 ? w : w < 2 ? 2 * w + ks : 2 + w; }
// K^T, Q^T: [dim_k / 16][C / 32][lane][8] of the tokens' type, one per key head; K, Q for narrow scans: [C / 16][dim_k / 32][lane][8].
template <typename E, int C> __device__ __forceinline__ int64_t kt_at(const DeltaArgs& a, const Where& w, int ch, int dkp) {
    return (((int64_t)w.b * a.heads_k + w.hk) * a.chunks + ch) * dkp * C;
}
// Gates: gam[C], end[C], beta[C], e^{G_last}.
template <int C> constexpr int GATES = 4 * C;
template <typename M> __device__ __forceinline__ typename M::X load_operand(const typename M::E* p) {
    if constexpr (sizeof(typename M::E) == 4) {
        FF f;
        const floatx4 a = *(const floatx4*)p, b = *(const floatx4*)(p + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) { f.v[i] = a[i]; f.v[4 + i] = b[i]; }
        return f;
    } else {
        return F1{*(const bf16x8*)p};
    }
}
__device__ __forceinline__ void store_operand(bf16_t* p, const F1& f) { *(bf16x8*)p = f.h; }
__device__ __forceinline__ void store_operand(float* p, const FF& f) {
    *(floatx4*)p = floatx4{f.v[0], f.v[1], f.v[2], f.v[3]};
    *(floatx4*)(p + 4) = floatx4{f.v[4], f.v[5], f.v[6], f.v[7]};
}
// An operand straight from a token row.
template <typename M, bool AL> __device__ __forceinline__ typename M::X row_operand(const typename M::E* row, int d, int dim, bool ok) {
    if constexpr (AL && sizeof(typename M::E) == 2) {
        F1 f = {};
        if (ok && d < dim) f.h = *(const bf16x8*)(row + d);
        return f;
    } else {
        float x[8];
        load8<typename M::E, AL>(row, d, dim, ok, x);
        return M::exact(x);
    }
}

// Token tensors of a loop over chunks.  AL (aligned rows, strides that keep a chunk's offsets below 2^30 bytes): through
// buffer descriptors, one per chunk; rows and elements that do not exist get an offset outside them, loads of which return
// zeros and stores of which are dropped.  No branch then stands between a chunk's loads and stores, and the compiler can
// tell which of them a use has to wait for.
constexpr int NOWHERE = 0x7ffffffc;
__device__ __forceinline__ __amdgpu_buffer_rsrc_t tokens(const char* p) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p), 0, 0x40000000, 0x00020000);
}
__device__ __forceinline__ void load_ff(__amdgpu_buffer_rsrc_t rs, int lane, int lane4, int at, FF& f) {
    const floatx4 a = __builtin_bit_cast(floatx4, __builtin_amdgcn_raw_buffer_load_b128(rs, lane, at, 0));
    const floatx4 b = __builtin_bit_cast(floatx4, __builtin_amdgcn_raw_buffer_load_b128(rs, lane4, at, 0));
#pragma unroll
    for (int i = 0; i < 4; ++i) { f.v[i] = a[i]; f.v[4 + i] = b[i]; }
}
// Everything a loop over chunks reads or writes walks with it: a scalar pointer that is moved by one chunk (C tokens, in the
// direction of the loop), lane offsets that do not change.  `go(false)` stays: the last chunk is requested twice.
// The operands of one wavefront's 16 token rows.
template <typename M, int C, int DK, bool AL> struct RowOperands {
    using E = typename M::E;
    static constexpr int ND = DK / 32, ES = sizeof(E);
    const char* p;
    int64_t step, stride;
    int left, turn, dk, row, q, lane;       // tokens from this chunk on, C or -C
    typename M::X f[ND];
    __device__ __forceinline__ RowOperands(const DeltaSeq& s, const void*, int64_t, const Where& w, int dk_, int row_, int q_, int ch, int dir)
        : p((const char*)at<E>(s, w.b, (int64_t)ch * C, w.hk)), step(dir * C * s.t * (int64_t)ES), stride(s.t * (int64_t)ES), left(w.len - ch * C), turn(dir * C), dk(dk_),
          row(row_), q(q_), lane(AL ? row_ * ((int)s.t * ES) + 8 * q_ * ES : 0) {}
    __device__ __forceinline__ void load() {
        const bool ok = row < left;
        if constexpr (AL) {
            const auto r = tokens(p);
#pragma unroll
            for (int d = 0; d < ND; ++d) {
                const int o = ok && 32 * d + 8 * q < dk ? lane + 32 * d * ES : NOWHERE - 16;
                if constexpr (ES == 2) f[d].h = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(r, o, 0, 0));
                else load_ff(r, o, ok && 32 * d + 8 * q + 4 < dk ? o + 16 : NOWHERE - 16, 0, f[d]);
            }
        } else {
#pragma unroll
            for (int d = 0; d < ND; ++d) f[d] = row_operand<M, false>((const E*)(p + row * stride), 32 * d + 8 * q, dk, ok);
        }
    }
    __device__ __forceinline__ void go(bool more) { p += more ? step : 0; left -= more ? turn : 0; }
};
// Token tensors in the layout of results, [4 tokens][column]: element (i0 + r, col + 16 n).
template <typename M, int C, int NT, bool AL> struct ColumnValues {
    using E = typename M::E;
    static constexpr int ES = sizeof(E);
    const char* p;
    int64_t step, stride;
    int left, turn, dim, i0, col, lane;
    unsigned raw[NT][4];
    __device__ __forceinline__ ColumnValues(const DeltaSeq& s, const Where& w, int dim_, int i0_, int col_, int ch, int dir)
        : p((const char*)at<E>(s, w.b, (int64_t)ch * C, w.h)), step(dir * C * s.t * (int64_t)ES), stride(s.t * (int64_t)ES), left(w.len - ch * C),
          turn(dir * C), dim(dim_), i0(i0_), col(col_), lane(AL ? i0_ * ((int)s.t * ES) + col_ * ES : 0) {}
    __device__ __forceinline__ void load() {
        const auto rs = tokens(p);
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const bool ok = i0 + r < left && col + 16 * n < dim;
                if constexpr (AL) {
                    const int o = ok ? lane + 16 * n * ES : NOWHERE;
                    if constexpr (ES == 2) raw[n][r] = (unsigned)(unsigned short)__builtin_amdgcn_raw_buffer_load_b16(rs, o, r * (int)stride, 0);
                    else raw[n][r] = __builtin_amdgcn_raw_buffer_load_b32(rs, o, r * (int)stride, 0);
                } else {
                    raw[n][r] = ok ? bits(*(const E*)(p + (i0 + r) * stride + (int64_t)(col + 16 * n) * ES)) : 0u;
                }
            }
    }
    static __device__ __forceinline__ unsigned bits(E x) {
        if constexpr (ES == 2) return __builtin_bit_cast(unsigned short, x);
        else return __builtin_bit_cast(unsigned, x);
    }
    __device__ __forceinline__ floatx4 get(int n) const {
        floatx4 x;
#pragma unroll
        for (int r = 0; r < 4; ++r) x[r] = __uint_as_float(ES == 2 ? raw[n][r] << 16 : raw[n][r]);
        return x;
    }
    // Writes x to the first `there` rows; rows behind the sequence's length are zeros.
    __device__ __forceinline__ void put(int there, const floatx4 (&x)[NT]) const {
        char* o8 = const_cast<char*>(p);
        const auto rs = tokens(p);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const bool ok = i0 + r < there && col + 16 * n < dim;
                const unsigned v = bits(from_float<E>(i0 + r < left ? x[n][r] : 0.f));
                if constexpr (AL) {
                    const int o = ok ? lane + 16 * n * ES : NOWHERE;
                    if constexpr (ES == 2) __builtin_amdgcn_raw_buffer_store_b16((unsigned short)v, rs, o, r * (int)stride, 0);
                    else __builtin_amdgcn_raw_buffer_store_b32(v, rs, o, r * (int)stride, 0);
                } else if (ok) {
                    char* o = o8 + (i0 + r) * stride + (int64_t)(col + 16 * n) * ES;
                    if constexpr (ES == 2) *(unsigned short*)o = (unsigned short)v;
                    else *(unsigned*)o = v;
                }
            }
    }
    __device__ __forceinline__ void go(bool more) { p += more ? step : 0; left -= more ? turn : 0; }
};
// An array of the library's own with a fixed number of bytes per chunk.
struct Chunks {
    const char* p;
    int64_t step;
    __device__ __forceinline__ Chunks(const void* base, int64_t first, int64_t bytes, int ch, int dir) : p((const char*)base + (first + ch) * bytes), step(dir * bytes) {}
    __device__ __forceinline__ void go(bool more) { p += more ? step : 0; }
};
// The same from the copy in operand order that the prepare kernel makes for narrow scans, 1 KB in a row a load; a load of the token rows
// touches 16 of them, and the eight wavefronts' loads keep the caches' front end busy for half of a chunk's time.  One
// sequence of 16384, 16 heads of 128 x 128, bf16: scan 437 us instead of 500, prepare 99 instead of 89.  Where a scan is not bound by
// its chain the copy costs more than it gives (1024 sequences and heads of 256 tokens, 64 x 64, fp32: 242 us instead of 198).
template <typename M, int C, int DK> struct OrderedRows {
    static constexpr int ND = DK / 32, ES = sizeof(typename M::E);
    Chunks p;
    int lane;
    typename M::X f[ND];
    __device__ __forceinline__ OrderedRows(const DeltaSeq&, const void* copy, int64_t first, const Where&, int, int row, int q, int ch, int dir)
        : p((const char*)copy + row / 16 * ND * 512 * ES, first, DK * C * ES, ch, dir), lane((row % 16 + 16 * q) * 8 * ES) {}
    __device__ __forceinline__ void load() {
        const auto rs = tokens(p.p);
#pragma unroll
        for (int d = 0; d < ND; ++d) {
            if constexpr (ES == 2) f[d].h = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(rs, lane, 512 * ES * d, 0));
            else load_ff(rs, lane, lane + 16, 512 * ES * d, f[d]);
        }
    }
    __device__ __forceinline__ void go(bool more) { p.go(more); }
};
template <typename M, int C, int DK, int NT, bool AL> struct RowsOf { typedef RowOperands<M, C, DK, AL> T; };
template <typename M, int C, int DK, bool AL> struct RowsOf<M, C, DK, 1, AL> { typedef OrderedRows<M, C, DK> T; };
// Results to a padded fp32 array, rows r0 + 4 q + r (lane = the byte offset of row 4 q plus the wavefront's and lane's column).
template <int NT> __device__ __forceinline__ void put_padded(const char* p, int lane, int r0, int ld4, const floatx4 (&x)[NT]) {
    const auto rs = tokens(p);
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(x[n][r]), rs, lane, (r0 + r) * ld4 + 64 * n, 0);
}

// One workgroup per chunk and value head, a wavefront per 16 tokens: K K^T and Q K^T (lower halves), the gates, the inverse, and
// all of it out in the order in which the scans' lanes want it, so that these load operands straight into registers; K^T and
// Q^T by one head of each group.  Bound by the latency of its steps, four workgroups to a CU, and by what it writes: long
// 98 us, sequences 57 us (each about 3 TB/s), windows 26 us; without the inverse 9 % less, without K^T and Q^T 18 to 34 %.
template <typename M, int C, int DK, bool AL>
__global__ __launch_bounds__(4 * C) void delta_prepare_kernel(DeltaArgs a) {
    using E = typename M::E;
    using KT = Tile<M, DK, C, true>;
    constexpr int NW = C / 16, KS = C / 32;
    extern __shared__ __align__(16) unsigned char lds[];
    __shared__ Gates s_g;
    Matrix<C>& s_m = *(Matrix<C>*)lds;
    Matrix<C>& s_t = *(Matrix<C>*)(lds + sizeof(Matrix<C>));     // P first, then T
    const Where w = where_of(a, blockIdx.y);
    const int ch = blockIdx.x, left = w.len - ch * C;
    if (left <= 0) return;
    const int len = min(left, C);
    const int64_t t0 = (int64_t)ch * C, at_chunk = (int64_t)w.bh * a.chunks + ch;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, c = l & 15, q = l >> 4;
    const E* kp = at<E>(a.k, w.b, t0, w.hk);
    const E* qp = at<E>(a.q, w.b, t0, w.hk);
    GateValues v;
    v.load(at<float>(a.g, w.b, t0, w.h), a.g.t, at<float>(a.beta, w.b, t0, w.h), a.beta.t, len);
    gates_of(s_g, v);
    if (w.h % a.group == 0) {               // this key head's transposes
        const KT tile(lds);
        for (int which = 0; which < (a.QT ? 2 : 1); ++which) {
            stage_transposed<M, C, DK, AL>(tile, which ? qp : kp, which ? a.q.t : a.k.t, len, a.dim_k);
            __syncthreads();
            E* o = (E*)(which ? a.QT : a.KT) + kt_at<E, C>(a, w, ch, DK);
            for (int i = threadIdx.x; i < DK / 16 * KS * 64; i += 4 * C) {
                const E* from = tile.p + ((i / (64 * KS)) * 16 + (i & 15)) * KT::LD + (i / 64 % KS) * 32 + (i >> 4 & 3) * 8;
                *(uint4*)(o + i * 8) = *(const uint4*)from;
                if (sizeof(E) == 4) *(uint4*)(o + i * 8 + 4) = *(const uint4*)(from + 4);
            }
            __syncthreads();
        }
    }
    floatx4 kk[NW] = {}, qk[NW] = {};
#pragma unroll
    for (int d = 0; d < DK; d += 32) {
        const int row = 16 * wave + c;
        const auto fk = row_operand<M, AL>(kp + row * a.k.t, d + 8 * q, a.dim_k, row < len);
        const auto fq = row_operand<M, AL>(qp + row * a.q.t, d + 8 * q, a.dim_k, row < len);
        if (a.narrow && w.h % a.group == 0) {       // this key head's rows in operand order
            const int64_t o = kt_at<E, C>(a, w, ch, DK) + ((DK / 32 * wave + d / 32) * 64 + l) * 8;
            store_operand((E*)a.KO + o, fk);
            store_operand((E*)a.QO + o, fq);
        }
#pragma unroll
        for (int n = 0; n < NW; ++n) {
            if (n > wave) break;
            const auto f = row_operand<M, AL>(kp + (16 * n + c) * a.k.t, d + 8 * q, a.dim_k, 16 * n + c < len);
            mma(kk[n], fk, f);
            mma(qk[n], fq, f);
        }
    }
    settle();
    __syncthreads();                        // gates are there
#pragma unroll
    for (int n = 0; n < NW; ++n) {
        const int j = 16 * n + c;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int i = 16 * wave + 4 * q + r;
            const float f = n <= wave && i >= j ? decay(s_g, i, j) : 0.f;
            s_t.v[i][j] = f * qk[n][r];
            s_m.v[i][j] = i > j ? f * kk[n][r] * s_g.beta[j] : 0.f;
        }
    }
    __syncthreads();
    // a matrix and its transpose in operand order
    auto put = [&](void* base, int i, const float* x) {      // eight values of block i / 64, lane i % 64
        E* o = (E*)base + at_chunk * TRI<M, C> + (i >> 6) * BLOCK<M> + (i & 63) * 8;
        const auto f = M::computed(x);
        if constexpr (M::PLANES == 3) {
            *(bf16x8*)o = f.h; *(bf16x8*)(o + 512) = f.m; *(bf16x8*)(o + 1024) = f.l;
        } else {
            *(floatx4*)o = floatx4{f.v[0], f.v[1], f.v[2], f.v[3]};
            *(floatx4*)(o + 4) = floatx4{f.v[4], f.v[5], f.v[6], f.v[7]};
        }
    };
    auto emit = [&](const Matrix<C>& x, void* rows, void* columns) {
        for (int i = threadIdx.x; i < BLOCKS<C> * 64; i += 4 * C) {
            const int blk = i >> 6, bw = C == 32 || blk < 2 ? blk : 2 + (blk - 2) / 2, ks = C == 32 || blk < 2 ? 0 : blk & 1;
            float y[8];
            load8(&x.v[16 * bw + (i & 15)][32 * ks + (i >> 4 & 3) * 8], y);
            put(rows, i, y);
            if (columns) {
                const int tw = C == 32 ? blk : blk < 4 ? blk / 2 : blk - 2, tk = C == 32 ? 0 : blk < 4 ? blk & 1 : 1;
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = x.v[32 * tk + (i >> 4 & 3) * 8 + j][16 * tw + (i & 15)];
                put(columns, i, y);
            }
        }
    };
    emit(s_t, a.P, a.PT);
    __syncthreads();
    invert<C>(s_m, s_t);
    emit(s_t, a.T, a.TT);
    float* g = a.G + at_chunk * GATES<C>;
    if (threadIdx.x < C) {
        g[threadIdx.x] = s_g.gam[threadIdx.x];
        g[C + threadIdx.x] = s_g.end[threadIdx.x];
        g[2 * C + threadIdx.x] = s_g.beta[threadIdx.x];
        if (threadIdx.x == 0) g[3 * C] = s_g.last;
    }
}

// =============================================================================================
// Chunks in order: outputs and states, 16 NT columns per workgroup.  Half of the wavefronts (one per SIMD, 16 tokens each)
// carry the chain K S, X, T X, K^T Y that every chunk has to wait for, the other half what only the outputs need, Q S and
// P Y, in the gaps of the first.  All operands of a chunk are requested into registers, the next chunk's K, V and T once the
// products that wait for LDS have asked for theirs, K^T two phases before it is used.  Bound by the chain: long 448 us, 1.75 us
// for each of 256 chunks (a quarter less if nothing had to be loaded), sequences 147 us, there with 0.33 GB of states and errors
// kept for the gradient, windows 53 us; long in fp32 812 us.  (Every wavefront doing both: long 662 us.)
// =============================================================================================
template <typename M, int C, int DK, int NT> struct ScanLds {
    using S = Tile<M, 16 * NT, DK, false>;          // S^T [column][dim_k]
    using X = Tile<M, 16 * NT, C, false>;           // X^T, Y^T, (e o Y)^T [column][token]
    static constexpr int S0 = 0, X0 = S0 + S::BYTES, Y0 = X0 + X::BYTES, Z0 = Y0 + X::BYTES, BYTES = Z0 + X::BYTES;
};
// By one wavefront.
template <typename E, int COLS> __device__ __forceinline__ void zero_rows(const DeltaSeq& s, const Where& w, int from, int to, int c0, int n) {
    each_of_rows<COLS>(threadIdx.x & 63, from, to, n, [&](int64_t t, int c) { at_out<E>(s, w.b, t, w.h)[c0 + c] = from_float<E>(0.f); });
}
// The C / 32 blocks of a wavefront's rows of T, P or their transposes.  Blocks that are zero are not there: they are asked for
// outside the descriptor and come as zeros, so that no branch stands among a chunk's loads and products.
template <typename M, int C, bool TRANSPOSED> __device__ __forceinline__ void load_tri(const Chunks& base, int wave, int l, typename M::Y (&x)[C / 32]) {
    const auto rs = tokens(base.p);
#pragma unroll
    for (int ks = 0; ks < C / 32; ++ks) {
        const bool there = TRANSPOSED ? ks >= wave / 2 : ks <= wave / 2;
        const int at = there ? (TRANSPOSED ? tri_block_t<C>(wave, ks) : tri_block<C>(wave, ks)) * BLOCK<M> * (int)sizeof(typename M::E) : 0;
        if constexpr (M::PLANES == 3) {
            const int lane = there ? 16 * l : NOWHERE;
            x[ks].h = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(rs, lane, at, 0));
            x[ks].m = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(rs, lane, at + 1024, 0));
            x[ks].l = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(rs, lane, at + 2048, 0));
        } else {
            const int lane = there ? 32 * l : NOWHERE - 32;
            load_ff(rs, lane, lane + 16, at, x[ks]);
        }
    }
}
// The wavefront's strips of K^T or Q^T.
template <typename M, int C, int RS> __device__ __forceinline__ void load_kt(const Chunks& base, int wave, int l, typename M::X (&x)[RS][C / 32]) {
    constexpr int ES = sizeof(typename M::E);
    const auto rs = tokens(base.p);
#pragma unroll
    for (int s = 0; s < RS; ++s)
#pragma unroll
        for (int k = 0; k < C / 32; ++k) {
            const int o = (C / 32 * (wave * RS + s) + k) * 512 * ES;
            if constexpr (ES == 2) x[s][k].h = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(rs, 16 * l, o, 0));
            else load_ff(rs, 32 * l, 32 * l + 16, o, x[s][k]);
        }
}
// The lane's number, found anew: what depends on it behind a loop is then not kept in registers over the loop.
__device__ __forceinline__ int lane_anew() { return __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u)); }
// A sequence and 16 NT columns of its state once more, token by token: for those in which something has come up that is not
// finite.  A product over a chunk has a factor of 0 wherever a token must not reach another one (behind a reset, or the later of
// the two), and that does not stop such a value; here tokens meet through the state alone, and the results are those of
// delta_step_kernel.  What the scans watch is enough: whatever such a value spoils in a chunk is not finite itself and shows in an output
// (dV in the gradient) or in the last state.  THREADS / COLS groups of rows, a column per thread, two barriers a token: 1.5 us a token (one of
// 16384, 16 heads of 128 x 128, bf16: 24 ms instead of 0.4; the windows 0.17 ms instead of 0.05); finite sequences pay nothing measurable.
template <int C, int DK, int NT> struct ByTokens {
    static constexpr int THREADS = 8 * C, COLS = 16 * NT, G = THREADS / COLS, R = DK / G;
    struct Lds { float k[DK], q[DK], a[G][COLS], b[G][COLS], qk[G]; };
    static constexpr int BYTES = 2 * sizeof(Lds);
    static_assert(DK % G == 0 && THREADS >= 2 * DK, "rows and loads go round evenly");
    Lds* s;
    int t, c, g, col;
    bool real;                                      // a column of the state, not padding
    __device__ __forceinline__ ByTokens(void* lds, int thread, int c0, int dv) : s((Lds*)lds), t(thread), c(t % COLS), g(t / COLS), col(c0 + c), real(col < dv) {}
    __device__ __forceinline__ int row(int i) const { return g + G * i; }
    template <typename E> __device__ __forceinline__ void tokens_in(Lds& l, const DeltaArgs& a, const Where& w, int n) const {
        if (t < DK) l.k[t] = t < a.dim_k ? to_float(at<E>(a.k, w.b, n, w.hk)[t]) : 0.f;
        else if (t < 2 * DK) l.q[t - DK] = t - DK < a.dim_k ? to_float(at<E>(a.q, w.b, n, w.hk)[t - DK]) : 0.f;
    }
    __device__ __forceinline__ void load(const float* p, const Where& w, const DeltaArgs& a, float (&x)[R]) const {
#pragma unroll
        for (int i = 0; i < R; ++i) x[i] = p && real && row(i) < a.dim_k ? p[((int64_t)w.bh * a.dim_k + row(i)) * a.dim_v + col] : 0.f;
    }
    __device__ __forceinline__ void store(float* p, const Where& w, const DeltaArgs& a, const float (&x)[R]) const {
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (p && real && row(i) < a.dim_k) p[((int64_t)w.bh * a.dim_k + row(i)) * a.dim_v + col] = x[i];
    }
    __device__ __forceinline__ void keep(float* p, int64_t chunk, const DeltaArgs& a, const float (&x)[R]) const {
#pragma unroll
        for (int i = 0; i < R; ++i) p[(chunk * DK + row(i)) * a.dvp + col] = x[i];
    }
    template <typename E> __device__ __forceinline__ void forward(const DeltaArgs& a, const Where& w, bool kept) const {
        const int64_t first = (int64_t)w.bh * a.chunks;
        float x[R];
        load(a.state, w, a, x);
        for (int n = 0; n < w.len; ++n) {
            Lds& l = s[n & 1];
            if (kept && n % C == 0) keep(a.S, first + n / C, a, x);
            tokens_in<E>(l, a, w, n);
            const float alpha = expf(*at<float>(a.g, w.b, n, w.h)), beta = *at<float>(a.beta, w.b, n, w.h);
            const float v = real ? to_float(at<E>(a.v, w.b, n, w.h)[col]) : 0.f;
            __syncthreads();
            float z = 0.f, o = 0.f, qk = 0.f;
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const float k = l.k[row(i)], q = l.q[row(i)];
                x[i] = damp(alpha, x[i]);
                z += x[i] * k; o += x[i] * q; qk += q * k;
            }
            l.a[g][c] = z; l.b[g][c] = o;
            if (c == 0) l.qk[g] = qk;
            __syncthreads();
            z = o = qk = 0.f;
            for (int i = 0; i < G; ++i) { z += l.a[i][c]; o += l.b[i][c]; qk += l.qk[i]; }
            const float r = real ? v - z : 0.f, u = real ? beta * r : 0.f;
#pragma unroll
            for (int i = 0; i < R; ++i) x[i] = row(i) < a.dim_k ? x[i] + l.k[row(i)] * u : 0.f;
            if (g == 0 && real) at_out<E>(a.out, w.b, n, w.h)[col] = from_float<E>(a.scale * (o + qk * u));
            if (g == 0 && kept) a.R[(first * C + n) * a.dvp + col] = r;
        }
        if (kept)
            for (int n = w.len + g; n % C != 0 && n / C == (w.len - 1) / C; n += G) a.R[(first * C + n) * a.dvp + col] = 0.f;
        store(a.state_out, w, a, x);
    }
    // y is the state's gradient without what the chunk's later tokens take of it: dY is what a chunk's products give.
    template <typename E> __device__ __forceinline__ void backward(const DeltaArgs& a, const Where& w) const {
        const int64_t first = (int64_t)w.bh * a.chunks;
        float x[R], y[R];
        load(a.state_grad, w, a, x);
        for (int n = w.len + g; n % C != 0 && n / C == (w.len - 1) / C; n += G) a.dX[(first * C + n) * a.dvp + col] = a.dY[(first * C + n) * a.dvp + col] = 0.f;
        for (int n = w.len - 1; n >= 0; --n) {
            Lds& l = s[n & 1];
            if (n == w.len - 1 || n % C == C - 1) {
                keep(a.dS, first + n / C, a, x);
#pragma unroll
                for (int i = 0; i < R; ++i) y[i] = x[i];
            }
            tokens_in<E>(l, a, w, n);
            const float alpha = expf(*at<float>(a.g, w.b, n, w.h)), beta = *at<float>(a.beta, w.b, n, w.h);
            const float o = real ? a.scale * to_float(at<E>(a.out_grad, w.b, n, w.h)[col]) : 0.f;
            __syncthreads();
            float zx = 0.f, zy = 0.f;
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const float k = l.k[row(i)], add = row(i) < a.dim_k && real ? l.q[row(i)] * o : 0.f;
                x[i] += add; y[i] += add;
                zx += x[i] * k; zy += y[i] * k;
            }
            l.a[g][c] = zx; l.b[g][c] = zy;
            __syncthreads();
            zx = zy = 0.f;
            for (int i = 0; i < G; ++i) { zx += l.a[i][c]; zy += l.b[i][c]; }
            const float dx = real ? beta * zx : 0.f;
#pragma unroll
            for (int i = 0; i < R; ++i) {
                x[i] = damp(alpha, row(i) < a.dim_k && real ? x[i] - l.k[row(i)] * dx : 0.f);
                y[i] = damp(alpha, y[i]);
            }
            if (g == 0) {
                a.dX[(first * C + n) * a.dvp + col] = dx;
                a.dY[(first * C + n) * a.dvp + col] = real ? zy : 0.f;
                if (real) at_out<E>(a.dv, w.b, n, w.h)[col] = from_float<E>(dx);
            }
        }
        store(a.dstate, w, a, x);
    }
};
struct ChunkGates {                         // of this lane's tokens i0 .. i0 + 3
    floatx4 gam, end, beta;
    float last;
    template <int C> __device__ __forceinline__ void load(const Chunks& base, int i0) {
        const auto rs = tokens(base.p);
        gam = __builtin_bit_cast(floatx4, __builtin_amdgcn_raw_buffer_load_b128(rs, 4 * i0, 0, 0));
        end = __builtin_bit_cast(floatx4, __builtin_amdgcn_raw_buffer_load_b128(rs, 4 * i0, 4 * C, 0));
        beta = __builtin_bit_cast(floatx4, __builtin_amdgcn_raw_buffer_load_b128(rs, 4 * i0, 8 * C, 0));
        last = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs, 0, 12 * C, 0));
    }
};
// The state (or its gradient) of a wavefront: rows 16 (wave RS + s) + 4 q + r, columns c0 + 16 n + c.
template <int RS, int NT> __device__ __forceinline__ void load_state(const float* p, const Where& w, int wave, int q, int col, int dk, int dv, floatx4 (&S)[RS][NT]) {
#pragma unroll
    for (int s = 0; s < RS; ++s)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int r0 = 16 * (wave * RS + s) + 4 * q;
#pragma unroll
            for (int r = 0; r < 4; ++r)
                S[s][n][r] = p && r0 + r < dk && col + 16 * n < dv ? p[((int64_t)w.bh * dk + r0 + r) * dv + col + 16 * n] : 0.f;
        }
}
template <int RS, int NT> __device__ __forceinline__ void store_state(float* p, const Where& w, int wave, int q, int col, int dk, int dv, const floatx4 (&S)[RS][NT]) {
    if (!p) return;
#pragma unroll
    for (int s = 0; s < RS; ++s)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int r0 = 16 * (wave * RS + s) + 4 * q;
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (r0 + r < dk && col + 16 * n < dv) p[((int64_t)w.bh * dk + r0 + r) * dv + col + 16 * n] = S[s][n][r];
        }
}
template <typename M, int C, int DK, int NT, bool AL, bool KEEP>
__global__ __launch_bounds__(8 * C) __attribute__((amdgpu_waves_per_eu(DK == 128 || !AL ? 2 : 4, DK == 128 || !AL ? 2 : 4))) void delta_scan_kernel(DeltaArgs a) {
    using E = typename M::E;
    using L = ScanLds<M, C, DK, NT>;
    constexpr int RS = DK / C, KS = C / 32, ND = DK / 32, NW = C / 16;      // 16-row strips of the state per wavefront, contraction steps
    extern __shared__ __align__(16) unsigned char lds[];
    const typename L::S tS(lds + L::S0);
    const typename L::X tX(lds + L::X0), tY(lds + L::Y0), tZ(lds + L::Z0);
    int bh, block;
    place_of(blockIdx.x, a.batch * a.heads_v, a.dvp / (16 * NT), bh, block);
    const Where w = where_of(a, bh);
    const int all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = all % NW, l = threadIdx.x & 63, c = l & 15, q = l >> 4, c0 = block * 16 * NT;
    const int dk = a.dim_k, dv = a.dim_v, row = 16 * wave + c, i0 = 16 * wave + 4 * q;
    const int chunks = (w.len + C - 1) / C;
    const int64_t first = (int64_t)w.bh * a.chunks;
    constexpr int64_t tri_bytes = TRI<M, C> * (int)sizeof(E), kt_bytes = DK * C * (int)sizeof(E);
    const int64_t first_k = ((int64_t)w.b * a.heads_k + w.hk) * a.chunks;
    ChunkGates G, Gn;                               // this chunk's, the next one's
    Chunks pG(a.G, first, GATES<C> * 4, 0, 1);
    __shared__ int s_odd;                           // whether anything that is not finite has come up
    if (threadIdx.x == 0) s_odd = 0;
    if (all < NW) {                                 // the chain
        typename RowsOf<M, C, DK, NT, AL>::T K(a.k, a.KO, first_k, w, dk, row, q, 0, 1);
        ColumnValues<M, C, NT, AL> V(a.v, w, dv, i0, c0 + c, 0, 1);
        Chunks pT(a.T, first, tri_bytes, 0, 1), pK(a.KT, first_k, kt_bytes, 0, 1);
        Chunks pS(a.S + c0, first, (int64_t)DK * a.dvp * 4, 0, 1), pR(a.R + c0, first, (int64_t)C * a.dvp * 4, 0, 1);
        const int ld4 = 4 * a.dvp, lane_s = (16 * wave * RS + 4 * q) * ld4 + 4 * c, lane_r = (16 * wave + 4 * q) * ld4 + 4 * c;
        typename M::X kt[RS][KS];
        typename M::Y T[KS];
        floatx4 S[RS][NT];
        if (chunks > 0) {
            K.load(); V.load(); G.load<C>(pG, i0);
            load_tri<M, C, false>(pT, wave, l, T);
        }
        load_state<RS, NT>(a.state, w, wave, q, c0 + c, dk, dv, S);
#pragma unroll
        for (int s = 0; s < RS; ++s)
#pragma unroll
            for (int n = 0; n < NT; ++n) tS.put4(16 * n + c, 16 * (wave * RS + s) + 4 * q, S[s][n]);
        for (int ch = 0; ch < chunks; ++ch) {
            const bool more = ch + 1 < chunks;
            __syncthreads();                        // 1: the state is in LDS
            Acc za[NT];
            {
                typename M::Y f[ND][NT];
                tS.template frags<ND, NT>(c, 8 * q, f);
                load_kt<M, C, RS>(pK, wave, l, kt);
                pK.go(true);
#pragma unroll
                for (int d = 0; d < ND; ++d)
#pragma unroll
                    for (int n = 0; n < NT; ++n) za[n].add(K.f[d], f[d][n]);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const floatx4 v = V.get(n), z = za[n].sum();
                floatx4 x;
#pragma unroll
                for (int r = 0; r < 4; ++r) x[r] = v[r] - damp(G.gam[r], z[r]);
                tX.put4(16 * n + c, i0, x);
            }
            __syncthreads();                        // 2: X
            Acc ra[NT];
            {
                typename M::Y f[KS][NT];
                tX.template frags<KS, NT>(c, 8 * q, f);
                pG.go(more);
                Gn.load<C>(pG, i0);
                K.go(more);
                K.load();
                V.go(more);
                V.load();
#pragma unroll
                for (int k = 0; k < KS; ++k) {
#pragma unroll
                    for (int n = 0; n < NT; ++n) ra[n].add(T[k], f[k][n]);
                }
            }
            floatx4 rr[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) rr[n] = ra[n].sum();
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const floatx4 y = G.beta * rr[n];
                tZ.put4(16 * n + c, i0, G.end * y);
                tY.put4(16 * n + c, i0, y);
            }
            const float last = G.last;
            if (KEEP) {
#pragma unroll
                for (int s = 0; s < RS; ++s) put_padded<NT>(pS.p, lane_s, 16 * s, ld4, S[s]);
                put_padded<NT>(pR.p, lane_r, 0, ld4, rr);
                pS.go(true);
                pR.go(true);
            }
            __syncthreads();                        // 3: Y; all have read the state
            typename M::Y f[KS][NT];
            tZ.template frags<KS, NT>(c, 8 * q, f);
            pT.go(more);
            load_tri<M, C, false>(pT, wave, l, T);
#pragma unroll
            for (int s = 0; s < RS; ++s) {
                const int r0 = 16 * (wave * RS + s);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) S[s][n][r] = damp(last, S[s][n][r]);
                    Acc sa;
                    sa.a[0] = S[s][n];
#pragma unroll
                    for (int k = 0; k < KS; ++k) sa.add(kt[s][k], f[k][n]);
                    S[s][n] = sa.sum();
                    tS.put4(16 * n + c, r0 + 4 * q, S[s][n]);
                }
            }
            G = Gn;
        }
        float odd = 0.f;
#pragma unroll
        for (int s = 0; s < RS; ++s)
#pragma unroll
            for (int n = 0; n < NT; ++n) odd = watch(odd, S[s][n]);
        if (chunks > 0) {
            if (odd != 0.f) s_odd = 1;
            __syncthreads();
        }
        if (chunks == 0 || !s_odd) {
            const int l = lane_anew();
            store_state<RS, NT>(a.state_out, w, wave, l >> 4, c0 + (l & 15), dk, dv, S);
            return;
        }
    } else {                                        // the outputs
        typename RowsOf<M, C, DK, NT, AL>::T Q(a.q, a.QO, first_k, w, dk, row, q, 0, 1);
        ColumnValues<M, C, NT, AL> O(a.out, w, dv, i0, c0 + c, 0, 1);
        Chunks pP(a.P, first, tri_bytes, 0, 1);
        typename M::Y P[KS];
        float odd = 0.f;
        if (chunks > 0) {
            Q.load(); G.load<C>(pG, i0);
            load_tri<M, C, false>(pP, wave, l, P);
        }
        for (int ch = 0; ch < chunks; ++ch) {
            const bool more = ch + 1 < chunks;
            __syncthreads();                        // 1
            floatx4 o[NT] = {};
            {
                typename M::Y f[ND][NT];
                tS.template frags<ND, NT>(c, 8 * q, f);
#pragma unroll
                for (int d = 0; d < ND; ++d)
#pragma unroll
                    for (int n = 0; n < NT; ++n) mma(o[n], Q.f[d], f[d][n]);
            }
            if constexpr (!AL) settle();            // loads of rows that are not aligned have branches
            pG.go(more);
            Gn.load<C>(pG, i0);
            Q.go(more);
            Q.load();
            __syncthreads();                        // 2
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int r = 0; r < 4; ++r) o[n][r] = damp(G.gam[r], o[n][r]);
            G = Gn;
            __syncthreads();                        // 3
            {
                typename M::Y f[KS][NT];
                tY.template frags<KS, NT>(c, 8 * q, f);
#pragma unroll
                for (int k = 0; k < KS; ++k) {
#pragma unroll
                    for (int n = 0; n < NT; ++n) mma(o[n], P[k], f[k][n]);
                }
            }
            pP.go(more);
            load_tri<M, C, false>(pP, wave, l, P);
#pragma unroll
            for (int n = 0; n < NT; ++n) { o[n] *= a.scale; odd = watch(odd, o[n]); }
            O.put(a.steps - ch * C, o);
            O.go(true);
        }
        const int n = min(16 * NT, dv - c0);
        if (n > 0 && a.steps > chunks * C && all == NW) zero_rows<E, 16 * NT>(a.out, w, chunks * C, a.steps, c0, n);
        if (chunks == 0) return;
        if (odd != 0.f) s_odd = 1;
        __syncthreads();
        if (!s_odd) return;
    }
    static_assert(ByTokens<C, DK, NT>::BYTES <= L::BYTES, "what goes by tokens takes the tiles' place");
    ByTokens<C, DK, NT>(lds, 64 * all + lane_anew(), c0, dv).template forward<E>(a, w, KEEP);
}

// =============================================================================================
// Gradient, chunks in reverse order: dV, and what delta_back_kernel needs of every chunk (dS1, dX, dY).  Again half of the
// wavefronts carry the chain K dS, dY, T^T dR, K^T dX; the other half find what it adds from outside, P^T dO and
// Q^T (gam o dO), one chunk ahead, and hand it over in LDS in the layout of the results.  Bound by the chain and by what it
// writes (dX, dY, dS: 0.4 GB in the sequences): sequences 163 us, windows 67 us; sequences in fp32 221 us.
// =============================================================================================
template <typename M, int C, int DK, int NT> struct BackScanLds {
    using S = Tile<M, 16 * NT, DK, false>;          // dS^T [column][dim_k]
    using O = Tile<M, 16 * NT, C, true>;            // dO^T [column][token]
    using X = Tile<M, 16 * NT, C, false>;           // dR^T, (gam o dX)^T, (gam o dO)^T [column][token]
    static constexpr int S0 = 0, O0 = S0 + S::BYTES, X0 = O0 + O::BYTES, Y0 = X0 + X::BYTES, G0 = Y0 + X::BYTES, P0 = G0 + X::BYTES,
                         Q0 = P0 + C * 16 * NT * 4, BYTES = Q0 + DK * 16 * NT * 4;      // P0, Q0: results of P^T dO, Q^T (gam o dO)
};
template <typename M, int C, int DK, int NT, bool AL>
__global__ __launch_bounds__(8 * C) __attribute__((amdgpu_waves_per_eu(DK == 128 ? 2 : AL ? 3 : 1, DK == 128 ? 2 : 8))) void delta_back_scan_kernel(DeltaArgs a) {
    using E = typename M::E;
    using L = BackScanLds<M, C, DK, NT>;
    constexpr int RS = DK / C, KS = C / 32, ND = DK / 32, NW = C / 16;
    extern __shared__ __align__(16) unsigned char lds[];
    const typename L::S tS(lds + L::S0);
    const typename L::O tO(lds + L::O0);
    const typename L::X tR(lds + L::X0), tX(lds + L::Y0), tG(lds + L::G0);
    int bh, block;
    place_of(blockIdx.x, a.batch * a.heads_v, a.dvp / (16 * NT), bh, block);
    const Where w = where_of(a, bh);
    const int all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = all % NW, l = threadIdx.x & 63, c = l & 15, q = l >> 4, c0 = block * 16 * NT;
    floatx4* const tP = (floatx4*)(lds + L::P0) + wave * NT * 64 + l;               // [n * 64]
    floatx4* const tQ = (floatx4*)(lds + L::Q0) + wave * RS * NT * 64 + l;          // [(s * NT + n) * 64]
    const int dk = a.dim_k, dv = a.dim_v, row = 16 * wave + c, i0 = 16 * wave + 4 * q;
    const int chunks = (w.len + C - 1) / C;
    const int64_t first = (int64_t)w.bh * a.chunks;
    constexpr int64_t tri_bytes = TRI<M, C> * (int)sizeof(E), kt_bytes = DK * C * (int)sizeof(E);
    const int64_t first_k = ((int64_t)w.b * a.heads_k + w.hk) * a.chunks;
    const int end = max(chunks - 1, 0);
    ChunkGates G, Gn;
    Chunks pG(a.G, first, GATES<C> * 4, end, -1);
    __shared__ int s_odd;
    if (threadIdx.x == 0) s_odd = 0;
    if (all < NW) {                                 // the chain
        typename RowsOf<M, C, DK, NT, AL>::T K(a.k, a.KO, first_k, w, dk, row, q, end, -1);
        ColumnValues<M, C, NT, AL> dV(a.dv, w, dv, i0, c0 + c, end, -1);
        Chunks pT(a.TT, first, tri_bytes, end, -1), pK(a.KT, first_k, kt_bytes, end, -1);
        Chunks pS(a.dS + c0, first, (int64_t)DK * a.dvp * 4, end, -1), pX(a.dX + c0, first, (int64_t)C * a.dvp * 4, end, -1),
            pY(a.dY + c0, first, (int64_t)C * a.dvp * 4, end, -1);
        const int ld4 = 4 * a.dvp, lane_s = (16 * wave * RS + 4 * q) * ld4 + 4 * c, lane_r = (16 * wave + 4 * q) * ld4 + 4 * c;
        typename M::X kt[RS][KS];
        typename M::Y T[KS];
        floatx4 S[RS][NT];
        float odd = 0.f;
        if (chunks > 0) {
            K.load(); G.load<C>(pG, i0);
            load_tri<M, C, true>(pT, wave, l, T);
            load_kt<M, C, RS>(pK, wave, l, kt);
        }
        load_state<RS, NT>(a.state_grad, w, wave, q, c0 + c, dk, dv, S);
#pragma unroll
        for (int s = 0; s < RS; ++s)
#pragma unroll
            for (int n = 0; n < NT; ++n) tS.put4(16 * n + c, 16 * (wave * RS + s) + 4 * q, S[s][n]);
        if (chunks > 0) __syncthreads();            // 0: the helpers' dO
        for (int ch = chunks - 1; ch >= 0; --ch) {
            const bool more = ch > 0;
            __syncthreads();                        // 1: dS, P^T dO, Q^T (gam o dO)
            floatx4 y[NT], gq[RS][NT];
            {
                Acc ya[NT];
                typename M::Y f[ND][NT];
                tS.template frags<ND, NT>(c, 8 * q, f);
#pragma unroll
                for (int d = 0; d < ND; ++d)
#pragma unroll
                    for (int n = 0; n < NT; ++n) ya[n].add(K.f[d], f[d][n]);
#pragma unroll
                for (int n = 0; n < NT; ++n) y[n] = ya[n].sum();
            }
            pG.go(more);
            Gn.load<C>(pG, i0);
            K.go(more);
            K.load();
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const floatx4 p = tP[n * 64];
#pragma unroll
                for (int r = 0; r < 4; ++r) y[n][r] = a.scale * p[r] + damp(G.end[r], y[n][r]);
                tR.put4(16 * n + c, i0, G.beta * y[n]);
            }
#pragma unroll
            for (int s = 0; s < RS; ++s)
#pragma unroll
                for (int n = 0; n < NT; ++n) gq[s][n] = tQ[(s * NT + n) * 64];
            __syncthreads();                        // 2: dR; P^T dO and Q^T (gam o dO) are taken
            floatx4 dx[NT];
            {
                Acc xa[NT];
                typename M::Y f[KS][NT];
                tR.template frags<KS, NT>(c, 8 * q, f);
#pragma unroll
                for (int k = 0; k < KS; ++k) {
#pragma unroll
                    for (int n = 0; n < NT; ++n) xa[n].add(T[k], f[k][n]);
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) dx[n] = xa[n].sum();
            }
            pT.go(more);
            load_tri<M, C, true>(pT, wave, l, T);
#pragma unroll
            for (int n = 0; n < NT; ++n) tX.put4(16 * n + c, i0, -G.gam * dx[n]);
            put_padded<NT>(pY.p, lane_r, 0, ld4, y);
            pY.go(true);
#pragma unroll
            for (int s = 0; s < RS; ++s) put_padded<NT>(pS.p, lane_s, 16 * s, ld4, S[s]);
            pS.go(true);
            const float last = G.last;
            __syncthreads();                        // 3: dX; all have read dS
            typename M::Y f[KS][NT];
            tX.template frags<KS, NT>(c, 8 * q, f);
#pragma unroll
            for (int s = 0; s < RS; ++s) {
                const int r0 = 16 * (wave * RS + s);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) S[s][n][r] = damp(last, S[s][n][r]) + gq[s][n][r];
                    Acc sa;
                    sa.a[0] = S[s][n];
#pragma unroll
                    for (int k = 0; k < KS; ++k) sa.add(kt[s][k], f[k][n]);
                    S[s][n] = sa.sum();
                    tS.put4(16 * n + c, r0 + 4 * q, S[s][n]);
                }
            }
            pK.go(more);
            load_kt<M, C, RS>(pK, wave, l, kt);
            G = Gn;
#pragma unroll
            for (int n = 0; n < NT; ++n) odd = watch(odd, dx[n]);
            put_padded<NT>(pX.p, lane_r, 0, ld4, dx);
            pX.go(true);
            dV.put(a.steps - ch * C, dx);
            dV.go(true);
        }
#pragma unroll
        for (int s = 0; s < RS; ++s)
#pragma unroll
            for (int n = 0; n < NT; ++n) odd = watch(odd, S[s][n]);
        if (chunks > 0) {
            if (odd != 0.f) s_odd = 1;
            __syncthreads();
        }
        if (chunks == 0 || !s_odd) {
            const int l = lane_anew();
            store_state<RS, NT>(a.dstate, w, wave, l >> 4, c0 + (l & 15), dk, dv, S);
            return;
        }
    } else {                                        // P^T dO and Q^T (gam o dO), a chunk ahead of the chain
        ColumnValues<M, C, NT, AL> O(a.out_grad, w, dv, i0, c0 + c, end, -1);
        Chunks pP(a.PT, first, tri_bytes, end, -1), pQ(a.QT, first_k, kt_bytes, end, -1);
        typename M::X qt[RS][KS];
        typename M::Y P[KS];
        auto load = [&] {
            load_tri<M, C, true>(pP, wave, l, P);
            load_kt<M, C, RS>(pQ, wave, l, qt);
        };
        auto load_next = [&](bool more) {
            pP.go(more);
            pQ.go(more);
            load();
        };
        auto load_o = [&](bool more) {
            O.go(more);
            O.load();
            pG.go(more);
            G.load<C>(pG, i0);
        };
        auto put = [&] {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const floatx4 o = O.get(n);
                tO.put4(16 * n + c, i0, o);
                tG.put4(16 * n + c, i0, a.scale * G.gam * o);
            }
        };
        floatx4 p[NT], g[RS][NT];
        auto products = [&] {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                p[n] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < KS; ++k) mma(p[n], P[k], tO.frag(16 * n + c, 32 * k + 8 * q));
#pragma unroll
                for (int s = 0; s < RS; ++s) {
                    g[s][n] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int k = 0; k < KS; ++k) mma(g[s][n], qt[s][k], tG.frag(16 * n + c, 32 * k + 8 * q));
                }
            }
        };
        auto hand_over = [&] {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                tP[n * 64] = p[n];
#pragma unroll
                for (int s = 0; s < RS; ++s) tQ[(s * NT + n) * 64] = g[s][n];
            }
        };
        if (chunks > 0) {
            load_o(false);
            load();
            put();
            load_o(chunks > 1);
            __syncthreads();                        // 0
            products();
            hand_over();
            load_next(chunks > 1);
        }
        for (int ch = chunks - 1; ch >= 0; --ch) {  // the chunk before `ch` here
            const bool more = ch > 1;
            __syncthreads();                        // 1: dO of the last chunk has been used
            put();
            load_o(more);
            __syncthreads();                        // 2: the new dO is there
            products();
            load_next(more);
            __syncthreads();                        // 3: and what was handed over before has been taken
            hand_over();
        }
        const int n = min(16 * NT, dv - c0);
        if (n > 0 && a.steps > chunks * C && all == NW) zero_rows<E, 16 * NT>(a.dv, w, chunks * C, a.steps, c0, n);
        if (chunks == 0) return;
        __syncthreads();
        if (!s_odd) return;
    }
    static_assert(ByTokens<C, DK, NT>::BYTES <= L::BYTES, "what goes by tokens takes the tiles' place");
    ByTokens<C, DK, NT>(lds, 64 * all + lane_anew(), c0, dv).template backward<E>(a, w);
}

// =============================================================================================
// Gradient, all chunks at once: dQ, dK, dbeta, dg.  Two wavefronts per 16 tokens, each with half of dim_k.  First the
// contractions over the columns, 32 at a time: everything but dO is brought from memory, split and put into LDS once for all
// wavefronts, the next 32 columns being on their way meanwhile; then those over tokens with E and F in LDS, K^T and Q^T
// straight from memory.  With a.heads_wg = group a workgroup takes the value heads of one key head one after the other and
// adds dQ and dK up in registers; where that leaves too few workgroups, it takes one, and delta_group_kernel adds.  With keys of
// 128 it fills a CU's LDS and registers alone, and is bound by LDS: sequences 220 us, 0.4 GB of states at 1.8 TB/s; windows 58 us.
// fp32 with keys of 128, chunks of 64 and several heads a workgroup keeps 27 to 36 registers in scratch memory: sequences in fp32 350 us.
// =============================================================================================
template <typename M, int C, int DK> struct BackLds {
    using R = Tile<M, C, 32, false>;        // R, Y, dX
    using S = Tile<M, DK, 32, false>;       // S0, dS1
    using W = Tile<M, C, C, false>;         // E, E^T, F diag(beta), F^T
    static constexpr int R0 = 0, Y0 = R0 + R::BYTES, X0 = Y0 + R::BYTES, S0 = X0 + R::BYTES, S1 = S0 + S::BYTES, FIRST = S1 + S::BYTES;
    static constexpr int E0 = 0, ET0 = E0 + W::BYTES, F0 = ET0 + W::BYTES, FT0 = F0 + W::BYTES, SECOND = FT0 + W::BYTES;
    static constexpr int BYTES = FIRST > SECOND ? FIRST : SECOND;
};
__device__ __forceinline__ float sum16(float x) {      // over the 16 lanes that hold one row of a result
#pragma unroll
    for (int d = 1; d < 16; d *= 2) x += __shfl_xor(x, d);
    return x;
}
template <typename M, int C, int DK, bool AL, bool MANY>
__global__ __launch_bounds__(8 * C) void delta_back_kernel(DeltaArgs a) {
    using E = typename M::E;
    using L = BackLds<M, C, DK>;
    constexpr int NW = C / 16, KS = C / 32, NK = DK / 32, THREADS = 8 * C, UN = 8 * DK / THREADS;      // NK: 16-column tiles of a wavefront's half
    extern __shared__ __align__(16) unsigned char lds[];
    __shared__ Gates s_g;
    __shared__ float s_dG[2][C], s_b[2][C], s_yr[C], s_ext[2 * NW];
    const typename L::R tR(lds + L::R0), tY(lds + L::Y0), tX(lds + L::X0);
    const typename L::S tS0(lds + L::S0), tS1(lds + L::S1);
    const typename L::W tE(lds + L::E0), tET(lds + L::ET0), tF(lds + L::F0), tFT(lds + L::FT0);
    const int heads = MANY ? a.heads_wg : 1, per_seq = a.heads_v / heads;
    Where w = where_of(a, MANY ? (int)blockIdx.y / per_seq * a.heads_v + (int)blockIdx.y % per_seq * heads : (int)blockIdx.y);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int strip = wave % NW, half = wave / NW, n0 = half * NK;
    const int dk = a.dim_k, ch = blockIdx.x, dvp = a.dvp;
    const int64_t t0 = (int64_t)ch * C;
    const int len = min(w.len - ch * C, C), rows = min(a.steps - ch * C, C);
    auto put = [&](const DeltaSeq& s, float* part, int i, int d, float x) {
        if (part) part[(((int64_t)w.b * a.steps + t0 + i) * a.heads_v + w.h) * dk + d] = x;
        else at_out<E>(s, w.b, t0 + i, w.hk)[d] = from_float<E>(x);
    };
    if (len <= 0) {
        for (int i = threadIdx.x; i < rows * dk; i += THREADS) { put(a.dq, a.part_q, i / dk, i % dk, 0.f); put(a.dk, a.part_k, i / dk, i % dk, 0.f); }
        for (int i = threadIdx.x; i < rows * heads; i += THREADS) {
            *at_out<float>(a.dg, w.b, t0 + i / heads, w.h + i % heads) = 0.f;
            *at_out<float>(a.dbeta, w.b, t0 + i / heads, w.h + i % heads) = 0.f;
        }
        return;
    }
    const int64_t kt0 = kt_at<E, C>(a, w, ch, DK);
    floatx4 sum_q[NK], sum_k[NK];
    if (MANY) {
#pragma unroll
        for (int n = 0; n < NK; ++n) sum_q[n] = sum_k[n] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    GateValues v;
    v.load(at<float>(a.g, w.b, t0, w.h), a.g.t, at<float>(a.beta, w.b, t0, w.h), a.beta.t, len);
    for (int head = 0; head < heads; ++head, ++w.h, ++w.bh) {
        // lane numbers anew for every head: what is worked out from them would otherwise be kept over the loop, in registers
        // that are not there
        int unit = threadIdx.x;
        if (MANY) asm volatile("" : "+v"(unit));
        const int l = unit & 63, c = l & 15, q = l >> 4, row = 16 * strip + c, i0 = 16 * strip + 4 * q;
        const int64_t at_chunk = (int64_t)w.bh * a.chunks + ch;
        if (head) __syncthreads();          // the last one's gates and sums have been used
        const bool first = unit < 4 * C;    // this thread's share of R and dY, or of dX: eight columns of one row
        const int ur = (first ? unit : unit - 4 * C) >> 2, uk = (unit & 3) * 8;
        const float* RX = (first ? a.R : a.dX) + (at_chunk * C + ur) * dvp + uk;
        const float* dY = a.dY + (at_chunk * C + ur) * dvp + uk;
        const float* S0 = a.S + (at_chunk * DK + (unit >> 3)) * dvp + (unit & 7) * 4;       // and of S0 and dS1: four columns of some rows
        const float* S1 = a.dS + (at_chunk * DK + (unit >> 3)) * dvp + (unit & 7) * 4;
        const E* dO = at<E>(a.out_grad, w.b, t0, w.h) + row * a.out_grad.t;
        float rx[8], dy[8];
        floatx4 s0[UN], s1[UN];
        typename M::X fo;
        auto load = [&](int d) {
            load8(RX + d, rx);
            if (first) load8(dY + d, dy);
#pragma unroll
            for (int i = 0; i < UN; ++i) {
                s0[i] = *(const floatx4*)(S0 + i * (THREADS / 8) * dvp + d);
                s1[i] = *(const floatx4*)(S1 + i * (THREADS / 8) * dvp + d);
            }
            fo = row_operand<M, AL>(dO, d + 8 * q, a.dim_v, row < len);
        };
        load(0);
        gates_of(s_g, v);
        if (MANY && head + 1 < heads) v.load(at<float>(a.g, w.b, t0, w.h + 1), a.g.t, at<float>(a.beta, w.b, t0, w.h + 1), a.beta.t, len);
        floatx4 dq[NK] = {}, ks[NK] = {}, ke[NK] = {}, ef[NW] = {};     // ef: E (first half of the wavefronts) or F
        float yr = 0.f, ss = 0.f;           // dY.R of row ur, <dS1, S0>: this thread's elements
        __syncthreads();                    // gates are there
        for (int d = 0; d < dvp; d += 32) {
            if (first) {
                const float beta = s_g.beta[ur];
                tR.put8(ur, uk, rx);
#pragma unroll
                for (int j = 0; j < 8; ++j) { yr += rx[j] * dy[j]; rx[j] *= beta; }
                tY.put8(ur, uk, rx);
            } else {
                tX.put8(ur, uk, rx);
            }
#pragma unroll
            for (int i = 0; i < UN; ++i) {
                const int r = (unit >> 3) + i * (THREADS / 8);
                tS0.put4(r, (unit & 7) * 4, s0[i]);
                tS1.put4(r, (unit & 7) * 4, s1[i]);
                const floatx4 p = s0[i] * s1[i];
                ss += p[0] + p[1] + p[2] + p[3];
            }
            const auto fd = fo;
            if (d + 32 < dvp) load(d + 32);
            __syncthreads();
            const auto fy = tY.frag(row, 8 * q);
            const auto fx = tX.frag(row, 8 * q);
            if (half == 0) {
#pragma unroll
                for (int n = 0; n < NW; ++n)
                    if (n <= strip) mma(ef[n], fd, tY.frag(16 * n + c, 8 * q));
            } else {
#pragma unroll
                for (int n = 0; n < NW; ++n)
                    if (n <= strip) mma(ef[n], fx, tR.frag(16 * n + c, 8 * q));
            }
#pragma unroll
            for (int n = 0; n < NK; ++n) {
                const auto g = tS0.frag(16 * (n0 + n) + c, 8 * q);
                mma(dq[n], fd, g);
                mma(ks[n], fx, g);
                mma(ke[n], fy, tS1.frag(16 * (n0 + n) + c, 8 * q));
            }
            settle();
            __syncthreads();
        }
        // K^T and Q^T of this half: right operands.  The same for every head, but too many registers to keep.
        int64_t kt = kt0;
        if (MANY) asm volatile("" : "+s"(kt));
        const E* KT = (const E*)a.KT + kt;
        const E* QT = (const E*)a.QT + kt;
        typename M::X fk[NK][KS], fq[NK][KS];
#pragma unroll
        for (int n = 0; n < NK; ++n)
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                fk[n][k] = load_operand<M>(KT + ((KS * (n0 + n) + k) * 64 + l) * 8);
                fq[n][k] = load_operand<M>(QT + ((KS * (n0 + n) + k) * 64 + l) * 8);
            }
        yr += __shfl_xor(yr, 1);
        yr += __shfl_xor(yr, 2);
        if (first && (unit & 3) == 0) s_yr[ur] = yr;
#pragma unroll
        for (int n = 0; n < NW; ++n) {
            const int j = 16 * n + c;
            const float beta = s_g.beta[j];
            floatx4 x = ef[n], y;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = i0 + r;
                const float g = n <= strip && i >= j ? decay(s_g, i, j) : 0.f;
                x[r] = half == 0 ? damp(a.scale * g, x[r]) : i > j ? damp(-g, x[r]) : 0.f;
                y[r] = half == 0 ? x[r] : damp(x[r], beta);
            }
            // rows of the transposes are columns here: four consecutive elements of one row each; of the others one at a time
            if (half == 0) {
                tET.put4(j, i0, x);
#pragma unroll
                for (int r = 0; r < 4; ++r) tE.put1(i0 + r, j, y[r]);
            } else {
                tFT.put4(j, i0, x);
#pragma unroll
                for (int r = 0; r < 4; ++r) tF.put1(i0 + r, j, y[r]);
            }
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float g = s_g.gam[i0 + r], en = s_g.end[i0 + r];
#pragma unroll
            for (int n = 0; n < NK; ++n) { dq[n][r] = damp(a.scale * g, dq[n][r]); ks[n][r] = damp(-g, ks[n][r]); ke[n][r] = damp(en, ke[n][r]); }
        }
        auto values = [&](const E* T, int n) {          // tokens i0 .. i0 + 3 of column 16 (n0 + n) + c
            const E* p = T + (KS * (n0 + n) + strip / 2) * 512 + (c + 16 * (2 * (strip & 1) + (q >> 1))) * 8 + 4 * (q & 1);
            floatx4 x;
            if constexpr (sizeof(E) == 4) {
                x = *(const floatx4*)p;
            } else {
                const bf16x4 h = *(const bf16x4*)p;
#pragma unroll
                for (int r = 0; r < 4; ++r) x[r] = (float)h[r];
            }
            return x;
        };
        floatx4 kv[NK], qv[NK];
#pragma unroll
        for (int n = 0; n < NK; ++n) { kv[n] = values(KT, n); qv[n] = values(QT, n); }
        __syncthreads();
        floatx4 ft[NK] = {};                // F^T K
        float ext = 0.f;
#pragma unroll
        for (int n = 0; n < NK; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r) ext += kv[n][r] * ke[n][r];   // before E^T Q joins it: the part of dG_last
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            if (k <= strip / 2) {           // E and F diag(beta): lower triangles
                const auto fe = tE.frag(row, 32 * k + 8 * q);
                const auto ff = tF.frag(row, 32 * k + 8 * q);
#pragma unroll
                for (int n = 0; n < NK; ++n) { mma(dq[n], fe, fk[n][k]); mma(ks[n], ff, fk[n][k]); }
            }
            if (k >= strip / 2) {
                const auto fe = tET.frag(row, 32 * k + 8 * q);
                const auto ff = tFT.frag(row, 32 * k + 8 * q);
#pragma unroll
                for (int n = 0; n < NK; ++n) { mma(ke[n], fe, fq[n][k]); mma(ft[n], ff, fk[n][k]); }
            }
        }
        settle();
        floatx4 kdot = {}, kft = {};
#pragma unroll
        for (int n = 0; n < NK; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                kft[r] += kv[n][r] * ft[n][r];
                const float rest = ke[n][r] + s_g.beta[i0 + r] * ft[n][r];
                kdot[r] += qv[n][r] * dq[n][r] + kv[n][r] * (ks[n][r] - rest);
                sum_q[n][r] = MANY ? sum_q[n][r] + dq[n][r] : dq[n][r];
                sum_k[n][r] = MANY ? sum_k[n][r] + ks[n][r] + rest : ks[n][r] + rest;
            }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float b = sum16(kft[r]), g = sum16(kdot[r]);
            if (c == 0) { s_dG[half][i0 + r] = g; s_b[half][i0 + r] = b; }
        }
        ext += damp(s_g.last, ss);
        ext = sum16(ext);
        ext += __shfl_xor(ext, 16);
        ext += __shfl_xor(ext, 32);
        if (l == 0) s_ext[wave] = ext;
        __syncthreads();
        if (wave == 0) {                    // sums from the end to each token, within its segment
            float x = l < C ? s_dG[0][l] + s_dG[1][l] : 0.f;
            if (l == C - 1)
#pragma unroll
                for (int i = 0; i < 2 * NW; ++i) x += s_ext[i];
            const int part = s_g.part[l];
            const bool reset = part != (l ? s_g.part[l - 1] : 0);       // a log decay that leaves nothing
#pragma unroll
            for (int d = 1; d < C; d *= 2) {
                const float o = __shfl_down(x, d);
                const int p = __shfl_down(part, d);
                if (l + d < C && p == part) x += o;
            }
            if (l < rows) {
                *at_out<float>(a.dg, w.b, t0 + l, w.h) = l < len && !reset ? x : 0.f;
                *at_out<float>(a.dbeta, w.b, t0 + l, w.h) = l < len ? s_yr[l] + s_b[0][l] + s_b[1][l] : 0.f;
            }
        }
    }
    const int c = threadIdx.x & 15, i0 = 16 * strip + ((threadIdx.x & 63) >> 4) * 4;
    w.h -= 1;                               // the head whose row of the partial sums this is (heads_wg = 1)
#pragma unroll
    for (int n = 0; n < NK; ++n) {
        const int d = 16 * (n0 + n) + c;
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (i0 + r < rows && d < dk) {
                const bool in = i0 + r < len;
                put(a.dq, a.part_q, i0 + r, d, in ? sum_q[n][r] : 0.f);
                put(a.dk, a.part_k, i0 + r, d, in ? sum_k[n][r] : 0.f);
            }
    }
}

// dq and dk of shared key heads: the sum over their value heads, in order.  5 sequences of up to 333 tokens: 5 us, a launch.
template <typename E>
__global__ __launch_bounds__(256) void delta_group_kernel(DeltaArgs a) {
    const int64_t all = (int64_t)a.batch * a.steps * a.heads_k * a.dim_k;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < 2 * all; i += (int64_t)gridDim.x * 256) {
        const bool second = i >= all;
        const int64_t j = second ? i - all : i;
        const int d = (int)(j % a.dim_k);
        const int64_t r = j / a.dim_k;      // (b, t, key head)
        const int h = (int)(r % a.heads_k);
        const int64_t bt = r / a.heads_k;
        const float* p = (second ? a.part_k : a.part_q) + (bt * a.heads_v + (int64_t)h * a.group) * a.dim_k + d;
        float x = p[0];
        for (int g = 1; g < a.group; ++g) x += p[(int64_t)g * a.dim_k];
        *(at_out<E>(second ? a.dk : a.dq, (int)(bt / a.steps), bt % a.steps, h) + d) = from_float<E>(x);
    }
}

// ---- launches -------------------------------------------------------------------------------
size_t up256(size_t x) { return (x + 255) / 256 * 256; }
struct Plan {                               // padded sizes, and where things lie in `saved` and the workspace
    int heads_wg;                           // value heads that one workgroup of delta_back_kernel takes: those of a key head where that fills the card
    int c, dkp, dvp, chunks;                // c: tokens per chunk
    bool narrow;
    size_t T, P, G, KT, KO, QO, forward;            // offsets in bytes; `forward`: what a call without `saved` needs
    size_t TT, PT, QT, R, S, saved;
    size_t dX, dY, dS, part_q, part_k, back;
};
bool shape_ok(const pql_delta_shape& s) {
    return s.batch >= 0 && s.steps >= 0 && s.heads_k >= 1 && s.heads_v >= 1 && s.heads_v % s.heads_k == 0 && s.dim_k >= 1 &&
           s.dim_k <= PQL_DELTA_MAX_DIM_K && s.dim_v >= 1 && s.dim_v <= PQL_DELTA_MAX_DIM_V && (s.dtype == PQL_F32 || s.dtype == PQL_BF16) &&
           s.scale == s.scale && s.steps <= (1 << 30) && s.heads_v <= 65535 && (int64_t)s.batch * s.heads_v <= 0x7fffffffLL / 256;
}
// Tokens per chunk, 32 or 64.  Chunks of 32 halve the work between tokens and let two to four workgroups share a CU; chunks of
// 64 halve the number of steps of a sequence, which is what bounds few and long ones, and with bf16 keys of 128 the gradient
// kernel moves the states of every chunk through LDS, which then takes longer than its products.  Measured with 32 and with 64
// tokens, us: forward, fp32, 64 x 64: 2048 sequences times heads of 32 tokens 66 and 123, 1024 of 256 198 and 246, 32 of 1024 65 and 59; bf16,
// 128 x 128: 256 of 128 51 and 57, 16 of 16384 690 and 533.  Forward and gradient, bf16, 128 x 128: 256 of 128 204
// and 170, 64 of 2048 815 and 579; few, 4 of 128, 49 and 58; fp32, 128 x 128: 256 of 256 465 and 477, 32 of 64 59 and 75.  Few and short,
// forward: fp32, 64 x 64: 1 of 64 13 and 19, 16 of 256 22 and 26, 32 of 512 34 and 37; bf16, 128 x 128: 1 of 64 14 and 17, 16 of 256 23 and 24, 32 of 512
// 37 and 35; just above, 16 of 1024: fp32 51 and 51, bf16 55 and 45.
int chunk_of(const pql_delta_shape& s, bool train) {
    const int64_t pairs = (int64_t)s.batch * s.heads_v;
    if (s.steps <= 32) return 32;
    if (train && s.dtype == PQL_BF16 && s.dim_k > 64) return s.steps <= 512 && pairs * s.steps <= 8192 ? 32 : 64;
    return s.steps <= 512 || pairs >= 256 ? 32 : 64;
}
Plan plan_of(const pql_delta_shape& s, bool train) {
    Plan p;
    p.dkp = s.dim_k <= 64 ? 64 : 128;
    p.dvp = (s.dim_v + 31) / 32 * 32;
    p.c = chunk_of(s, train);
    p.chunks = (s.steps + p.c - 1) / p.c;
    const size_t n = (size_t)s.batch * s.heads_v * p.chunks, nk = (size_t)s.batch * s.heads_k * p.chunks, es = s.dtype == PQL_F32 ? 4 : 2;
    const size_t tri = s.dtype == PQL_F32 ? (p.c == 32 ? TRI<ModeF, 32> : TRI<ModeF, 64>) * sizeof(float) : (p.c == 32 ? TRI<ModeB, 32> : TRI<ModeB, 64>) * sizeof(bf16_t);
    size_t o = 0;
    auto take = [&](size_t bytes) { const size_t at = o; o += up256(bytes); return at; };
    p.T = take(n * tri); p.P = take(n * tri); p.G = take(n * 4 * p.c * 4); p.KT = take(nk * p.dkp * p.c * es);
    // 16 columns of the state per workgroup instead of 32 while those are fewer than the card's CUs: a chunk's chain is
    // shorter then, and there are more of them.  Forward, sequences of 2048, 16 heads of 128 x 128, bf16, 16 and 32 columns: one
    // sequence (64 workgroups of 32) 66 and 102 us, four (256) 159 and 135 us.
    p.narrow = (int64_t)s.batch * s.heads_v * (p.dvp / 32) < 256;
    p.KO = take(p.narrow ? nk * p.dkp * p.c * es : 0); p.QO = take(p.narrow ? nk * p.dkp * p.c * es : 0);
    p.forward = o;
    p.TT = take(n * tri); p.PT = take(n * tri); p.QT = take(nk * p.dkp * p.c * es);
    p.R = take(n * p.c * p.dvp * 4); p.S = take(n * p.dkp * p.dvp * 4);
    p.saved = o;
    o = 0;
    p.dX = take(n * p.c * p.dvp * 4); p.dY = take(n * p.c * p.dvp * 4); p.dS = take(n * p.dkp * p.dvp * 4);
    // with all value heads of a key head and with one a workgroup, us: 128 x 128, 2 value heads a key head: 1024 workgroups 380
    // and 464, 256 131 and 156; 72 x 100: 90 108 and 74
    p.heads_wg = (int64_t)s.batch * s.heads_k * p.chunks < 256 ? 1 : s.heads_v / s.heads_k;
    const size_t part = s.heads_v == s.heads_k || p.heads_wg > 1 ? 0 : (size_t)s.batch * s.steps * s.heads_v * s.dim_k;
    p.part_q = take(part * 4); p.part_k = take(part * 4);
    p.back = o;
    return p;
}
DeltaSeq seq(const pql_seq& s) { return DeltaSeq{s.data, s.stride_b, s.stride_t, s.stride_h}; }
// Whether a chunk of tokens can be reached with 32-bit offsets, and whether, beyond that, 16 bytes of a row may be loaded at a time.
bool rows_near(const pql_seq& s) { return s.stride_t >= 0 && s.stride_t < (1 << 21); }
bool rows_aligned(const pql_seq& s, int dim, int dtype) {
    const int n = dtype == PQL_F32 ? 4 : 8;             // elements in 16 bytes
    return ((uintptr_t)s.data & 15) == 0 && s.stride_b % n == 0 && s.stride_t % n == 0 && s.stride_h % n == 0 && dim % n == 0 && rows_near(s);
}
// Elements of an output must not share a place: a stride of 0 is for inputs only.
bool apart(const pql_seq& s, const pql_delta_shape& x, int heads) {
    return (x.batch <= 1 || s.stride_b != 0) && (x.steps <= 1 || s.stride_t != 0) && (heads <= 1 || s.stride_h != 0);
}
DeltaArgs args_of(const pql_delta_shape& s, const pql_delta_input& in) {
    DeltaArgs a{};
    a.batch = s.batch; a.steps = s.steps; a.heads_k = s.heads_k; a.heads_v = s.heads_v; a.group = s.heads_v / s.heads_k;
    a.dim_k = s.dim_k; a.dim_v = s.dim_v; a.scale = s.scale;
    a.q = seq(in.q); a.k = seq(in.k); a.v = seq(in.v); a.g = seq(in.log_decay); a.beta = seq(in.beta);
    a.lengths = in.lengths; a.state = in.state;
    return a;
}
int32_t check_input(pql_ctx* c, const pql_delta_shape* s, const pql_delta_input* in, const char* shape_text, const char* null_text, const char* align_text) {
    if (!s || !in) return ctx_fail(c, PQL_ERR_NULL, null_text);
    if (!shape_ok(*s)) return ctx_fail(c, PQL_ERR_INVALID_ARG, shape_text);
    if (s->batch == 0) return PQL_OK;
    const unsigned es = s->dtype == PQL_F32 ? 4 : 2;
    if (s->steps > 0 && (!in->q.data || !in->k.data || !in->v.data || !in->log_decay.data || !in->beta.data)) return ctx_fail(c, PQL_ERR_NULL, null_text);
    if (((uintptr_t)in->q.data | (uintptr_t)in->k.data | (uintptr_t)in->v.data) & (es - 1)) return ctx_fail(c, PQL_ERR_ALIGNMENT, align_text);
    if ((((uintptr_t)in->log_decay.data | (uintptr_t)in->beta.data | (uintptr_t)in->lengths) & 3) || ((uintptr_t)in->state & 15))
        return ctx_fail(c, PQL_ERR_ALIGNMENT, align_text);
    return PQL_OK;
}

template <typename E, int LX, bool VEC> hipError_t step_launch(const DeltaArgs& a, hipStream_t st) {
    const double states = 8.0 * a.batch * a.heads_v * a.dim_k * a.dim_v;
    const double tokens = (double)a.batch * a.steps * (2.0 * a.heads_k * a.dim_k + 2.0 * a.heads_v * a.dim_v) * sizeof(E);
    const ProfSlot ps = prof_slot();
    PQL_LAUNCH(ps, (delta_step_kernel<E, LX, VEC>), dim3((unsigned)(a.batch * a.heads_v), (unsigned)((a.dim_v + 4 * LX - 1) / (4 * LX))), dim3(256), 0, st, a);
    prof_commit(ps, KID_DELTA_STEP, 6.0 * a.batch * a.steps * a.heads_v * a.dim_k * a.dim_v, states + tokens);
    return hipGetLastError();
}
template <typename E> hipError_t step_dispatch(const DeltaArgs& a, hipStream_t st) {
    const bool vec = a.dim_v % 4 == 0;
    if (a.dim_v <= 32) return vec ? step_launch<E, 8, true>(a, st) : step_launch<E, 8, false>(a, st);
    if (a.dim_v <= 64) return vec ? step_launch<E, 16, true>(a, st) : step_launch<E, 16, false>(a, st);
    return vec ? step_launch<E, 32, true>(a, st) : step_launch<E, 32, false>(a, st);
}

// blockIdx.y counts sequences times heads, at most 65535 a launch: batches are cut.
template <typename F> hipError_t by_batch(const DeltaArgs& a, F&& f) {
    const int most = 65535 / a.heads_v;
    for (int b = 0; b < a.batch; b += most) {
        DeltaArgs x = a;
        x.batch = a.batch - b < most ? a.batch - b : most;
        x.bh0 = b * a.heads_v;
        const hipError_t e = f(x);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
template <typename K> hipError_t launch(K kernel, LdsLimit& lim, size_t lds, dim3 grid, int threads, const DeltaArgs& a, int kid, double flops, double bytes, hipStream_t st) {
    if (lds > 32768) {
        const hipError_t e = set_lds_limit((const void*)kernel, lds, lim);
        if (e != hipSuccess) return e;
    }
    const ProfSlot ps = prof_slot();
    PQL_LAUNCH(ps, kernel, grid, dim3(threads), lds, st, a);
    prof_commit(ps, kid, flops, bytes);
    return hipGetLastError();
}
// Work of one token and value head that the chunked form cannot do without, and the token tensors' bytes.
double token_heads(const DeltaArgs& a) { return (double)a.batch * a.steps * a.heads_v; }
template <typename M, int C, int DK, bool AL> struct Chunked {
    static hipError_t forward(const DeltaArgs& all, hipStream_t st) {
        return by_batch(all, [&](const DeltaArgs& a) {
            static LdsLimit l_prep, lim[4];
            const double th = token_heads(a), es = sizeof(typename M::E);
            const double flops = th * (6.0 * a.dim_k + 4.0 * C) * a.dim_v, bytes = th * (es * (2 * a.dim_k + 2 * a.dim_v) + 8.0 * C);
            hipError_t e = hipSuccess;
            if (a.chunks > 0)
                e = launch(delta_prepare_kernel<M, C, DK, AL>, l_prep, prepare_lds(), dim3(a.chunks, a.batch * a.heads_v), 4 * C, a, KID_DELTA_PREPARE,
                           th * 4.0 * C * a.dim_k, th * (2 * es * a.dim_k + 8.0 * C), st);
            if (e != hipSuccess) return e;
            auto scan = [&](auto kernel, LdsLimit& lim, int nt, size_t lds) {
                return launch(kernel, lim, lds, dim3(a.dvp / (16 * nt) * a.batch * a.heads_v), 8 * C, a, KID_DELTA_SCAN, flops, bytes, st);
            };
            if (a.narrow) return a.S ? scan(delta_scan_kernel<M, C, DK, 1, AL, true>, lim[0], 1, ScanLds<M, C, DK, 1>::BYTES)
                                      : scan(delta_scan_kernel<M, C, DK, 1, AL, false>, lim[1], 1, ScanLds<M, C, DK, 1>::BYTES);
            return a.S ? scan(delta_scan_kernel<M, C, DK, 2, AL, true>, lim[2], 2, ScanLds<M, C, DK, 2>::BYTES)
                       : scan(delta_scan_kernel<M, C, DK, 2, AL, false>, lim[3], 2, ScanLds<M, C, DK, 2>::BYTES);
        });
    }
    static hipError_t backward(const DeltaArgs& all, hipStream_t st) {
        const hipError_t e = by_batch(all, [&](const DeltaArgs& a) {
            static LdsLimit l_scan, l_narrow, l_back[2];
            const double th = token_heads(a), es = sizeof(typename M::E);
            const double flops = th * (6.0 * a.dim_k + 4.0 * C) * a.dim_v, bytes = th * (es * (2 * a.dim_k + 2 * a.dim_v) + 8.0 * C + 8.0 * a.dim_v);
            hipError_t e = a.narrow ? launch(delta_back_scan_kernel<M, C, DK, 1, AL>, l_narrow, BackScanLds<M, C, DK, 1>::BYTES,
                                              dim3(a.dvp / 16 * a.batch * a.heads_v), 8 * C, a, KID_DELTA_BACK_SCAN, flops, bytes, st)
                                     : launch(delta_back_scan_kernel<M, C, DK, 2, AL>, l_scan, BackScanLds<M, C, DK, 2>::BYTES,
                                              dim3(a.dvp / 32 * a.batch * a.heads_v), 8 * C, a, KID_DELTA_BACK_SCAN, flops, bytes, st);
            if (e != hipSuccess || a.chunks == 0) return e;
            auto parallel = [&](auto kernel, LdsLimit& lim) {
                return launch(kernel, lim, BackLds<M, C, DK>::BYTES, dim3(a.chunks, a.batch * (a.heads_v / a.heads_wg)), 8 * C, a, KID_DELTA_BACK,
                              th * (6.0 * a.dim_k * a.dim_v + 4.0 * C * a.dim_v + 8.0 * C * a.dim_k), th * (es * (4 * a.dim_k + a.dim_v) + 12.0 * a.dim_v), st);
            };
            return a.heads_wg > 1 ? parallel(delta_back_kernel<M, C, DK, AL, true>, l_back[0]) : parallel(delta_back_kernel<M, C, DK, AL, false>, l_back[1]);
        });
        if (e != hipSuccess || all.part_q == nullptr || all.steps == 0) return e;
        const int64_t n = 2 * (int64_t)all.batch * all.steps * all.heads_k * all.dim_k;
        const int64_t blocks = (n + 255) / 256 < 4096 ? (n + 255) / 256 : 4096;
        const ProfSlot ps = prof_slot();
        PQL_LAUNCH(ps, delta_group_kernel<typename M::E>, dim3((unsigned)blocks), dim3(256), 0, st, all);
        prof_commit(ps, KID_DELTA_GROUP, 0.0, (double)n * (4.0 * all.group + sizeof(typename M::E)));
        return hipGetLastError();
    }
    static size_t prepare_lds() {
        const size_t m = 2 * sizeof(Matrix<C>), t = Tile<M, DK, C, true>::BYTES;
        return m > t ? m : t;
    }
    static hipError_t run(const DeltaArgs& a, bool back, hipStream_t st) { return back ? backward(a, st) : forward(a, st); }
};
template <typename M> hipError_t chunks_dispatch(const DeltaArgs& a, bool back, bool al, const Plan& p, hipStream_t st) {
    if (p.c == 32) {
        if (p.dkp == 64) return al ? Chunked<M, 32, 64, true>::run(a, back, st) : Chunked<M, 32, 64, false>::run(a, back, st);
        return al ? Chunked<M, 32, 128, true>::run(a, back, st) : Chunked<M, 32, 128, false>::run(a, back, st);
    }
    if (p.dkp == 64) return al ? Chunked<M, 64, 64, true>::run(a, back, st) : Chunked<M, 64, 64, false>::run(a, back, st);
    return al ? Chunked<M, 64, 128, true>::run(a, back, st) : Chunked<M, 64, 128, false>::run(a, back, st);
}
void set_saved(DeltaArgs& a, const Plan& p, char* base, bool keep) {
    a.chunks = p.chunks; a.dvp = p.dvp; a.narrow = p.narrow;
    a.T = base + p.T; a.P = base + p.P; a.G = (float*)(base + p.G); a.KT = base + p.KT; a.KO = base + p.KO; a.QO = base + p.QO;
    if (!keep) return;
    a.TT = base + p.TT; a.PT = base + p.PT; a.QT = base + p.QT;
    a.R = (float*)(base + p.R); a.S = (float*)(base + p.S);
}
}  // namespace
}  // namespace pql

using namespace pql;

extern "C" {

int32_t pql_delta_step(pql_ctx* c, const pql_delta_shape* s, const pql_delta_input* in, float* state_out, pql_seq out, void* stream) {
    if (!c) return PQL_ERR_NULL;
    const int32_t rc = check_input(c, s, in, "pql_delta_step: bad shape", "pql_delta_step: null pointer", "pql_delta_step: misaligned pointer");
    if (rc != PQL_OK || s->batch == 0) return rc;
    if (!state_out || (!out.data && s->steps > 0)) return ctx_fail(c, PQL_ERR_NULL, "pql_delta_step: null pointer");
    if (!apart(out, *s, s->heads_v)) return ctx_fail(c, PQL_ERR_INVALID_ARG, "pql_delta_step: outputs share memory (stride 0)");
    if (((uintptr_t)state_out & 15) || ((uintptr_t)out.data & (s->dtype == PQL_F32 ? 3 : 1)))
        return ctx_fail(c, PQL_ERR_ALIGNMENT, "pql_delta_step: misaligned pointer");
    DeltaArgs a = args_of(*s, *in);
    a.out = seq(out); a.state_out = state_out;
    const hipError_t e = s->dtype == PQL_F32 ? step_dispatch<float>(a, (hipStream_t)stream) : step_dispatch<bf16_t>(a, (hipStream_t)stream);
    return e == hipSuccess ? PQL_OK : ctx_fail(c, PQL_ERR_HIP, "pql_delta_step", e);
}

int64_t pql_delta_saved_bytes(const pql_delta_shape* s) {
    if (!s) return PQL_ERR_NULL;
    return shape_ok(*s) ? (int64_t)plan_of(*s, true).saved : PQL_ERR_INVALID_ARG;
}
int64_t pql_delta_workspace_bytes(const pql_delta_shape* s, int32_t backward) {
    if (!s) return PQL_ERR_NULL;
    if (!shape_ok(*s)) return PQL_ERR_INVALID_ARG;
    const size_t forward = plan_of(*s, false).forward, back = plan_of(*s, true).back;
    return (int64_t)(backward && back > forward ? back : forward);
}

int32_t pql_delta_forward(pql_ctx* c, const pql_delta_shape* s, const pql_delta_input* in, pql_seq out, float* state_out, void* saved,
                          void* workspace, void* stream) {
    if (!c) return PQL_ERR_NULL;
    const int32_t rc = check_input(c, s, in, "pql_delta_forward: bad shape", "pql_delta_forward: null pointer", "pql_delta_forward: misaligned pointer");
    if (rc != PQL_OK || s->batch == 0) return rc;
    if (s->steps > 0 && (!out.data || (!saved && !workspace))) return ctx_fail(c, PQL_ERR_NULL, "pql_delta_forward: null pointer");
    if (!apart(out, *s, s->heads_v)) return ctx_fail(c, PQL_ERR_INVALID_ARG, "pql_delta_forward: outputs share memory (stride 0)");
    if (((uintptr_t)state_out & 15) || ((uintptr_t)out.data & (s->dtype == PQL_F32 ? 3 : 1)) || ((uintptr_t)saved & 255) || ((uintptr_t)workspace & 255))
        return ctx_fail(c, PQL_ERR_ALIGNMENT, "pql_delta_forward: misaligned pointer");
    const Plan p = plan_of(*s, saved != nullptr);
    DeltaArgs a = args_of(*s, *in);
    a.out = seq(out); a.state_out = state_out;
    set_saved(a, p, (char*)(saved ? saved : workspace), saved != nullptr);
    const bool al = rows_aligned(in->q, s->dim_k, s->dtype) && rows_aligned(in->k, s->dim_k, s->dtype) && rows_near(in->v) && rows_near(out);
    const hipError_t e = s->dtype == PQL_F32 ? chunks_dispatch<ModeF>(a, false, al, p, (hipStream_t)stream)
                                             : chunks_dispatch<ModeB>(a, false, al, p, (hipStream_t)stream);
    return e == hipSuccess ? PQL_OK : ctx_fail(c, PQL_ERR_HIP, "pql_delta_forward", e);
}

int32_t pql_delta_backward(pql_ctx* c, const pql_delta_shape* s, const pql_delta_input* in, const void* saved, pql_seq out_grad,
                           const float* state_out_grad, const pql_delta_grad* g, void* workspace, void* stream) {
    if (!c) return PQL_ERR_NULL;
    const int32_t rc = check_input(c, s, in, "pql_delta_backward: bad shape", "pql_delta_backward: null pointer", "pql_delta_backward: misaligned pointer");
    if (rc != PQL_OK || (s->batch == 0 && g)) return rc;
    if (!g || (s->steps > 0 && (!saved || !workspace || !out_grad.data || !g->q.data || !g->k.data || !g->v.data || !g->log_decay.data || !g->beta.data)))
        return ctx_fail(c, PQL_ERR_NULL, "pql_delta_backward: null pointer");
    if (!apart(g->q, *s, s->heads_k) || !apart(g->k, *s, s->heads_k) || !apart(g->v, *s, s->heads_v) ||
        !apart(g->log_decay, *s, s->heads_v) || !apart(g->beta, *s, s->heads_v))
        return ctx_fail(c, PQL_ERR_INVALID_ARG, "pql_delta_backward: gradients share memory (stride 0)");
    const unsigned es = s->dtype == PQL_F32 ? 4 : 2;
    if ((((uintptr_t)out_grad.data | (uintptr_t)g->q.data | (uintptr_t)g->k.data | (uintptr_t)g->v.data) & (es - 1)) ||
        (((uintptr_t)g->log_decay.data | (uintptr_t)g->beta.data) & 3) || (((uintptr_t)state_out_grad | (uintptr_t)g->state) & 15) ||
        (((uintptr_t)saved | (uintptr_t)workspace) & 255))
        return ctx_fail(c, PQL_ERR_ALIGNMENT, "pql_delta_backward: misaligned pointer");
    const Plan p = plan_of(*s, true);
    DeltaArgs a = args_of(*s, *in);
    set_saved(a, p, (char*)saved, true);
    char* w = (char*)workspace;
    a.out_grad = seq(out_grad); a.state_grad = state_out_grad;
    a.dq = seq(g->q); a.dk = seq(g->k); a.dv = seq(g->v); a.dg = seq(g->log_decay); a.dbeta = seq(g->beta); a.dstate = g->state;
    a.dX = (float*)(w + p.dX); a.dY = (float*)(w + p.dY); a.dS = (float*)(w + p.dS);
    a.heads_wg = p.heads_wg;
    if (a.group > 1 && p.heads_wg == 1) { a.part_q = (float*)(w + p.part_q); a.part_k = (float*)(w + p.part_k); }
    const bool al = rows_aligned(in->q, s->dim_k, s->dtype) && rows_aligned(in->k, s->dim_k, s->dtype) && rows_aligned(out_grad, s->dim_v, s->dtype) && rows_near(g->v);
    const hipError_t e = s->dtype == PQL_F32 ? chunks_dispatch<ModeF>(a, true, al, p, (hipStream_t)stream)
                                             : chunks_dispatch<ModeB>(a, true, al, p, (hipStream_t)stream);
    return e == hipSuccess ? PQL_OK : ctx_fail(c, PQL_ERR_HIP, "pql_delta_backward", e);
}

}  // extern "C"
