// Operators on rows of logits (include/pql_student.h): a teacher's largest logits of every row, and the
// distillation loss against such lists with its gradient.  All of them are bound by reading the logits once and, where
// there is a gradient, writing it once; everything else is arranged around that.
//
// Rows of at most SMALL_VOCAB logits are held by a group of 8 to 64 lanes of one wavefront, one element per lane and
// register, so that a wavefront works on up to eight rows and its reductions take three to six steps.  Longer rows have
// a workgroup each, which reads 16 bytes per lane and keeps the row in registers between the two uses; few long rows are
// cut into pieces, joined by a second launch through the workspace.
#include "pql_student_internal.h"

namespace pql {
namespace {

constexpr int SMALL_VOCAB = 1024;
constexpr float LOG2E = 1.4426950408889634f;
constexpr float NEG_INF = -__builtin_inff();

// The gradient by itself takes q = exp(z / t - lse) from the one number a row's caller keeps, which is rounded three times on its way: up to
// 2e-7 |lse| of every q.  Beyond this bound (6e-6) rows work out their maximum and sum again, as the loss does.
constexpr float FAR = 32.f;

// 2^x by the one instruction: results below 2^-126 become 0, which no sum or gradient here can tell from their value.
__device__ __forceinline__ float exp2_raw(float x) { return __builtin_amdgcn_exp2f(x); }

// ---- reductions -----------------------------------------------------------------------------
// Lane i gets the value of the lane that differs in one bit of the number; below 16 as a modifier of the instruction that
// uses it (mirrors instead of the bits 4 and 8: lanes of one half hold equal values by then), above through the LDS crossbar.
template <int D> __device__ __forceinline__ int other(int x) {
    if constexpr (D == 1) return __builtin_amdgcn_update_dpp(x, x, 0xB1, 0xf, 0xf, false);
    else if constexpr (D == 2) return __builtin_amdgcn_update_dpp(x, x, 0x4E, 0xf, 0xf, false);
    else if constexpr (D == 4) return __builtin_amdgcn_update_dpp(x, x, 0x141, 0xf, 0xf, false);
    else if constexpr (D == 8) return __builtin_amdgcn_update_dpp(x, x, 0x140, 0xf, 0xf, false);
    else return __shfl_xor(x, D);
}
template <int D> __device__ __forceinline__ float other(float x) { return __int_as_float(other<D>(__float_as_int(x))); }
template <int D> __device__ __forceinline__ unsigned other(unsigned x) { return (unsigned)other<D>((int)x); }
template <int G, int D = 1, typename V, typename F> __device__ __forceinline__ V group_reduce(V x, F f) {
    if constexpr (D < G) return group_reduce<G, 2 * D>(f(x, other<D>(x)), f);
    else return x;
}
template <int G> __device__ __forceinline__ float group_max(float x) { return group_reduce<G>(x, [](float a, float b) { return fmaxf(a, b); }); }
template <int G> __device__ __forceinline__ unsigned group_max(unsigned x) { return group_reduce<G>(x, [](unsigned a, unsigned b) { return a > b ? a : b; }); }
template <int G> __device__ __forceinline__ int group_min(int x) { return group_reduce<G>(x, [](int a, int b) { return a < b ? a : b; }); }
template <int G, typename V> __device__ __forceinline__ V group_sum(V x) { return group_reduce<G>(x, [](V a, V b) { return a + b; }); }
// Over a workgroup of NT threads; every thread gets the result.  `s` holds NT / 64 values and may be used again after the
// next barrier (each call begins with one).
template <int NT> __device__ __forceinline__ float block_max(float x, float* s) {
    x = group_max<64>(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = x;
    __syncthreads();
    x = s[0];
#pragma unroll
    for (int i = 1; i < NT / 64; ++i) x = fmaxf(x, s[i]);
    return x;
}
template <int NT, typename V> __device__ __forceinline__ V block_sum(V x, V* s) {
    x = group_sum<64>(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = x;
    __syncthreads();
    x = s[0];
#pragma unroll
    for (int i = 1; i < NT / 64; ++i) x += s[i];
    return x;
}

// ---- a stretch of one row, read 16 bytes per lane --------------------------------------------
// Elements [0, len) at p, of any alignment: `head` elements up to the first 16-byte boundary, `vecs` granules of VEC
// elements, `tail` elements.  Head and tail together are fewer than 2 * VEC <= 16, one for each of the first threads.
template <typename E> struct Stretch {
    static constexpr int VEC = 16 / (int)sizeof(E);
    const E* p;
    int len, head, vecs, tail;
    __device__ __forceinline__ Stretch(const E* q, int n) : p(q), len(n) {
        const int to = (int)((16 - ((uintptr_t)q & 15)) & 15) / (int)sizeof(E);
        head = to < n ? to : n;
        vecs = (n - head) / VEC;
        tail = n - head - vecs * VEC;
    }
    // the place of this thread's single element, or -1
    __device__ __forceinline__ int single(int t) const {
        return t < head ? t : t < head + tail ? len - tail + (t - head) : -1;
    }
    __device__ __forceinline__ int place(int v) const { return head + v * VEC; }
    __device__ __forceinline__ uint4 granule(int v) const { return *(const uint4*)(p + place(v)); }
};
template <typename E> __device__ __forceinline__ void unpack(uint4 g, float* x);
template <> __device__ __forceinline__ void unpack<float>(uint4 g, float* x) {
    x[0] = __uint_as_float(g.x); x[1] = __uint_as_float(g.y); x[2] = __uint_as_float(g.z); x[3] = __uint_as_float(g.w);
}
template <> __device__ __forceinline__ void unpack<bf16_t>(uint4 g, float* x) {
    const unsigned u[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(u[i] << 16); x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
}
// A stretch held in registers, NV granules and at most one single element per thread of NT; what lies behind it is -inf.
template <typename E, int NT, int NV> struct Held {
    static constexpr int VEC = Stretch<E>::VEC;
    uint4 g[NV];
    float one;
    int at;                                 // place of the single element, or -1
    __device__ __forceinline__ explicit Held(const Stretch<E>& st, int t = threadIdx.x) {
        const unsigned low = sizeof(E) == 4 ? 0xff800000u : 0xff80ff80u;
        at = st.single(t);
        one = at >= 0 ? to_float(st.p[at]) : NEG_INF;
        // all requests go out together: places behind the end read the last granule, and are overwritten
        if (st.vecs == 0) {
#pragma unroll
            for (int i = 0; i < NV; ++i) g[i] = make_uint4(low, low, low, low);
            return;
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) g[i] = st.granule(min(t + i * NT, st.vecs - 1));
        if (st.vecs < NT * NV) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (t + i * NT >= st.vecs) g[i] = make_uint4(low, low, low, low);
        }
    }
    // The granule's values.  Taken apart anew at every use: kept, the values of 16-bit granules would need twice the registers.
    __device__ __forceinline__ void values(int i, float* x) {
        if (sizeof(E) == 2) asm volatile("" : "+v"(g[i].x), "+v"(g[i].y), "+v"(g[i].z), "+v"(g[i].w));
        unpack<E>(g[i], x);
    }
    template <typename F> __device__ __forceinline__ void each(F&& f) {       // f(value, its place in the granule)
        f(one, 0);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float x[VEC];
            values(i, x);
#pragma unroll
            for (int j = 0; j < VEC; ++j) f(x[j], j);
        }
    }
};
// Packed by hand: written as elements in both branches, the two become one that stores them singly.
__device__ __forceinline__ unsigned pack2(float x, float y) {
    typedef float f2 __attribute__((ext_vector_type(2)));
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(unsigned, __builtin_convertvector((f2{x, y}), b2));
}
template <typename E> __device__ __forceinline__ void store_granule(E* p, bool aligned, const float* x) {
    uint4 u;
    if constexpr (sizeof(E) == 4) u = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    else u = make_uint4(pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7]));
    if (aligned) {
        *(uint4*)p = u;
        return;
    }
    const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(E) == 4) {
            ((unsigned*)p)[i] = w[i];
        } else {
            ((unsigned short*)p)[2 * i] = (unsigned short)w[i];
            ((unsigned short*)p)[2 * i + 1] = (unsigned short)(w[i] >> 16);
        }
    }
}

// ---- the teacher's list ------------------------------------------------------------------------
// p_k = softmax of the valid entries' values / t, by the first `top` threads of a workgroup.  Entries of one answer are
// added up at the first of them, in the order of the list: `sum` is the whole mass of this thread's answer if it is that
// first entry (`owner`).
struct Entry { int index; float y, p, log_p, sum; bool owner; };
// What of a row's list and weight this thread holds: requested together, one wait.
__device__ __forceinline__ float entry_of(const DistillArgs& a, int64_t n, Entry& e) {
    const int k = threadIdx.x;
    int i = -1;
    float y = NEG_INF;
    if (k < a.top) { i = a.index[n * a.top + k]; y = a.value[n * a.top + k]; }
    const float w = a.weight ? a.weight[n] : 1.f;
    const bool ok = (unsigned)i < (unsigned)a.vocab && y != NEG_INF;
    e.index = ok ? i : -1;
    e.y = ok ? y : NEG_INF;
    return w;
}
// The mass of one answer, entry k's, over a list that is padded with -1 to a multiple of four; whether k is its first entry.
// No early end: the reads of the whole list are then on their way together.
__device__ __forceinline__ void sum_of_answer(const int* s_index, const float* s_p, int top, int k, int index, bool& owner, float& sum) {
    owner = true;
    sum = 0.f;
#pragma unroll 4
    for (int i = 0; i < top; i += 4) {
        const int4 j = *(const int4*)(s_index + i);
        const float4 p = *(const float4*)(s_p + i);
        owner = owner && !((j.x == index && i < k) || (j.y == index && i + 1 < k) || (j.z == index && i + 2 < k) || (j.w == index && i + 3 < k));
        sum += j.x == index ? p.x : 0.f;
        sum += j.y == index ? p.y : 0.f;
        sum += j.z == index ? p.z : 0.f;
        sum += j.w == index ? p.w : 0.f;
    }
}
template <int NT>
__device__ __forceinline__ void entry_masses(const DistillArgs& a, Entry& e, int* s_index, float* s_p, float* s_red) {      // the sums only where there is a gradient
    const int k = threadIdx.x;
    e.p = 0.f; e.log_p = 0.f; e.sum = 0.f; e.owner = false;
    const float big = block_max<NT>(e.y, s_red);
    const float x = (e.y - (big == NEG_INF ? 0.f : big)) * a.inv_temp, m = e.index >= 0 ? expf(x) : 0.f;
    const float total = block_sum<NT>(m, s_red);
    if (e.index >= 0) { e.p = m / total; e.log_p = x - logf(total); }
    if (!a.grad) return;
    if (k < PQL_MAX_TOP) { s_index[k] = e.index; s_p[k] = e.p; }     // -1 behind the list
    __syncthreads();
    if (e.index >= 0) sum_of_answer(s_index, s_p, a.top, k, e.index, e.owner, e.sum);
}
// One entry's share of the loss: p (log p - log q) with log q = (z - m) / t - log(s); nothing for p = 0, +inf where the
// student has the answer at -inf (also in a row that holds nothing else).
__device__ __forceinline__ float entry_loss(const Entry& e, float z, float m, float inv_temp, float log_s) {
    return e.p == 0.f ? 0.f : z == NEG_INF ? -NEG_INF : e.p * (e.log_p - ((z - m) * inv_temp - log_s));
}

// =============================================================================================
// Small vocabularies: a group of G lanes per row, which it reads once and holds; bound by memory.  327680 rows of 51, fp32, lists
// of 8, loss and gradient: 45 us, 3.5 TB/s (34 us where the caches hold them); loss and gradient in calls of their own 29 and 31 us.
// =============================================================================================
template <typename E, int G, int R, bool BACK>
__global__ __launch_bounds__(256) void distill_small_kernel(DistillArgs a) {
    constexpr int ROWS = 256 / G;
    extern __shared__ float lds[];
    const int g = threadIdx.x / G, l = threadIdx.x & (G - 1);
    float* s_p = lds + (size_t)g * (2 * a.top);             // the list's masses, then its indices
    int* s_index = (int*)(s_p + a.top);
    float* s_t = lds + (size_t)ROWS * 2 * a.top + (size_t)g * a.vocab;      // target mass of every answer
    const int64_t n = (int64_t)blockIdx.x * ROWS + g;
    const bool in = n < a.rows;
    const float w = !in ? 0.f : a.weight ? a.weight[n] : 1.f;
    float big = NEG_INF;
    int valid = 0;
    for (int k = l; k < a.top; k += G) {
        const int i = in ? a.index[n * a.top + k] : -1;
        const float y = (unsigned)i < (unsigned)a.vocab ? a.value[n * a.top + k] : NEG_INF;
        const bool ok = y != NEG_INF;
        s_index[k] = ok ? i : -1;
        s_p[k] = y;
        valid |= ok;
        big = fmaxf(big, y);
    }
    big = group_max<G>(big);
    const bool read = w != 0.f && group_sum<G>(valid) != 0;
    float z[R];
    const E* row = (const E*)a.z + n * a.stride;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int j = l + G * r;
        z[r] = read && j < a.vocab ? to_float(row[j]) : NEG_INF;
        if (j < a.vocab) s_t[j] = 0.f;
    }
    const float shift = big == NEG_INF ? 0.f : big;
    float total = 0.f;
    for (int k = l; k < a.top; k += G) total += s_index[k] >= 0 ? expf((s_p[k] - shift) * a.inv_temp) : 0.f;
    total = group_sum<G>(total);
    const float log_total = logf(total);
    float plogp = 0.f;
    for (int k = l; k < a.top; k += G) {
        if (s_index[k] < 0) continue;
        const float x = (s_p[k] - shift) * a.inv_temp, p = expf(x) / total;
        if (p != 0.f) plogp += p * (x - log_total);
        s_p[k] = p;
    }
    __syncthreads();
    for (int k = l; k < a.top; k += G) {                    // entries of one answer are added in the list's order
        const int i = s_index[k];
        if (i < 0) continue;
        float sum = 0.f;
        bool owner = true;
#pragma unroll 8
        for (int q = 0; q < a.top; ++q) {
            const bool same = s_index[q] == i;
            owner = owner && !(same && q < k);
            sum += same ? s_p[q] : 0.f;
        }
        if (owner) s_t[i] = sum;
    }
    __syncthreads();
    const float c = LOG2E * a.inv_temp;
    float m = BACK && read ? a.lse[n] : 0.f, t_m = a.temp, inv = 1.f;      // q = exp((z - m t_m) / t) inv
    const bool stats = !BACK || __any(fabsf(m) > FAR);      // -inf among them
    if (stats) {
        m = z[0];
#pragma unroll
        for (int r = 1; r < R; ++r) m = fmaxf(m, z[r]);
        m = group_max<G>(m);
        if (m == NEG_INF) m = 0.f;
        t_m = 1.f;
    }
    float s = 0.f, q[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        q[r] = exp2_raw(fmaf(-m, t_m, z[r]) * c);
        s += q[r];
    }
    if (stats) {
        s = group_sum<G>(s);
        inv = s > 0.f || s != s ? 1.f / s : 0.f;
    }
    if (!BACK) {
        const float log_s = logf(s);
        float loss = plogp;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int j = l + G * r;
            const float t = j < a.vocab ? s_t[j] : 0.f;
            if (t != 0.f) loss -= z[r] == NEG_INF ? NEG_INF : t * ((z[r] - m) * a.inv_temp - log_s);
        }
        loss = group_sum<G>(loss);
        if (l == 0 && in) {
            a.loss_out[n] = read ? w * a.temp * a.temp * loss : 0.f;
            a.lse_out[n] = read ? m * a.inv_temp + log_s : 0.f;
        }
    }
    if (a.grad == nullptr || !in) return;
    E* out = (E*)a.grad + n * a.grad_stride;
    const float f = w * a.temp;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int j = l + G * r;
        if (j < a.vocab) out[j] = from_float<E>(read ? f * ((inv > 0.f || inv != inv ? q[r] * inv : 0.f) - s_t[j]) : 0.f);
    }
}

// =============================================================================================
// Rows of up to 64 NV granules: one wavefront per row, the row in its registers.  A workgroup per row would spend more time
// in barriers and waiting for its own first loads than on the row (65536 rows of 1500 bf16, loss and gradient: 121 and 263 us).
// =============================================================================================
__device__ __forceinline__ void wave_fence() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); __builtin_amdgcn_wave_barrier(); }

template <typename E, int NV, bool BACK>
__global__ __launch_bounds__(256) void distill_wave_kernel(DistillArgs a) {
    constexpr int VEC = Stretch<E>::VEC, Q = PQL_MAX_TOP / 64;
    __shared__ __align__(16) int s_index_all[4][PQL_MAX_TOP];
    __shared__ __align__(16) float s_p_all[4][PQL_MAX_TOP];
    const int wave = threadIdx.x >> 6, l = threadIdx.x & 63;
    const int64_t n = (int64_t)blockIdx.x * 4 + wave;
    if (n >= a.rows) return;                // wavefronts share nothing
    int* s_index = s_index_all[wave];
    float* s_p = s_p_all[wave];
    int index[Q];
    float y[Q], zk[Q] = {}, sum[Q] = {}, big = NEG_INF;
    const float w = a.weight ? a.weight[n] : 1.f;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        const int k = l + 64 * q;
        index[q] = -1; y[q] = NEG_INF;
        if (k < a.top) { index[q] = a.index[n * a.top + k]; y[q] = a.value[n * a.top + k]; }
    }
    bool some = false;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        const bool ok = (unsigned)index[q] < (unsigned)a.vocab && y[q] != NEG_INF;
        if (!ok) { index[q] = -1; y[q] = NEG_INF; }
        some |= ok;
        big = fmaxf(big, y[q]);
    }
    E* out = (E*)a.grad + n * a.grad_stride;
    if (!__any(some) || w == 0.f) {
        if (!BACK && l == 0) { a.loss_out[n] = 0.f; a.lse_out[n] = 0.f; }
        if (a.grad) for (int j = l; j < a.vocab; j += 64) out[j] = from_float<E>(0.f);
        return;
    }
    const E* row = (const E*)a.z + n * a.stride;
    const Stretch<E> st(row, a.vocab);
    Held<E, 64, NV> h(st, l);
#pragma unroll
    for (int q = 0; q < Q; ++q) if (index[q] >= 0) zk[q] = to_float(row[index[q]]);
    const float lse = BACK ? a.lse[n] : 0.f;
    // the list's masses; entries of one answer are added up at the first of them, in the order of the list
    big = group_max<64>(big);
    if (big == NEG_INF) big = 0.f;
    float total = 0.f;
#pragma unroll
    for (int q = 0; q < Q; ++q) total += index[q] >= 0 ? expf((y[q] - big) * a.inv_temp) : 0.f;
    total = group_sum<64>(total);
    const float log_total = logf(total);
    bool owner[Q];
    float lp[Q];                            // log p
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        const int k = l + 64 * q;
        const float x = (y[q] - big) * a.inv_temp;
        lp[q] = x - log_total;
        owner[q] = index[q] >= 0;
        y[q] = owner[q] ? expf(x) / total : 0.f;                     // p from here on
        if (64 * q < a.top) { s_index[k] = index[q]; s_p[k] = y[q]; }      // -1 behind the list
    }
    wave_fence();
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        if (64 * q >= a.top) break;
        bool first;
        sum_of_answer(s_index, s_p, a.top, l + 64 * q, index[q], first, sum[q]);
        owner[q] = owner[q] && first;
    }
    const float c = LOG2E * a.inv_temp;
    float m = lse, inv = 1.f, t_m = a.temp;
    if (!BACK || fabsf(lse) > FAR) {
        t_m = 1.f;
        m = NEG_INF;
        h.each([&](float x, int) { m = fmaxf(m, x); });
        m = group_max<64>(m);
        if (m == NEG_INF) m = 0.f;
        float part[4] = {};
        h.each([&](float x, int j) { part[j & 3] += exp2_raw((x - m) * c); });
        const float s = group_sum<64>((part[0] + part[1]) + (part[2] + part[3])), log_s = logf(s);
        inv = s > 0.f || s != s ? 1.f / s : 0.f;
        if (!BACK) {
            float loss = 0.f;
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                Entry e;
                e.p = y[q];
                e.log_p = lp[q];
                if (index[q] >= 0) loss += entry_loss(e, zk[q], m, a.inv_temp, log_s);
            }
            loss = group_sum<64>(loss);
            if (l == 0) {
                a.loss_out[n] = w * a.temp * a.temp * loss;
                a.lse_out[n] = m * a.inv_temp + log_s;
            }
            if (!a.grad) return;
        }
    }
#pragma unroll
    for (int q = 0; q < Q; ++q) asm volatile("" ::"v"(zk[q]));       // they are there before the gradient may be written over them
    const float f = w * a.temp, fi = f * inv;
    const bool aligned = (((uintptr_t)(out + st.head)) & 15) == 0;
    if (h.at >= 0) out[h.at] = from_float<E>(exp2_raw(fmaf(-m, t_m, h.one) * c) * fi);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int v = l + i * 64;
        if (v >= st.vecs) break;
        float x[VEC];
        h.values(i, x);
#pragma unroll
        for (int j = 0; j < VEC; ++j) x[j] = exp2_raw(fmaf(-m, t_m, x[j]) * c) * fi;
        store_granule<E>(out + st.place(v), aligned, x);
    }
    wave_fence();                           // the dense gradient of the listed answers lies before its correction
#pragma unroll
    for (int q = 0; q < Q; ++q)
        if (owner[q]) out[index[q]] = from_float<E>(f * ((inv != 0.f ? exp2_raw(fmaf(-m, t_m, zk[q]) * c) * inv : 0.f) - sum[q]));
}

// =============================================================================================
// Long rows.  A piece is a stretch of a row; one workgroup per piece.
// =============================================================================================
// Running maximum and sum of exp((z - m) c) over a stretch, of this thread's elements.
template <typename E, int NT>
__device__ __forceinline__ void stretch_stats(const Stretch<E>& st, float c, float& m, float& s) {
    constexpr int VEC = Stretch<E>::VEC, UNROLL = 4;
    m = NEG_INF; s = 0.f;
    const int t = threadIdx.x;
    const int one = st.single(t);
    if (one >= 0) { m = to_float(st.p[one]); s = m == NEG_INF ? 0.f : 1.f; }
    int v = t;
    for (; v < st.vecs; v += UNROLL * NT) {
        uint4 g[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) if (v + u * NT < st.vecs) g[u] = st.granule(v + u * NT);
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            if (v + u * NT >= st.vecs) break;
            float x[VEC], b = m;
            unpack<E>(g[u], x);
#pragma unroll
            for (int i = 0; i < VEC; ++i) b = fmaxf(b, x[i]);
            const float ref = b == NEG_INF ? 0.f : b;
            s *= exp2_raw((m - ref) * c);
#pragma unroll
            for (int i = 0; i < VEC; ++i) s += exp2_raw((x[i] - ref) * c);
            m = b;
        }
    }
}
// The same joined over the workgroup; m is 0 where the stretch holds nothing but -inf (and s = 0).
template <int NT> __device__ __forceinline__ void join_stats(float c, float& m, float& s, float* s_red) {
    const float b = block_max<NT>(m, s_red), ref = b == NEG_INF ? 0.f : b;
    s *= exp2_raw((m - ref) * c);
    if (m == NEG_INF) s = s != s ? s : 0.f;
    s = block_sum<NT>(s, s_red);
    m = ref;
}
// Gradient of a stretch: f * exp2((z - m t) c) * inv for every element, the listed answers patched afterwards.  m t is
// the row's maximum (t = 1), or the log-sum-exp times the temperature: one rounding of a difference that is small where
// the result is not.
template <typename E, int NT>
__device__ __forceinline__ void stretch_grad(const Stretch<E>& st, E* out, float c, float m, float t_m, float inv, float f) {
    constexpr int VEC = Stretch<E>::VEC, UNROLL = 4;
    const int t = threadIdx.x;
    const float fi = f * inv;
    const bool aligned = (((uintptr_t)(out + st.head)) & 15) == 0;
    const int one = st.single(t);
    if (one >= 0) out[one] = from_float<E>(exp2_raw(fmaf(-m, t_m, to_float(st.p[one])) * c) * fi);
    for (int v = t; v < st.vecs; v += UNROLL * NT) {
        uint4 g[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) if (v + u * NT < st.vecs) g[u] = st.granule(v + u * NT);
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            if (v + u * NT >= st.vecs) break;
            float x[VEC];
            unpack<E>(g[u], x);
#pragma unroll
            for (int i = 0; i < VEC; ++i) x[i] = exp2_raw(fmaf(-m, t_m, x[i]) * c) * fi;
            store_granule<E>(out + st.place(v + u * NT), aligned, x);
        }
    }
}
template <typename E, int NT> __device__ __forceinline__ void zero_stretch(E* out, int len) {
    for (int j = threadIdx.x; j < len; j += NT) out[j] = from_float<E>(0.f);
}

// One workgroup per row; bound by memory: 4096 rows of 65536, bf16, lists of 64, loss and gradient 201 us, 5.3 TB/s; loss
// alone 130 us.  NV > 0: the row stays in registers between its statistics and its gradient, NV granules a thread;
// NV = 0, rows that do not fit: it is read again.
template <typename E, int NT, int NV>
__global__ __launch_bounds__(NT) void distill_row_kernel(DistillArgs a) {
    constexpr int VEC = Stretch<E>::VEC;
    __shared__ __align__(16) int s_index[PQL_MAX_TOP];
    __shared__ __align__(16) float s_p[PQL_MAX_TOP], s_red[NT / 64];
    const int64_t n = blockIdx.x;
    E* out = (E*)a.grad + n * a.grad_stride;
    const E* row = (const E*)a.z + n * a.stride;
    Entry e;
    const float w = entry_of(a, n, e);
    if (!__syncthreads_or(e.index >= 0) || w == 0.f) {
        if (threadIdx.x == 0) { a.loss_out[n] = 0.f; a.lse_out[n] = 0.f; }
        if (a.grad) zero_stretch<E, NT>(out, a.vocab);
        return;
    }
    const Stretch<E> st(row, a.vocab);
    const float c = LOG2E * a.inv_temp;
    const float zk = e.index >= 0 ? to_float(row[e.index]) : 0.f;
    float m, s;
    if constexpr (NV > 0) {
        Held<E, NT, NV> h(st);              // on its way while the list is worked out
        entry_masses<NT>(a, e, s_index, s_p, s_red);
        m = NEG_INF;
        h.each([&](float x, int) { m = fmaxf(m, x); });
        m = block_max<NT>(m, s_red);
        if (m == NEG_INF) m = 0.f;
        float part[4] = {};                 // four sums: one would wait for itself
        h.each([&](float x, int j) { part[j & 3] += exp2_raw((x - m) * c); });
        s = block_sum<NT>((part[0] + part[1]) + (part[2] + part[3]), s_red);
        const float log_s = logf(s), inv = s > 0.f || s != s ? 1.f / s : 0.f;
        const float loss = block_sum<NT>(e.index >= 0 ? entry_loss(e, zk, m, a.inv_temp, log_s) : 0.f, s_red);
        if (threadIdx.x == 0) {
            a.loss_out[n] = w * a.temp * a.temp * loss;
            a.lse_out[n] = m * a.inv_temp + log_s;
        }
        if (!a.grad) return;
        const float f = w * a.temp, fi = f * inv;
        const bool aligned = (((uintptr_t)(out + st.head)) & 15) == 0;
        if (h.at >= 0) out[h.at] = from_float<E>(exp2_raw((h.one - m) * c) * fi);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = threadIdx.x + i * NT;
            if (v >= st.vecs) break;
            float x[VEC];
            h.values(i, x);
#pragma unroll
            for (int j = 0; j < VEC; ++j) x[j] = exp2_raw((x[j] - m) * c) * fi;
            store_granule<E>(out + st.place(v), aligned, x);
        }
        __syncthreads();                    // the dense gradient of the listed answers lies before its correction
        if (e.owner) out[e.index] = from_float<E>(f * ((inv != 0.f ? exp2_raw((zk - m) * c) * inv : 0.f) - e.sum));
    } else {
        entry_masses<NT>(a, e, s_index, s_p, s_red);
        stretch_stats<E, NT>(st, c, m, s);
        join_stats<NT>(c, m, s, s_red);
        const float log_s = logf(s), inv = s > 0.f || s != s ? 1.f / s : 0.f;
        const float loss = block_sum<NT>(e.index >= 0 ? entry_loss(e, zk, m, a.inv_temp, log_s) : 0.f, s_red);
        if (threadIdx.x == 0) {
            a.loss_out[n] = w * a.temp * a.temp * loss;
            a.lse_out[n] = m * a.inv_temp + log_s;
        }
        if (!a.grad) return;
        const float f = w * a.temp;
        stretch_grad<E, NT>(st, out, c, m, 1.f, inv, f);
        __syncthreads();
        if (e.owner) out[e.index] = from_float<E>(f * ((inv != 0.f ? exp2_raw((zk - m) * c) * inv : 0.f) - e.sum));
    }
}

// Few rows: pieces of a.piece elements.  First launch: each piece's maximum and sum, and the logits of the listed
// answers that lie in it (a second launch that writes over the logits could no longer read them).  16 rows of 131072, fp32:
// 4 us each launch, and 11 us for the gradient in a call of its own (8.4 MB read, 8.4 MB written: 3.5 us at a copy's rate; bf16 9 us; 4096 rows
// of 65536, bf16, 160 us).
template <typename E, int NT>
__global__ __launch_bounds__(NT) void distill_part_kernel(DistillArgs a) {
    __shared__ float s_red[NT / 64];
    const int64_t n = blockIdx.y;
    const int j0 = blockIdx.x * a.piece, len = min(a.piece, a.vocab - j0);
    if (a.weight && a.weight[n] == 0.f) return;
    const E* row = (const E*)a.z + n * a.stride;
    for (int k = threadIdx.x; k < a.top; k += NT) {
        const int i = a.index[n * a.top + k];
        if (i >= j0 && i < j0 + len) a.part_z[n * a.top + k] = to_float(row[i]);
    }
    float m, s;
    const float c = LOG2E * a.inv_temp;
    stretch_stats<E, NT>(Stretch<E>(row + j0, len), c, m, s);
    join_stats<NT>(c, m, s, s_red);
    if (threadIdx.x == 0) {
        float* o = a.part + 2 * (n * a.pieces + blockIdx.x);
        o[0] = s == 0.f ? NEG_INF : m;
        o[1] = s;
    }
}
// Second launch (JOIN), or the whole backward call: the gradient of one piece.  A piece of a FAR row reads the whole row first; where
// the gradient takes the logits' place and rows have several pieces, those rows go in a launch of their own, a workgroup each (a.part_rows).
template <typename E, int NT, bool JOIN>
__global__ __launch_bounds__(NT) void distill_piece_kernel(DistillArgs a) {
    __shared__ __align__(16) int s_index[PQL_MAX_TOP];
    __shared__ __align__(16) float s_p[PQL_MAX_TOP], s_red[NT / 64];
    const int64_t n = blockIdx.y;
    const int j0 = blockIdx.x * a.piece, len = min(a.piece, a.vocab - j0);
    Entry e;
    const float w = entry_of(a, n, e);
    E* out = (E*)a.grad + n * a.grad_stride + j0;
    if (!__syncthreads_or(e.index >= 0) || w == 0.f) {          // in both launches of a call in parts
        if (JOIN && blockIdx.x == 0 && threadIdx.x == 0) { a.loss_out[n] = 0.f; a.lse_out[n] = 0.f; }
        if (a.grad) zero_stretch<E, NT>(out, len);
        return;
    }
    const E* row = (const E*)a.z + n * a.stride + j0;
    const float c = LOG2E * a.inv_temp, f = w * a.temp;
    float m, inv, zk = 0.f, t_m = 1.f;
    const bool mine = e.index >= j0 && e.index < j0 + len;
    if (JOIN) {
        float pm = NEG_INF, ps = 0.f;
        if ((int)threadIdx.x < a.pieces) {
            pm = a.part[2 * (n * a.pieces + threadIdx.x)];
            ps = a.part[2 * (n * a.pieces + threadIdx.x) + 1];
        }
        if (e.index >= 0) zk = a.part_z[n * a.top + threadIdx.x];
        join_stats<NT>(c, pm, ps, s_red);
        m = pm;
        const float log_s = logf(ps);
        inv = ps > 0.f || ps != ps ? 1.f / ps : 0.f;
        if (a.grad) stretch_grad<E, NT>(Stretch<E>(row, len), out, c, m, t_m, inv, f);
        entry_masses<NT>(a, e, s_index, s_p, s_red);        // meanwhile
        if (blockIdx.x == 0) {
            const float loss = block_sum<NT>(e.index >= 0 ? entry_loss(e, zk, m, a.inv_temp, log_s) : 0.f, s_red);
            if (threadIdx.x == 0) {
                a.loss_out[n] = w * a.temp * a.temp * loss;
                a.lse_out[n] = m * a.inv_temp + log_s;
            }
        }
        if (!a.grad) return;
    } else {
        m = a.lse[n];                                       // exp(z / t - lse) = exp2((z - t lse) c)
        t_m = a.temp;
        inv = 1.f;
        const bool far = fabsf(m) > FAR;
        if (a.part_rows != ROWS_ALL && far != (a.part_rows == ROWS_FAR)) return;
        if (far) {
            float s;
            stretch_stats<E, NT>(Stretch<E>(row - j0, a.vocab), c, m, s);
            join_stats<NT>(c, m, s, s_red);
            inv = s > 0.f || s != s ? 1.f / s : 0.f;
            t_m = 1.f;
        }
        if (mine) zk = to_float(row[e.index - j0]);
        __syncthreads();                                    // read before the gradient may be written over the logits
        stretch_grad<E, NT>(Stretch<E>(row, len), out, c, m, t_m, inv, f);
        entry_masses<NT>(a, e, s_index, s_p, s_red);        // meanwhile
    }
    __syncthreads();                        // the dense gradient of the listed answers lies before its correction
    if (e.owner && mine) out[e.index - j0] = from_float<E>(f * ((inv != 0.f ? exp2_raw(fmaf(-m, t_m, zk) * c) * inv : 0.f) - e.sum));
}

// =============================================================================================
// The largest logits of every row.  Order: by value, equal values by ascending index.  Values are compared through
// unsigned keys in the same order; 0 stands for -inf and NaN, which are never selected.
// =============================================================================================
__device__ __forceinline__ unsigned key_of(float x) {
    const unsigned u = __float_as_uint(x);
    const unsigned k = u & 0x80000000u ? ~u : u | 0x80000000u;
    return x != x || x == NEG_INF ? 0u : x == 0.f ? 0x80000000u : k;      // -0 and +0 are equal
}
// the value in the bits it had: zeros come back as +0
__device__ __forceinline__ float value_of(unsigned k) {
    return k == 0u ? NEG_INF : __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

// Small vocabularies: G lanes per row.  The K-th largest key is found bit by bit (largest t with at least K keys >= t),
// the keys above it and, in index order, as many equal ones as there is room for go to LDS, and each is written at its
// rank among them.  Bound by the 32 counts: 16384 rows of 1000, fp32, lists of 32: 47 us, 1.5 TB/s.
template <typename E, int G, int R>
__global__ __launch_bounds__(256) void top_small_kernel(TopArgs a) {
    constexpr int ROWS = 256 / G;
    extern __shared__ unsigned lds_u[];
    const int g = threadIdx.x / G, l = threadIdx.x & (G - 1);
    unsigned* s_key = lds_u + (size_t)g * 2 * a.top;
    int* s_index = (int*)(s_key + a.top);
    const int64_t n = (int64_t)blockIdx.x * ROWS + g;
    const bool in = n < a.rows;
    const E* row = (const E*)a.z + n * a.stride;
    unsigned key[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int j = l + G * r;
        key[r] = in && j < a.vocab ? key_of(to_float(row[j])) : 0u;
    }
    unsigned t = 0;
    int at_least = G * R;                   // keys >= t
    for (int bit = 31; bit >= 0; --bit) {
        const unsigned u = t | (1u << bit);
        int cnt = 0;
#pragma unroll
        for (int r = 0; r < R; ++r) cnt += key[r] >= u;
        cnt = group_sum<G>(cnt);
        if (at_least != a.top && cnt >= a.top) { t = u; at_least = cnt; }
        if (__all(at_least == a.top)) break;
    }
    if (t == 0) t = 1;                      // fewer than K keys that may be selected: all of them
    // places: keys above t first, then equal ones by index; lanes in order within a register, registers in order
    int above = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) above += key[r] > t;
    int base = above;                       // exclusive prefix of `above` over the group's lanes
#pragma unroll
    for (int d = 1; d < G; d *= 2) { const int o = __shfl_up(base, d, G); if (l >= d) base += o; }
    const int n_above = __shfl(base, G - 1, G);
    base -= above;
    int eq_base = n_above;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (key[r] > t) { s_key[base] = key[r]; s_index[base] = l + G * r; ++base; }
        const unsigned long long mask = __ballot(key[r] == t) >> ((threadIdx.x & 63) / G * G);
        const unsigned long long grp = G == 64 ? mask : mask & ((1ull << (G & 63)) - 1);
        const int pos = eq_base + __popcll(grp & ((1ull << l) - 1));
        if (key[r] == t && pos < a.top) { s_key[pos] = key[r]; s_index[pos] = l + G * r; }
        eq_base += __popcll(grp);
    }
    const int found = min(eq_base, a.top);
    __syncthreads();
    if (!in) return;
    for (int k = l; k < a.top; k += G) {
        int rank = k, index = -1;
        unsigned mine = 0;
        if (k < found) {
            mine = s_key[k]; index = s_index[k];
            rank = 0;
            for (int i = 0; i < found; ++i) {
                const unsigned o = s_key[i];
                rank += o > mine || (o == mine && s_index[i] < index);
            }
        }
        a.index_out[n * a.top + rank] = index;
        a.value_out[n * a.top + rank] = value_of(mine);
    }
}

// Short lists of small vocabularies: K rounds of the largest key left.  A key's low bits make room for its index, reversed, so
// that one comparison finds the value and the lowest place of equal ones, and the element found is the only one that equals
// it.  16-bit values lose nothing by that.  Where two of the K + 1 largest of a row agree in the bits that are left, the
// wavefront starts again with whole keys.
template <int G, int R, bool EXACT, typename F>
__device__ __forceinline__ void top_rounds(unsigned (&key)[R], int l, int rounds, F&& found) {
#pragma unroll 1
    for (int k = 0; k < rounds; ++k) {
        unsigned big = key[0];
#pragma unroll
        for (int r = 1; r < R; ++r) big = max(big, key[r]);
        big = group_max<G>(big);
        int at = 0;
        if (EXACT) {
            at = 0x7fffffff;
#pragma unroll
            for (int r = R - 1; r >= 0; --r) at = key[r] == big ? l + G * r : at;
            at = group_min<G>(at);
        }
#pragma unroll
        for (int r = 0; r < R; ++r) key[r] = (EXACT ? l + G * r == at : key[r] == big) ? 0u : key[r];
        found(k, big, at);
    }
}
template <typename E, int G, int R>
__global__ __launch_bounds__(256) void top_rounds_kernel(TopArgs a) {
    constexpr int ROWS = 256 / G, ALL = G * R, BITS = ALL <= 32 ? 5 : ALL <= 64 ? 6 : ALL <= 128 ? 7 : ALL <= 256 ? 8 : ALL <= 512 ? 9 : 10;
    constexpr unsigned LOW = (1u << BITS) - 1;
    const int g = threadIdx.x / G, l = threadIdx.x & (G - 1);
    const int64_t n = (int64_t)blockIdx.x * ROWS + g;
    if ((int64_t)blockIdx.x * ROWS + (threadIdx.x & ~63) / G >= a.rows) return;       // whole wavefronts
    const bool in = n < a.rows;
    const E* row = (const E*)a.z + n * a.stride;
    unsigned key[R];
    auto load = [&] {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int j = l + G * r;
            key[r] = in && j < a.vocab ? key_of(to_float(row[j])) : 0u;
        }
    };
    // results stay with the lanes until a group's row of them can be written together
    int index = -1;
    auto write = [&](int k) {
        if ((k & (G - 1)) != G - 1 && k != a.top - 1) return;
        const int place = (k & ~(G - 1)) + l;
        if (in && place <= k) {
            a.index_out[n * a.top + place] = index;
            a.value_out[n * a.top + place] = index < 0 ? NEG_INF : to_float(row[index]) + 0.f;        // + 0: zeros come back as +0
        }
    };
    load();
#pragma unroll
    for (int r = 0; r < R; ++r) key[r] = key[r] ? (key[r] & ~LOW) | (unsigned)(ALL - 1 - (l + G * r)) : 0u;
    unsigned last = 0;
    bool near = false;
    top_rounds<G, R, false>(key, l, a.top + (sizeof(E) == 4 ? 1 : 0), [&](int k, unsigned big, int) {
        near |= k > 0 && big != 0 && ((big ^ last) & ~LOW) == 0;
        last = big;
        if (k >= a.top) return;
        if ((k & (G - 1)) == l) index = big ? ALL - 1 - (int)(big & LOW) : -1;
        write(k);
    });
    if (sizeof(E) == 2 || !__any(near)) return;
    load();
    top_rounds<G, R, true>(key, l, a.top, [&](int k, unsigned big, int at) {
        if ((k & (G - 1)) == l) index = big ? at : -1;
        write(k);
    });
}

// Long rows.  Every thread's largest key is found in one pass; the K-th largest of those bounds the row's K-th largest
// from below, and few elements reach it: a second pass collects them, and each is written at its rank.  Where more than
// CAND reach it (many equal values), the K-th largest key of the row itself is found by digits, and equal ones are taken
// in index order.
constexpr int CAND = 2048;
template <int NT>
__device__ __forceinline__ unsigned kth_largest_of_threads(unsigned mine, int k, unsigned (*s_cnt)[NT / 64]) {
    unsigned t = 0;                         // the largest t with at least k of the threads' keys >= t, two bits a round
#pragma unroll 1
    for (int bit = 30; bit >= 0; bit -= 2) {
        const unsigned u = 1u << bit;
        // counts of three thresholds, at most NT <= 1023 each
        const unsigned c = __popcll(__ballot(mine >= t + u)) | __popcll(__ballot(mine >= t + 2 * u)) << 10 | __popcll(__ballot(mine >= t + 3 * u)) << 20;
        unsigned* s = s_cnt[bit >> 1 & 1];  // two buffers: one barrier a round
        if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = c;
        __syncthreads();
        unsigned all = 0;
#pragma unroll
        for (int i = 0; i < NT / 64; ++i) all += s[i];
        const int kk = k;
        t += (int)(all >> 20) >= kk ? 3 * u : (int)(all >> 10 & 1023) >= kk ? 2 * u : (int)(all & 1023) >= kk ? u : 0u;
    }
    return t;
}
// The value that a key t >= 1 stands for, as a bound for comparisons: x >= bound exactly where key_of(x) >= t.
__device__ __forceinline__ float bound_of(unsigned t) { return t <= 0x00800000u ? -3.402823466e38f : value_of(t); }
template <typename E, int NT, typename F>
__device__ __forceinline__ void for_each(const Stretch<E>& st, F&& f) {        // f(value, place)
    constexpr int VEC = Stretch<E>::VEC, UNROLL = 4;
    const int t = threadIdx.x, one = st.single(t);
    if (one >= 0) f(to_float(st.p[one]), one);
    for (int v = t; v < st.vecs; v += UNROLL * NT) {
        uint4 g[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) if (v + u * NT < st.vecs) g[u] = st.granule(v + u * NT);
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            if (v + u * NT >= st.vecs) break;
            float x[VEC];
            unpack<E>(g[u], x);
#pragma unroll
            for (int i = 0; i < VEC; ++i) f(x[i], st.place(v + u * NT) + i);
        }
    }
}
template <typename E, int NT, typename F>
__device__ __forceinline__ void for_each_key(const Stretch<E>& st, F&& f) {
    for_each<E, NT>(st, [&](float x, int j) { f(key_of(x), j); });
}
// Writes n candidates (at most CAND, distinct; keys 16-byte aligned) at their ranks; places without one get -1.
template <int NT>
__device__ __forceinline__ void write_ranked(const unsigned* s_key, const int* s_index, int n, int top, int base, int* index_out, float* value_out, int t = threadIdx.x) {
    for (int k = t; k < n; k += NT) {
        const unsigned mine = s_key[k];
        const int index = s_index[k];
        int rank = 0, same = 0;
        const uint4* four = (const uint4*)s_key;
#pragma unroll 4
        for (int i = 0; i < n / 4; ++i) {       // reads that do not depend on each other
            const uint4 o = four[i];
            rank += (o.x > mine) + (o.y > mine) + (o.z > mine) + (o.w > mine);
            same += (o.x == mine) + (o.y == mine) + (o.z == mine) + (o.w == mine);
        }
        for (int i = n & ~3; i < n; ++i) { rank += s_key[i] > mine; same += s_key[i] == mine; }
        if (same > 1)
            for (int i = 0; i < n; ++i) rank += s_key[i] == mine && s_index[i] < index;
        if (rank < top) { index_out[rank] = base + index; value_out[rank] = value_of(mine); }
    }
    for (int k = t; k < top; k += NT)
        if (k >= n) { index_out[k] = -1; value_out[k] = NEG_INF; }
}
// Rows of up to 64 NV granules and lists of up to 64: one wavefront per row, the same steps without barriers.
template <typename E, int NV>
__global__ __launch_bounds__(256) void top_wave_kernel(TopArgs a) {
    constexpr int SOME = 256, VEC = Stretch<E>::VEC;
    __shared__ __align__(16) unsigned s_key_all[4][SOME];
    __shared__ int s_index_all[4][SOME], s_n_all[4];
    const int wave = threadIdx.x >> 6, l = threadIdx.x & 63;
    const int64_t n = (int64_t)blockIdx.x * 4 + wave;
    if (n >= a.rows) return;                // wavefronts share nothing
    unsigned* s_key = s_key_all[wave];
    int* s_index = s_index_all[wave];
    int* s_n = &s_n_all[wave];
    const Stretch<E> st((const E*)a.z + n * a.stride, a.vocab);
    Held<E, 64, NV> h(st, l);
    if (l == 0) *s_n = 0;
    float most = NEG_INF;
    h.each([&](float x, int) { most = fmaxf(most, x); });
    const unsigned big = key_of(most);
    unsigned t = 0;                         // the largest t with at least K lanes' keys >= t
    for (int bit = 31; bit >= 0; --bit) {
        const unsigned u = t | (1u << bit);
        if (__popcll(__ballot(big >= u)) >= a.top) t = u;
    }
    if (t == 0) t = 1;
    wave_fence();
    const float bound = bound_of(t);
    auto collect = [&](float x, int j, bool room) {
        const int at = atomicAdd(s_n, 1);
        if (room || at < SOME) { s_key[at] = key_of(x); s_index[at] = j; }
    };
    if (h.one >= bound) collect(h.one, h.at, false);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        float x[VEC], b = NEG_INF;
        h.values(i, x);
#pragma unroll
        for (int j = 0; j < VEC; ++j) b = fmaxf(b, x[j]);
        if (b >= bound) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) if (x[j] >= bound) collect(x[j], st.place(l + i * 64) + j, false);
        }
    }
    wave_fence();
    int found = *(volatile int*)s_n;
    if (found > SOME) {                     // many equal values: the K-th largest key itself, then equal ones by index
        unsigned lo = 0;
#pragma unroll 1
        for (int bit = 31; bit >= 0; --bit) {
            const unsigned u = lo | (1u << bit);
            int c = 0;
            h.each([&](float x, int) { c += key_of(x) >= u; });
            if (group_sum<64>(c) >= a.top) lo = u;
        }
        if (lo == 0) lo = 1;
        wave_fence();
        if (l == 0) *s_n = 0;
        wave_fence();
        if (key_of(h.one) > lo) collect(h.one, h.at, true);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float x[VEC];
            h.values(i, x);
#pragma unroll
            for (int j = 0; j < VEC; ++j) if (key_of(x[j]) > lo) collect(x[j], st.place(l + i * 64) + j, true);     // fewer than K
        }
        wave_fence();
        found = *(volatile int*)s_n;
        for (int b = 0; b < a.vocab && found < a.top; b += 64) {
            const int j = b + l;
            const bool eq = j < a.vocab && key_of(to_float(st.p[j])) == lo;
            const unsigned long long mask = __ballot(eq);
            const int at = found + __popcll(mask & ((1ull << l) - 1));
            if (eq && at < a.top) { s_key[at] = lo; s_index[at] = j; }
            found = min(a.top, found + __popcll(mask));
        }
        wave_fence();
    }
    write_ranked<64>(s_key, s_index, found, a.top, 0, a.index_out + n * a.top, a.value_out + n * a.top, l);
}

// One workgroup per row or piece.  NV > 0: the stretch stays in registers between the two passes, NV granules a thread; else it
// is read again, from L2 for the most part.  1024 rows of 131072, lists of 64: bf16 82 us, 3.3 TB/s, fp32 150 us, 3.6 TB/s.
template <typename E, int NT, int NV, bool MERGE>
__device__ __forceinline__ void top_of_stretch(const TopArgs& a) {
    __shared__ __align__(16) unsigned s_key[CAND];
    __shared__ unsigned s_two[2][NT / 64];
    __shared__ int s_index[CAND], s_cnt[NT / 64], s_n;
    const int64_t n = blockIdx.y;
    const int j0 = blockIdx.x * a.piece, len = min(a.piece, a.vocab - j0);
    const Stretch<E> st((const E*)a.z + n * a.stride + j0, len);
    const int64_t o = (n * gridDim.x + blockIdx.x) * a.top;
    unsigned big = 0;
    if (threadIdx.x == 0) s_n = 0;
    auto collect = [&](unsigned k, int j, unsigned t) {
        if (k >= t) {
            const int at = atomicAdd(&s_n, 1);
            if (at < CAND) { s_key[at] = k; s_index[at] = j; }
        }
    };
    if constexpr (NV > 0) {
        Held<E, NT, NV> h(st);
        float most = NEG_INF;               // compared as they are; only the threads' results as keys
        h.each([&](float x, int) { most = fmaxf(most, x); });
        big = key_of(most);
        unsigned t = kth_largest_of_threads<NT>(big, a.top, s_two);
        if (t == 0) t = 1;                  // fewer than K threads hold one that may be selected
        if (big >= t) {                     // few threads
            const float bound = bound_of(t);
            if (h.one >= bound) collect(key_of(h.one), h.at, t);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float x[Stretch<E>::VEC], b = NEG_INF;
                h.values(i, x);
#pragma unroll
                for (int j = 0; j < Stretch<E>::VEC; ++j) b = fmaxf(b, x[j]);
                if (b >= bound) {
#pragma unroll
                    for (int j = 0; j < Stretch<E>::VEC; ++j)
                        if (x[j] >= bound) collect(key_of(x[j]), st.place(threadIdx.x + i * NT) + j, t);
                }
            }
        }
    } else {
        float most = NEG_INF;
        for_each<E, NT>(st, [&](float x, int) { most = fmaxf(most, x); });
        big = key_of(most);
        unsigned t = kth_largest_of_threads<NT>(big, a.top, s_two);
        if (t == 0) t = 1;
        const float bound = bound_of(t);
        if (big >= t) for_each<E, NT>(st, [&](float x, int j) { if (x >= bound) collect(key_of(x), j, t); });
    }
    __syncthreads();
    int found = s_n;
    if (found > CAND) {
        // the K-th largest key of the stretch, bit by bit from the bound on; then the keys above it in any order and
        // the equal ones by index
        unsigned lo = 0;
        for (int bit = 31; bit >= 0; --bit) {
            const unsigned u = lo | (1u << bit);
            int c = 0;
            for_each_key<E, NT>(st, [&](unsigned k, int) { c += k >= u; });
            if (block_sum<NT>(c, s_cnt) >= a.top) lo = u;
        }
        if (lo == 0) lo = 1;
        __syncthreads();
        if (threadIdx.x == 0) s_n = 0;
        __syncthreads();
        for_each_key<E, NT>(st, [&](unsigned k, int j) {
            if (k > lo) { const int at = atomicAdd(&s_n, 1); s_key[at] = k; s_index[at] = j; }     // fewer than K
        });
        __syncthreads();
        found = s_n;
        for (int b = 0; b < len && found < a.top; b += NT) {        // in index order, NT elements at a time
            const int j = b + threadIdx.x;
            const bool eq = j < len && key_of(to_float(st.p[j])) == lo;
            const unsigned long long mask = __ballot(eq);
            __syncthreads();
            if ((threadIdx.x & 63) == 0) s_cnt[threadIdx.x >> 6] = __popcll(mask);
            __syncthreads();
            int at = found + __popcll(mask & ((1ull << (threadIdx.x & 63)) - 1));
            int all = 0;
            for (int i = 0; i < NT / 64; ++i) { if (i < (int)(threadIdx.x >> 6)) at += s_cnt[i]; all += s_cnt[i]; }
            if (eq && at < a.top) { s_key[at] = lo; s_index[at] = j; }
            found = min(a.top, found + all);
        }
        __syncthreads();
    }
    if constexpr (MERGE) {
        for (int i = threadIdx.x; i < min(found, CAND); i += NT) s_index[i] = a.part_index[n * a.vocab + s_index[i]];
        __syncthreads();
    }
    write_ranked<NT>(s_key, s_index, found, a.top, j0, a.pieces > 1 ? a.part_index + o : a.index_out + o,
                     a.pieces > 1 ? a.part_value + o : a.value_out + o);
}
template <typename E, int NT, int NV>
__global__ __launch_bounds__(NT) void top_row_kernel(TopArgs a) { top_of_stretch<E, NT, NV, false>(a); }
// Joins the lists of a row's pieces: the same selection from their values, the places found being looked up in the lists'
// indices.  Equal values lie in index order (within a list by its order, lists by that of the pieces), so places rank as
// indices would.
template <int NV>
__global__ __launch_bounds__(256) void top_merge_kernel(TopArgs a) { top_of_stretch<float, 256, NV, true>(a); }

// ---- launches -------------------------------------------------------------------------------
constexpr int NT_LONG = 512;
// One wavefront per row: rows of at most 16 KB, and enough of them to give every SIMD two.  Loss and gradient, bf16, by
// wavefronts and by workgroups: 2048 rows of 1500 8 and 12 us, of 4000 12 and 14, of 8000 19 and 18; 65536 rows of 1500 121
// and 263, of 4000 208 and 318, of 8000 415 and 414; 512 rows of 8000 11 and 9.  Selection of 32, 65536 rows: 116 and 357,
// 158 and 384, 289 and 408 us.  fp32, loss and gradient: 2048 rows of 1100 10 and 10, of 2000 13 and 12, of 4000 20 and 20; 65536 rows 182 and 229, 262 and 298,
// 480 and 446; selection: 2048 rows 7 and 14, 10 and 15, 12 and 16; 65536 rows 96 and 313, 113 and 329, 218 and 342.
constexpr int64_t WAVE_VECS = 64 * 16, WAVE_ROWS = 2048;
constexpr int64_t MAX_GRID = 0x7fffffff;

// Pieces of a long row, of `least` elements or more: as many as give 1024 workgroups, but one where `most_rows` rows or more
// (of 131072 logits; in proportion more of longer ones) keep the CUs busy by themselves.
int pieces_of(int64_t rows, int vocab, int least, int most, int most_rows) {
    if (rows >= 256 || vocab <= SMALL_VOCAB || rows * 131072 > (int64_t)most_rows * (vocab > 131072 ? vocab : 131072)) return 1;
    int64_t p = (1024 + rows - 1) / (rows > 0 ? rows : 1);
    const int64_t by_len = vocab / least;
    if (p > by_len) p = by_len;
    if (p > most) p = most;
    return (int)(p < 1 ? 1 : p);
}
// A second launch takes 4 us, so rows have to be long: of 80 KB for loss and gradient, of 192 KB for the loss alone.  In pieces and whole, us, fp32:
// loss and gradient, 1 row of 20000 9 and 11, 64 of 40000 14 and 18, 128 of 131072 42 and 53, 192 58 and 54, 160 of 600000 290 and
// 367; loss, 1 row of 40000 9 and 7, 1 of 131072 8 and 13, 128 17 and 16.  bf16, loss and gradient: 1 row of 20000 9 and 8, of 40000 10 and 11.
int distill_pieces(const pql_logits& z, bool grad) {
    const int64_t bytes = (int64_t)z.vocab * (z.dtype == PQL_F32 ? 4 : 2);
    return bytes < (grad ? 80000 : 192000) ? 1 : pieces_of(z.rows, z.vocab, 4096, 256, 128);
}
int piece_len(int vocab, int pieces) {      // a multiple of 64 elements: pieces keep the row's alignment
    const int len = (vocab + pieces - 1) / pieces;
    return pieces == 1 ? vocab : (len + 63) / 64 * 64;
}
bool dtype_ok(int32_t d) { return d == PQL_F32 || d == PQL_BF16; }
int elem(int32_t d) { return d == PQL_F32 ? 4 : 2; }
bool logits_ok(const pql_logits& z) {
    return z.rows >= 0 && z.rows <= MAX_GRID && z.vocab >= 1 && z.vocab <= (1 << 30) && z.stride >= z.vocab && dtype_ok(z.dtype);
}
size_t up256(size_t x) { return (x + 255) / 256 * 256; }

// Seven registers a lane, for 33 to 56 logits: 327680 rows of 40, fp32, loss and gradient 31.6 us, with eight 32.5; 8 largest 31.8 and 32.9.
#define SMALL_CASES(X) X(8, 4) X(8, 7) X(8, 8) X(16, 8) X(32, 8) X(64, 8) X(64, 16)
template <typename E, bool BACK> hipError_t distill_small_launch(const DistillArgs& a, int kid, double bytes, hipStream_t st) {
#define PQL_SMALL(G, R)                                                                                              \
    if (a.vocab <= G * R) {                                                                                          \
        constexpr int ROWS = 256 / G;                                                                                \
        const size_t lds = (size_t)ROWS * (2 * a.top + a.vocab) * 4;                                                 \
        const ProfSlot ps = prof_slot();                                                                             \
        PQL_LAUNCH(ps, (distill_small_kernel<E, G, R, BACK>), dim3((unsigned)((a.rows + ROWS - 1) / ROWS)), dim3(256), lds, st, a); \
        prof_commit(ps, kid, 0.0, bytes);                                                                            \
        return hipGetLastError();                                                                                    \
    }
    SMALL_CASES(PQL_SMALL)
#undef PQL_SMALL
    return hipErrorInvalidValue;
}
// Longest list that is taken by rounds, one entry each, in a group of G lanes; longer ones by bits of the key.  By rounds and by
// bits, fp32: 327680 rows of 51, list of 16 53 and 62 us, of 48 127 and 219; 150000 of 100, list of 16 50 and 53, of 24 71
// and 65; 16384 of 1000, list of 8 36 and 41, of 12 43 and 42, of 16 52 and 44.
constexpr int ROUNDS(int g) { return g == 8 ? 64 : g == 64 ? 12 : 16; }
template <typename E> hipError_t top_small_launch(const TopArgs& a, double bytes, hipStream_t st) {
#define PQL_SMALL(G, R)                                                                                              \
    if (a.vocab <= G * R) {                                                                                          \
        constexpr int ROWS = 256 / G;                                                                                \
        const ProfSlot ps = prof_slot();                                                                             \
        const dim3 grid((unsigned)((a.rows + ROWS - 1) / ROWS));                                                     \
        if (a.top <= ROUNDS(G)) PQL_LAUNCH(ps, (top_rounds_kernel<E, G, R>), grid, dim3(256), 0, st, a);             \
        else if constexpr (G > 8)                                                                                    \
            PQL_LAUNCH(ps, (top_small_kernel<E, G, R>), grid, dim3(256), (size_t)ROWS * 2 * a.top * 4, st, a);       \
        prof_commit(ps, KID_TOP_LOGITS, 0.0, bytes);                                                                 \
        return hipGetLastError();                                                                                    \
    }
    SMALL_CASES(PQL_SMALL)
#undef PQL_SMALL
    return hipErrorInvalidValue;
}

// grid.y holds at most 65535 rows, and a grid at most 2^32 - 1 threads, which rows of up to 512 threads each reach: longer calls go in parts
constexpr int64_t ROWS_PER_LAUNCH = 65535, ROWS_PER_PART = 1 << 22;
template <typename E> DistillArgs from_row(DistillArgs a, int64_t n, int64_t rows) {
    a.z = (const E*)a.z + n * a.stride;
    if (a.grad) a.grad = (E*)a.grad + n * a.grad_stride;
    a.index += n * a.top; a.value += n * a.top;
    if (a.weight) a.weight += n;
    if (a.lse) a.lse += n;
    if (a.loss_out) a.loss_out += n;
    if (a.lse_out) a.lse_out += n;
    a.rows = rows;
    return a;
}
template <typename E> hipError_t distill_part(const DistillArgs& a, bool back, hipStream_t st) {
    const double read = (double)a.rows * a.vocab * sizeof(E), lists = (double)a.rows * a.top * 8;
    const double bytes = read * (a.grad ? 2 : 1) + lists + 12.0 * a.rows;
    if (a.vocab <= SMALL_VOCAB)
        return back ? distill_small_launch<E, true>(a, KID_DISTILL_GRAD, bytes, st) : distill_small_launch<E, false>(a, KID_DISTILL, bytes, st);
    const int64_t vecs = (int64_t)a.vocab * (int)sizeof(E) / 16;
    const dim3 by_row((unsigned)a.rows), by_wave((unsigned)((a.rows + 3) / 4));
    if (vecs <= WAVE_VECS && a.rows >= WAVE_ROWS) {
        const ProfSlot ps = prof_slot();
#define PQL_WAVE(NV)                                                                                            \
    if (back) PQL_LAUNCH(ps, (distill_wave_kernel<E, NV, true>), by_wave, dim3(256), 0, st, a);                 \
    else PQL_LAUNCH(ps, (distill_wave_kernel<E, NV, false>), by_wave, dim3(256), 0, st, a)
        if (vecs <= 64 * 4) { PQL_WAVE(4); } else if (vecs <= 64 * 8) { PQL_WAVE(8); } else { PQL_WAVE(16); }
#undef PQL_WAVE
        prof_commit(ps, back ? KID_DISTILL_GRAD : KID_DISTILL, 0.0, bytes);
    } else if (back) {
        // in the logits' place, rows that read all of themselves for every piece would find some of it written over
        const bool apart = a.grad == a.z && a.pieces > 1;
        for (int64_t n = 0; n < a.rows; n += ROWS_PER_LAUNCH) {
            DistillArgs b = from_row<E>(a, n, a.rows - n < ROWS_PER_LAUNCH ? a.rows - n : ROWS_PER_LAUNCH);
            b.part_rows = apart ? ROWS_NEAR : ROWS_ALL;
            ProfSlot ps = prof_slot();
            PQL_LAUNCH(ps, (distill_piece_kernel<E, NT_LONG, false>), dim3(a.pieces, (unsigned)b.rows), dim3(NT_LONG), 0, st, b);
            prof_commit(ps, KID_DISTILL_GRAD, 0.0, bytes * b.rows / a.rows);
            if (!apart) continue;
            b.part_rows = ROWS_FAR;
            b.pieces = 1;
            b.piece = a.vocab;
            ps = prof_slot();
            PQL_LAUNCH(ps, (distill_piece_kernel<E, NT_LONG, false>), dim3(1, (unsigned)b.rows), dim3(NT_LONG), 0, st, b);
            prof_commit(ps, KID_DISTILL_GRAD, 0.0, 0.0);
        }
    } else if (a.pieces > 1) {
        ProfSlot ps = prof_slot();
        PQL_LAUNCH(ps, (distill_part_kernel<E, NT_LONG>), dim3(a.pieces, (unsigned)a.rows), dim3(NT_LONG), 0, st, a);
        prof_commit(ps, KID_DISTILL, 0.0, read);
        ps = prof_slot();
        PQL_LAUNCH(ps, (distill_piece_kernel<E, NT_LONG, true>), dim3(a.grad ? a.pieces : 1, (unsigned)a.rows), dim3(NT_LONG), 0, st, a);
        prof_commit(ps, KID_DISTILL_JOIN, 0.0, a.grad ? bytes : lists);
    } else {
        const ProfSlot ps = prof_slot();
        // the loss alone needs every logit once; rows over 128 KB do not stay in registers
        if (!a.grad || vecs > 512 * 16) PQL_LAUNCH(ps, (distill_row_kernel<E, 512, 0>), by_row, dim3(512), 0, st, a);
        else if (vecs <= 256 * 4) PQL_LAUNCH(ps, (distill_row_kernel<E, 256, 4>), by_row, dim3(256), 0, st, a);
        else if (vecs <= 256 * 8) PQL_LAUNCH(ps, (distill_row_kernel<E, 256, 8>), by_row, dim3(256), 0, st, a);
        else if (vecs <= 512 * 8) PQL_LAUNCH(ps, (distill_row_kernel<E, 512, 8>), by_row, dim3(512), 0, st, a);
        else PQL_LAUNCH(ps, (distill_row_kernel<E, 512, 16>), by_row, dim3(512), 0, st, a);
        prof_commit(ps, KID_DISTILL, 0.0, bytes);
    }
    return hipGetLastError();
}
template <typename E> hipError_t distill_launch(const DistillArgs& a, bool back, hipStream_t st) {
    hipError_t e = hipSuccess;
    for (int64_t n = 0; n < a.rows && e == hipSuccess; n += ROWS_PER_PART)
        e = distill_part<E>(from_row<E>(a, n, a.rows - n < ROWS_PER_PART ? a.rows - n : ROWS_PER_PART), back, st);
    return e;
}
template <typename E> TopArgs from_row(TopArgs a, int64_t n, int64_t rows) {
    a.z = (const E*)a.z + n * a.stride;
    a.index_out += n * a.top; a.value_out += n * a.top;
    a.rows = rows;
    return a;
}
template <typename E> hipError_t top_part(const TopArgs& a, hipStream_t st) {
    const double bytes = (double)a.rows * a.vocab * sizeof(E) + (double)a.rows * a.top * 8;
    if (a.vocab <= SMALL_VOCAB) return top_small_launch<E>(a, bytes, st);
    const int64_t vecs = (int64_t)a.piece * (int)sizeof(E) / 16;
    if (a.pieces == 1 && vecs <= WAVE_VECS && a.top <= 64 && a.rows >= WAVE_ROWS) {
        const dim3 grid((unsigned)((a.rows + 3) / 4));
        const ProfSlot ps = prof_slot();
        if (vecs <= 64 * 4) PQL_LAUNCH(ps, (top_wave_kernel<E, 4>), grid, dim3(256), 0, st, a);
        else if (vecs <= 64 * 8) PQL_LAUNCH(ps, (top_wave_kernel<E, 8>), grid, dim3(256), 0, st, a);
        else PQL_LAUNCH(ps, (top_wave_kernel<E, 16>), grid, dim3(256), 0, st, a);
        prof_commit(ps, KID_TOP_LOGITS, 0.0, bytes);
        return hipGetLastError();
    }
    for (int64_t n = 0; n < a.rows; n += ROWS_PER_LAUNCH) {
        const TopArgs b = from_row<E>(a, n, a.rows - n < ROWS_PER_LAUNCH ? a.rows - n : ROWS_PER_LAUNCH);
        const ProfSlot ps = prof_slot();
        const dim3 grid(a.pieces, (unsigned)b.rows);
        if (vecs <= 256 * 4) PQL_LAUNCH(ps, (top_row_kernel<E, 256, 4>), grid, dim3(256), 0, st, b);
        else if (vecs <= 256 * 8) PQL_LAUNCH(ps, (top_row_kernel<E, 256, 8>), grid, dim3(256), 0, st, b);
        else if (vecs <= 512 * 8) PQL_LAUNCH(ps, (top_row_kernel<E, 512, 8>), grid, dim3(512), 0, st, b);
        else PQL_LAUNCH(ps, (top_row_kernel<E, 512, 0>), grid, dim3(512), 0, st, b);
        prof_commit(ps, KID_TOP_LOGITS, 0.0, bytes * b.rows / a.rows);
    }
    if (a.pieces > 1) {
        const ProfSlot ps = prof_slot();
        TopArgs m = a;
        m.z = a.part_value; m.vocab = m.piece = a.pieces * a.top; m.stride = m.vocab; m.pieces = 1;
        if (m.vocab <= 256 * 4 * 4) PQL_LAUNCH(ps, top_merge_kernel<4>, dim3(1, (unsigned)a.rows), dim3(256), 0, st, m);
        else PQL_LAUNCH(ps, top_merge_kernel<8>, dim3(1, (unsigned)a.rows), dim3(256), 0, st, m);
        prof_commit(ps, KID_TOP_MERGE, 0.0, (double)a.rows * a.top * 8 * (a.pieces + 1));
    }
    return hipGetLastError();
}
template <typename E> hipError_t top_launch(const TopArgs& a, hipStream_t st) {
    hipError_t e = hipSuccess;
    for (int64_t n = 0; n < a.rows && e == hipSuccess; n += ROWS_PER_PART)
        e = top_part<E>(from_row<E>(a, n, a.rows - n < ROWS_PER_PART ? a.rows - n : ROWS_PER_PART), st);
    return e;
}
// The lists of a row's pieces are merged in registers: at most 8192 entries.  That costs the more the longer the lists, and the more of
// their values are equal, as many 16-bit ones are.  In pieces and whole, us, fp32: the 8 largest of 1 row of 65536 16 and 16, of 1 of 131072 15 and 21,
// of 128 26 and 29, of 192 34 and 33; the 64 largest of 1 21 and 25, of 64 36 and 27, of 64 of 600000 62 and 115; the 128 largest of 1 of 200000
// 50 and 35.  bf16: the 8 largest of 1 of 131072 17 and 20, the 24 largest 25 and 22, the 64 largest 63 and 27.
int top_pieces(const pql_logits& z, int top) {
    const int weight = z.dtype == PQL_F32 ? top : 2 * top;
    return z.vocab < 131072 || weight > 64 ? 1 : pieces_of(z.rows, z.vocab, 16384, 8192 / top, weight <= 32 ? 128 : 48);
}
bool misaligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) != 0; }
int32_t check_logits(pql_ctx* c, const pql_logits& z, const char* text) {
    if (!logits_ok(z)) return ctx_fail(c, PQL_ERR_INVALID_ARG, text);
    return PQL_OK;
}
}  // namespace
}  // namespace pql

using namespace pql;

extern "C" {

int64_t pql_top_logits_workspace_bytes(const pql_logits* z, int32_t top) {
    if (!z) return PQL_ERR_NULL;
    if (!logits_ok(*z) || top < 1 || top > PQL_MAX_TOP || top > z->vocab) return PQL_ERR_INVALID_ARG;
    const int p = top_pieces(*z, top);
    return p > 1 ? (int64_t)up256((size_t)z->rows * p * top * 8) : 0;
}

int32_t pql_top_logits(pql_ctx* c, pql_logits z, int32_t top, int32_t* index_out, float* value_out, void* workspace, void* stream) {
    if (!c) return PQL_ERR_NULL;
    if (check_logits(c, z, "pql_top_logits: bad rows, vocab, stride or dtype") != PQL_OK) return PQL_ERR_INVALID_ARG;
    if (top < 1 || top > PQL_MAX_TOP || top > z.vocab) return ctx_fail(c, PQL_ERR_INVALID_ARG, "pql_top_logits: bad top");
    if (z.rows == 0) return PQL_OK;
    if (!z.data || !index_out || !value_out) return ctx_fail(c, PQL_ERR_NULL, "pql_top_logits: null pointer");
    TopArgs a{};
    a.pieces = top_pieces(z, top);
    if (a.pieces > 1 && !workspace) return ctx_fail(c, PQL_ERR_NULL, "pql_top_logits: null workspace");
    if (misaligned(z.data, elem(z.dtype)) || misaligned(index_out, 4) || misaligned(value_out, 4) || misaligned(workspace, 256))
        return ctx_fail(c, PQL_ERR_ALIGNMENT, "pql_top_logits: misaligned pointer");
    a.z = z.data; a.rows = z.rows; a.stride = z.stride; a.vocab = z.vocab; a.top = top;
    a.piece = piece_len(z.vocab, a.pieces);
    a.pieces = (z.vocab + a.piece - 1) / a.piece;
    a.index_out = index_out; a.value_out = value_out;
    a.part_index = (int*)workspace;
    a.part_value = (float*)workspace + (size_t)z.rows * a.pieces * top;
    const hipError_t e = z.dtype == PQL_F32 ? top_launch<float>(a, (hipStream_t)stream) : top_launch<bf16_t>(a, (hipStream_t)stream);
    return e == hipSuccess ? PQL_OK : ctx_fail(c, PQL_ERR_HIP, "pql_top_logits", e);
}

int64_t pql_distill_workspace_bytes(const pql_logits* z) {
    if (!z) return PQL_ERR_NULL;
    if (!logits_ok(*z)) return PQL_ERR_INVALID_ARG;
    const int p = distill_pieces(*z, true);
    return p > 1 ? (int64_t)up256((size_t)z->rows * (2 * p + PQL_MAX_TOP) * 4) : 0;
}

static int32_t distill_check(pql_ctx* c, const pql_logits& z, const pql_teacher& t, float temperature, const pql_logits& grad, bool need_grad) {
    if (check_logits(c, z, "pql_distill: bad rows, vocab, stride or dtype of the logits") != PQL_OK) return PQL_ERR_INVALID_ARG;
    if (t.top < 1 || t.top > PQL_MAX_TOP || t.top > z.vocab) return ctx_fail(c, PQL_ERR_INVALID_ARG, "pql_distill: bad top");
    if (!(temperature > 0.f) || temperature > 3.0e38f || 1.f / temperature > 3.0e38f) return ctx_fail(c, PQL_ERR_INVALID_ARG, "pql_distill: bad temperature");
    if (grad.data || need_grad) {
        if (check_logits(c, grad, "pql_distill: bad rows, vocab, stride or dtype of the gradient") != PQL_OK) return PQL_ERR_INVALID_ARG;
        if (grad.rows != z.rows || grad.vocab != z.vocab || grad.dtype != z.dtype)
            return ctx_fail(c, PQL_ERR_INVALID_ARG, "pql_distill: gradient of another shape or type than the logits");
        if (grad.data == z.data && grad.stride != z.stride && z.rows > 1)
            return ctx_fail(c, PQL_ERR_INVALID_ARG, "pql_distill: a gradient in the logits' place needs their stride");
    }
    if (z.rows == 0) return PQL_OK;
    if (!z.data || !t.index || !t.value || (need_grad && !grad.data)) return ctx_fail(c, PQL_ERR_NULL, "pql_distill: null pointer");
    if (misaligned(z.data, elem(z.dtype)) || misaligned(grad.data, elem(z.dtype)) || misaligned(t.index, 4) || misaligned(t.value, 4))
        return ctx_fail(c, PQL_ERR_ALIGNMENT, "pql_distill: misaligned pointer");
    return PQL_OK;
}
static DistillArgs distill_args(const pql_logits& z, const pql_teacher& t, float temperature, const float* weight, const pql_logits& grad, int pieces) {
    DistillArgs a{};
    a.z = z.data; a.rows = z.rows; a.stride = z.stride; a.vocab = z.vocab;
    a.index = t.index; a.value = t.value; a.top = t.top;
    a.temp = temperature; a.inv_temp = 1.f / temperature;
    a.weight = weight;
    a.grad = grad.data; a.grad_stride = grad.stride;
    a.piece = piece_len(z.vocab, pieces);
    a.pieces = (z.vocab + a.piece - 1) / a.piece;
    return a;
}

int32_t pql_distill_loss(pql_ctx* c, pql_logits z, pql_teacher t, float temperature, const float* row_weight,
                         float* loss_out, float* lse_out, pql_logits grad, void* workspace, void* stream) {
    if (!c) return PQL_ERR_NULL;
    const int32_t rc = distill_check(c, z, t, temperature, grad, false);
    if (rc != PQL_OK || z.rows == 0) return rc;
    if (!loss_out || !lse_out) return ctx_fail(c, PQL_ERR_NULL, "pql_distill_loss: null pointer");
    const int pieces = distill_pieces(z, grad.data != nullptr);
    if (pieces > 1 && !workspace) return ctx_fail(c, PQL_ERR_NULL, "pql_distill_loss: null workspace");
    if (misaligned(workspace, 256) || misaligned(loss_out, 4) || misaligned(lse_out, 4) || misaligned(row_weight, 4))
        return ctx_fail(c, PQL_ERR_ALIGNMENT, "pql_distill_loss: misaligned pointer");
    DistillArgs a = distill_args(z, t, temperature, row_weight, grad, pieces);
    a.loss_out = loss_out; a.lse_out = lse_out;
    a.part = (float*)workspace;
    a.part_z = (float*)workspace + (size_t)z.rows * 2 * a.pieces;
    const hipError_t e = z.dtype == PQL_F32 ? distill_launch<float>(a, false, (hipStream_t)stream)
                                            : distill_launch<bf16_t>(a, false, (hipStream_t)stream);
    return e == hipSuccess ? PQL_OK : ctx_fail(c, PQL_ERR_HIP, "pql_distill_loss", e);
}

int32_t pql_distill_backward(pql_ctx* c, pql_logits z, pql_teacher t, float temperature, const float* lse,
                             const float* loss_grad, pql_logits grad, void* stream) {
    if (!c) return PQL_ERR_NULL;
    const int32_t rc = distill_check(c, z, t, temperature, grad, true);
    if (rc != PQL_OK || z.rows == 0) return rc;
    if (!lse || !loss_grad) return ctx_fail(c, PQL_ERR_NULL, "pql_distill_backward: null pointer");
    if (misaligned(lse, 4) || misaligned(loss_grad, 4)) return ctx_fail(c, PQL_ERR_ALIGNMENT, "pql_distill_backward: misaligned pointer");
    // every piece works out the list's masses anew: 16384 elements keep that below a tenth of it; fewer where there are few rows
    int pieces = z.vocab <= SMALL_VOCAB ? 1 : (z.vocab + 16383) / 16384;
    const int few = pieces_of(z.rows, z.vocab, 4096, 1 << 30, 256);
    if (few > pieces) pieces = few;
    DistillArgs a = distill_args(z, t, temperature, loss_grad, grad, pieces);
    a.lse = lse;
    const hipError_t e = z.dtype == PQL_F32 ? distill_launch<float>(a, true, (hipStream_t)stream)
                                            : distill_launch<bf16_t>(a, true, (hipStream_t)stream);
    return e == hipSuccess ? PQL_OK : ctx_fail(c, PQL_ERR_HIP, "pql_distill_backward", e);
}

}  // extern "C"
