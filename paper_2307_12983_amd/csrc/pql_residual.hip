// Norms before and after a block with its gate and residual sum (include/pql_block.h):
//     r = (mean_part(y^2) + e)^-1/2,  h = ax x + ay act(g) w r y,  s = (mean(h^2) + e')^-1/2,  next = p s h.
// Gradient, from dh' (of the sum) and du (of next), with c = mean(p du h) s^2:
//     dh = dh' + s (p du - c h),  dx = ax dh,  dz = ay dh,  dw = sum dz act(g) r y,  dg = dz w r y act'(g),
//     dn = dz act(g) w,  dy = r (dn - r y mean_part(dn r y)),  dp = sum du s h.
//
// Bound by memory: every tensor is read or written once, a row stays in registers from its loads to its stores, and the
// gradient works h out again instead of reading it (which would also be rounded).  A part of a row is held by `lanes`
// lanes (a power of two), 8 elements each; a row's parts lie in one workgroup.  Workgroups stay for many rows: they keep
// the weights, and the sums of the weights' gradients, in registers.  16384 rows of 1024 in bf16, all parts: 37 us, 4.5 TB/s; 8192 rows of
// 2048, half of them counting: 33 us forward, 47 us back, and 5 us to join the weights' gradients.
#include "pql_block_internal.h"
#include "pql_lanes.h"

namespace pql {
namespace {

struct ResidualArgs {
    Live live;
    unsigned rows;
    int dim, groups, part, lanes;           // part = dim / groups elements by `lanes` lanes
    int gate_act, gate_part;                // gate_part: one value of the gate for each part
    float eps_post, eps_pre, scale_x, scale_y;
    const void *x, *y, *gate;
    int64_t x_stride, y_stride, gate_stride;
    const float *post, *pre;
    void *sum, *next;                       // gradient: read
    int64_t sum_stride, next_stride;
    void *dx, *dy, *dgate;
    int64_t dx_stride, dy_stride, dgate_stride;
    float *dpost, *dpre, *partial;          // partial: [workgroups][2][dim]
};

// ---- a thread's elements of one row ----------------------------------------------------------------
// AL: granules of 16 bytes, element i at granule i / V of this lane; otherwise every lanes-th element.
constexpr int EPT = 8;                      // elements a thread
template <typename E, bool AL> struct Slice {
    static constexpr int V = AL ? VEC_OF<E> : 1, N = EPT / V;
    int base, lane, lanes, part;
    bool on;
    __device__ __forceinline__ int place(int i) const { return (i * lanes + lane) * V; }           // within the part, of granule i
    __device__ __forceinline__ bool there(int i) const { return on && place(i) < part; }
    // As they come from memory, and as floats.
    struct Raw { uint4 g[AL ? N : 1]; float x[AL ? 1 : N]; };
    __device__ __forceinline__ void fetch(const E* p, Raw& r) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if constexpr (AL) r.g[i] = there(i) ? *(const uint4*)(p + base + place(i)) : make_uint4(0, 0, 0, 0);
            else r.x[i] = there(i) ? to_float(p[base + place(i)]) : 0.f;
        }
    }
    __device__ __forceinline__ void open(const Raw& r, float* x) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if constexpr (AL) widen(r.g[i], x + i * V, E{}); else x[i] = r.x[i];
        }
    }
    __device__ __forceinline__ void load_weights(const float* p, float* x) const {
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int k = 0; k < V; ++k) x[i * V + k] = there(i) ? (p ? p[base + place(i) + k] : 1.f) : 0.f;
    }
    __device__ __forceinline__ void store(E* p, const float* x) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (!there(i)) continue;
            if constexpr (AL) *(uint4*)(p + base + place(i)) = narrow(x + i * V, E{});
            else p[base + place(i)] = from_float<E>(x[i]);
        }
    }
    __device__ __forceinline__ void store_floats(float* p, const float* x) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (!there(i)) continue;
#pragma unroll
            for (int k = 0; k < V; ++k) p[base + place(i) + k] = x[i * V + k];
        }
    }
};

// Sum over the lanes of one part.  Parts of more than 64 lanes go through LDS, so that all threads have to come here.
struct Sums {
    float* lds;                             // [2][threads / 64]
    int lanes;
    template <int N> __device__ __forceinline__ void of_part(float (&x)[N]) const {
#pragma unroll
        for (int n = 0; n < N; ++n) x[n] = lane_sum(x[n], lanes);
        if (lanes <= 64) return;
        const int waves = lanes >> 6, wave = threadIdx.x >> 6, first = wave & ~(waves - 1);
        __syncthreads();
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int n = 0; n < N; ++n) lds[wave * N + n] = x[n];
        __syncthreads();
#pragma unroll
        for (int n = 0; n < N; ++n) {
            float s = 0.f;
            for (int w = 0; w < waves; ++w) s += lds[(first + w) * N + n];
            x[n] = s;
        }
    }
    // over the `groups` parts of a row, `unit` the number of this thread's part in the workgroup
    template <int N> __device__ __forceinline__ void of_row(float (&x)[N], int groups, int unit, float* units) const {
        of_part(x);
        if (groups == 1) return;
        __syncthreads();
        if ((threadIdx.x & (lanes - 1)) == 0)
#pragma unroll
            for (int n = 0; n < N; ++n) units[unit * N + n] = x[n];
        __syncthreads();
        const int first = unit - unit % groups;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            float s = 0.f;
            for (int g = 0; g < groups; ++g) s += units[(first + g) * N + n];
            x[n] = s;
        }
    }
};

// What is read of one row, asked for while the row before is worked on.
template <typename E, bool AL, bool BACK> struct Row {
    using S = Slice<E, AL>;
    typename S::Raw x, y, gate, sum, next;
    float one;                              // the gate's value for the part
    unsigned row;
    bool here, live, work;                  // work: the workgroup's, whether any of its rows may count
    __device__ __forceinline__ void fetch(const ResidualArgs& a, S s, unsigned first, int slot, int slots, int group) {
        row = first + slot;
        here = first < a.rows && slot < slots && row < a.rows;
        live = here && a.live(row);
        work = slots > 1 || (first < a.rows && a.live(first));
        s.on = live;
        if (a.x) s.fetch((const E*)a.x + row * a.x_stride, x);
        if (a.y) s.fetch((const E*)a.y + row * a.y_stride, y);
        if (a.gate) {
            if (a.gate_part) one = live ? to_float(((const E*)a.gate)[row * a.gate_stride + group]) : 0.f;
            else s.fetch((const E*)a.gate + row * a.gate_stride, gate);
        }
        if constexpr (BACK) {
            if (a.sum) s.fetch((const E*)a.sum + row * a.sum_stride, sum);
            if (a.next) s.fetch((const E*)a.next + row * a.next_stride, next);
        }
    }
    // The gate opened: g = act(gate), d = act'(gate); ones without a gate.
    __device__ __forceinline__ void open_gate(const ResidualArgs& a, const S& s, float (&g)[EPT], float (&d)[EPT]) const {
        if (!a.gate) {
#pragma unroll
            for (int i = 0; i < EPT; ++i) { g[i] = 1.f; d[i] = 0.f; }
        } else if (a.gate_part) {
            float f[1] = {one}, slope[1];
            activate_all<E>(a.gate_act, f, f, slope);
#pragma unroll
            for (int i = 0; i < EPT; ++i) { g[i] = f[0]; d[i] = slope[0]; }
        } else {
            s.open(gate, g);
            activate_all<E>(a.gate_act, g, g, d);
        }
    }
};

// Wavefronts a SIMD: what registers allow where rows are read 16 bytes at a time, less by one than without a bound on them; more spill
// (8192 rows of 2048, half of them counting, bf16: gradient 72 us with two, 57 with three, 92 with four; 16384 rows of 1024 forward 41 us with
// four, 37 with five).
constexpr int wavefronts(bool al, int threads, bool back) { return threads == 1024 ? 4 : back ? (al ? 3 : 2) : (al ? 5 : 4); }

// ---- forward ---------------------------------------------------------------------------------------
template <typename E, bool AL, int NT> __global__ void __launch_bounds__(NT, wavefronts(AL, NT, false)) residual_kernel(ResidualArgs a) {
    constexpr bool KEEP = NT < 1024;        // the weights, between rows: 1024 threads have 128 registers each
    __shared__ float lds[2 * 16], units[2 * 1024];
    const int unit = threadIdx.x / a.lanes, group = unit % a.groups, slot = unit / a.groups, slots = (int)blockDim.x / (a.lanes * a.groups);
    Slice<E, AL> s{group * a.part, (int)threadIdx.x & (a.lanes - 1), a.lanes, a.part, false};
    const Sums sums{lds, a.lanes};
    float post[EPT], pre[EPT];
    s.on = slot < slots;
    if constexpr (KEEP) { s.load_weights(a.post, post); s.load_weights(a.pre, pre); }
    Row<E, AL, false> now, after;
    after.fetch(a, s, blockIdx.x * slots, slot, slots, group);
    for (unsigned first = blockIdx.x * slots; first < a.rows; first += gridDim.x * slots) {
        now = after;
        after.fetch(a, s, first + gridDim.x * slots, slot, slots, group);
        const unsigned row = now.row;
        const bool here = now.here, live = now.live;
        s.on = live;
        if constexpr (!KEEP) { s.load_weights(a.post, post); s.load_weights(a.pre, pre); }
        float h[EPT] = {}, f = 1.f;
        if (now.work) {                         // rows that do not count: 37 us become 33 at 8192 rows of 2048 with half of them, bf16
            if (a.x) {
                s.open(now.x, h);
#pragma unroll
                for (int i = 0; i < EPT; ++i) h[i] *= a.scale_x;
            }
            if (a.y) {
                float y[EPT], g[EPT], d[EPT];
                s.open(now.y, y);
                now.open_gate(a, s, g, d);
                float r = 1.f;
                if (a.eps_post > 0.f) {
                    float q[1] = {};
#pragma unroll
                    for (int i = 0; i < EPT; ++i) q[0] += y[i] * y[i];
                    sums.of_part(q);
                    r = 1.f / sqrtf(q[0] / a.part + a.eps_post);
                }
                r *= a.scale_y;
#pragma unroll
                for (int i = 0; i < EPT; ++i) h[i] += r * y[i] * (g[i] * post[i]);
            }
            if (a.next && a.eps_pre > 0.f) {
                float q[1] = {};
#pragma unroll
                for (int i = 0; i < EPT; ++i) q[0] += h[i] * h[i];
                sums.of_row(q, a.groups, unit, units);
                f = 1.f / sqrtf(q[0] / a.dim + a.eps_pre);
            }
        }
        s.on = here;
        if (a.sum) {
            float out[EPT];
#pragma unroll
            for (int i = 0; i < EPT; ++i) out[i] = live ? h[i] : 0.f;
            s.store((E*)a.sum + row * a.sum_stride, out);
        }
        if (a.next) {
#pragma unroll
            for (int i = 0; i < EPT; ++i) h[i] = live ? h[i] * (f * pre[i]) : 0.f;
            s.store((E*)a.next + row * a.next_stride, h);
        }
    }
}

// ---- gradient --------------------------------------------------------------------------------------
template <typename E, bool AL, int NT> __global__ void __launch_bounds__(NT, wavefronts(AL, NT, true)) residual_back_kernel(ResidualArgs a) {
    constexpr bool KEEP = NT < 1024;        // the weights, between rows: 1024 threads have 128 registers each
    __shared__ float lds[2 * 16], units[2 * 1024];
    const int unit = threadIdx.x / a.lanes, group = unit % a.groups, slot = unit / a.groups, slots = (int)blockDim.x / (a.lanes * a.groups);
    Slice<E, AL> s{group * a.part, (int)threadIdx.x & (a.lanes - 1), a.lanes, a.part, false};
    const Sums sums{lds, a.lanes};
    float post[EPT], pre[EPT], dpost[EPT] = {}, dpre[EPT] = {};
    s.on = slot < slots;
    if constexpr (KEEP) { s.load_weights(a.post, post); s.load_weights(a.pre, pre); }
    const float over_part = 1.f / a.part, over_dim = 1.f / a.dim;
    Row<E, AL, true> now, after;
    after.fetch(a, s, blockIdx.x * slots, slot, slots, group);
    for (unsigned first = blockIdx.x * slots; first < a.rows; first += gridDim.x * slots) {
        now = after;
        after.fetch(a, s, first + gridDim.x * slots, slot, slots, group);
        const unsigned row = now.row;
        const bool here = now.here;
        s.on = now.live;
        if (!now.work) {                        // 57 us become 48 there
            const float zero[EPT] = {};
            s.on = here;
            if (a.dx) s.store((E*)a.dx + row * a.dx_stride, zero);
            if (a.dy) s.store((E*)a.dy + row * a.dy_stride, zero);
            if (a.dgate) {
                if (!a.gate_part) s.store((E*)a.dgate + row * a.dgate_stride, zero);
                else if (here && s.lane == 0) ((E*)a.dgate)[row * a.dgate_stride + group] = from_float<E>(0.f);
            }
            continue;
        }
        if constexpr (!KEEP) { s.load_weights(a.post, post); s.load_weights(a.pre, pre); }
        float y[EPT] = {}, g[EPT], slope[EPT], h[EPT] = {}, dh[EPT] = {};
        float r = 1.f;
        if (a.x) {
            s.open(now.x, h);
#pragma unroll
            for (int i = 0; i < EPT; ++i) h[i] *= a.scale_x;
        }
        if (a.sum) s.open(now.sum, dh);
        if (a.y) {
            s.open(now.y, y);
            now.open_gate(a, s, g, slope);
            if (a.eps_post > 0.f) {
                float q[1] = {};
#pragma unroll
                for (int i = 0; i < EPT; ++i) q[0] += y[i] * y[i];
                sums.of_part(q);
                r = 1.f / sqrtf(q[0] * over_part + a.eps_post);
            }
#pragma unroll
            for (int i = 0; i < EPT; ++i) {
                y[i] *= r;                                          // the normed y from here on
                h[i] += a.scale_y * y[i] * (g[i] * post[i]);
            }
        }
        // rows that do not count, beside others that do: weights that are not finite must not make anything of their zeros
        if (!s.on)
#pragma unroll
            for (int i = 0; i < EPT; ++i) h[i] = 0.f;
        if (a.next) {
            float du[EPT];
            s.open(now.next, du);
            float f = 1.f, c = 0.f;
            if (a.eps_pre > 0.f) {
                float q[2] = {};
#pragma unroll
                for (int i = 0; i < EPT; ++i) { q[0] += h[i] * h[i]; q[1] += du[i] * pre[i] * h[i]; }
                sums.of_row(q, a.groups, unit, units);
                f = 1.f / sqrtf(q[0] * over_dim + a.eps_pre);
                c = q[1] * over_dim * f * f;
            }
#pragma unroll
            for (int i = 0; i < EPT; ++i) {
                dpre[i] += du[i] * (h[i] * f);
                dh[i] += f * (du[i] * pre[i] - c * h[i]);
            }
        }
        const bool live = s.on;
        if (!live)
#pragma unroll
            for (int i = 0; i < EPT; ++i) dh[i] = 0.f;
        if (a.dx) {
            float out[EPT];
#pragma unroll
            for (int i = 0; i < EPT; ++i) out[i] = live ? a.scale_x * dh[i] : 0.f;
            s.on = here;
            s.store((E*)a.dx + row * a.dx_stride, out);
            s.on = live;
        }
        if (!a.y) continue;
        float dgate = 0.f, mean[1] = {};
#pragma unroll
        for (int i = 0; i < EPT; ++i) {
            const float dz = a.scale_y * dh[i], zy = dz * y[i];
            dpost[i] += zy * g[i];
            slope[i] *= zy * post[i];                               // the gate's gradient
            dgate += slope[i];
            dh[i] = dz * (g[i] * post[i]);                          // that of the normed y
            mean[0] += dh[i] * y[i];
        }
        if (a.dgate) {
            if (a.gate_part) {
                float q[1] = {dgate};
                sums.of_part(q);
                if (here && s.lane == 0) ((E*)a.dgate)[row * a.dgate_stride + group] = from_float<E>(live ? q[0] : 0.f);
            } else {
#pragma unroll
                for (int i = 0; i < EPT; ++i) slope[i] = live ? slope[i] : 0.f;
                s.on = here;
                s.store((E*)a.dgate + row * a.dgate_stride, slope);
                s.on = live;
            }
        }
        if (a.dy) {
            float c = 0.f;
            if (a.eps_post > 0.f) {
                sums.of_part(mean);
                c = mean[0] * over_part;
            }
#pragma unroll
            for (int i = 0; i < EPT; ++i) dh[i] = live ? r * (dh[i] - c * y[i]) : 0.f;
            s.on = here;
            s.store((E*)a.dy + row * a.dy_stride, dh);
        }
    }
    if (!a.partial) return;
    // the workgroup's sums, over its rows' slots in order (slots * dim is at most 256 * 8 where there are several)
    float* p = a.partial + (int64_t)blockIdx.x * 2 * a.dim;
    s.on = slot < slots;
    if (slots == 1) {
        s.store_floats(p, dpost);
        s.store_floats(p + a.dim, dpre);
        return;
    }
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        __syncthreads();
        if (s.on) s.store_floats(units + slot * a.dim, which ? dpre : dpost);
        __syncthreads();
        for (int col = threadIdx.x; col < a.dim; col += blockDim.x) {
            float sum = 0.f;
            for (int i = 0; i < slots; ++i) sum += units[i * a.dim + col];
            p[which * a.dim + col] = sum;
        }
    }
}
// Sums over the workgroups, in order within 32 stretches of it and over those: 64 columns a workgroup, half a wavefront a stretch.
__global__ void __launch_bounds__(1024) residual_join_kernel(const float* partial, int parts, int dim, float* dpost, float* dpre) {
    __shared__ float2 sums[32][32];
    const int stretch = threadIdx.x >> 5, each = (parts + 31) / 32, from = stretch * each, to = min(from + each, parts);
    const int col = blockIdx.x * 64 + (threadIdx.x & 31) * 2;           // 2 * dim columns: pairs are whole
    float2 s = {0.f, 0.f};
    if (col < 2 * dim) {
#pragma unroll 8
        for (int p = from; p < to; ++p) {
            const float2 x = *(const float2*)(partial + (int64_t)p * 2 * dim + col);
            s.x += x.x;
            s.y += x.y;
        }
    }
    sums[stretch][threadIdx.x & 31] = s;
    __syncthreads();
    const int mine = blockIdx.x * 64 + threadIdx.x;
    if (threadIdx.x >= 64 || mine >= 2 * dim) return;
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) t += ((const float*)sums[i])[threadIdx.x];
    if (mine < dim) { if (dpost) dpost[mine] = t; }
    else if (dpre) dpre[mine - dim] = t;
}

// ---- host ------------------------------------------------------------------------------------------
// Lanes a part: a power of two.
int part_lanes(const pql_residual_shape& s) {
    int lanes = 1;
    while (lanes * EPT < s.dim / s.groups) lanes *= 2;
    return lanes;
}
bool finite(float x) { return x - x == 0.f; }
bool residual_ok(const pql_residual_shape& s) {
    const bool ok = s.batch >= 0 && s.steps >= 0 && (double)s.batch * s.steps < 2147483648.0 && s.dim >= 1 && s.dim <= PQL_RESIDUAL_MAX_DIM &&
           s.groups >= 1 && s.groups <= PQL_RESIDUAL_MAX_GROUPS && s.dim % s.groups == 0 && (s.dtype == PQL_F32 || s.dtype == PQL_BF16) &&
           (s.gate_cols == 0 || s.gate_cols == s.groups || s.gate_cols == s.dim) && s.gate_act >= PQL_ACT_NONE && s.gate_act <= PQL_ACT_RELU &&
           s.eps_post >= 0.f && s.eps_pre >= 0.f && finite(s.eps_post) && finite(s.eps_pre) && finite(s.scale_x) && finite(s.scale_y);
    return ok && part_lanes(s) * s.groups * EPT <= PQL_RESIDUAL_MAX_DIM;
}
unsigned residual_rows(const pql_residual_shape& s) { return (unsigned)((int64_t)s.batch * s.steps); }

struct ResidualPlan { int lanes, threads, slots; unsigned grid; };
// As many workgroups as run at a time: they stay for several rows.
ResidualPlan residual_plan(const pql_residual_shape& s, bool back, bool al) {
    ResidualPlan p{};
    p.lanes = part_lanes(s);
    const int threads = p.lanes * s.groups;
    p.threads = threads <= 256 ? 256 : (threads + 63) / 64 * 64;
    p.slots = p.threads / threads;
    const unsigned rows = residual_rows(s), all = (rows + p.slots - 1) / p.slots;
    const int of = p.threads <= 256 ? 256 : p.threads <= 512 ? 512 : 1024;
    const unsigned most = 256u * (wavefronts(al, of, back) * 256 / of);
    p.grid = all < most ? all : most;
    return p;
}
// An output in the place of an input lies row on row.
bool same_place(const pql_rows& to, const pql_rows& from, int64_t rows) { return !to.data || to.data != from.data || to.stride == from.stride || rows <= 1; }
int32_t residual_check(pql_ctx* c, const pql_residual_shape* s, const pql_residual_input* in, const pql_rows* sum, const pql_rows* next, bool back) {
    if (!s || !in || !sum || !next) return ctx_fail(c, PQL_ERR_NULL, "pql_residual: null pointer");
    if (!residual_ok(*s)) return ctx_fail(c, PQL_ERR_INVALID_ARG, "pql_residual: bad shape");
    const int64_t rows = residual_rows(*s);
    auto bad = [&](const pql_rows& r, int cols, bool write) { return r.data && !(write ? own_rows(r, rows, cols) : read_rows(r)); };
    if (bad(in->x, s->dim, false) || bad(in->y, s->dim, false) || bad(in->gate, s->gate_cols, false) || bad(*sum, s->dim, !back) ||
        bad(*next, s->dim, !back))
        return ctx_fail(c, PQL_ERR_INVALID_ARG, "pql_residual: bad stride");
    if (!back && (!same_place(*sum, in->x, rows) || !same_place(*sum, in->y, rows) || !same_place(*next, in->y, rows)))
        return ctx_fail(c, PQL_ERR_INVALID_ARG, "pql_residual: an output in an input's place needs its stride");
    if (rows == 0 && !back) return PQL_OK;
    if (rows > 0 && ((!in->x.data && !in->y.data) || (!sum->data && !next->data) || (s->gate_cols > 0 && in->y.data && !in->gate.data)))
        return ctx_fail(c, PQL_ERR_NULL, "pql_residual: null pointer");
    const size_t e = elem_size(s->dtype);
    if (off_by(in->x.data, e) || off_by(in->y.data, e) || off_by(in->gate.data, e) || off_by(sum->data, e) || off_by(next->data, e) ||
        off_by(in->post, 4) || off_by(in->pre, 4) || off_by(in->lengths, 4))
        return ctx_fail(c, PQL_ERR_ALIGNMENT, "pql_residual: misaligned pointer");
    return PQL_OK;
}
ResidualArgs residual_args(const pql_residual_shape& s, const pql_residual_input& in, const pql_rows& sum, const pql_rows& next) {
    ResidualArgs a{};
    a.live = {in.lengths, (unsigned)s.steps};
    a.rows = residual_rows(s);
    a.dim = s.dim; a.groups = s.groups; a.part = s.dim / s.groups; a.lanes = part_lanes(s);
    a.gate_act = s.gate_act; a.gate_part = s.gate_cols != s.dim;
    a.eps_post = s.eps_post; a.eps_pre = s.eps_pre; a.scale_x = s.scale_x; a.scale_y = s.scale_y;
    a.x = in.x.data; a.x_stride = in.x.stride;
    a.y = in.y.data; a.y_stride = in.y.stride;
    if (s.gate_cols > 0 && in.y.data) { a.gate = in.gate.data; a.gate_stride = in.gate.stride; }
    a.post = in.post; a.pre = in.pre;
    a.sum = sum.data; a.sum_stride = sum.stride;
    a.next = next.data; a.next_stride = next.stride;
    return a;
}
// Whether every tensor of elements can be read and written 16 bytes at a time.
bool residual_aligned(const pql_residual_shape& s, const ResidualArgs& a) {
    const int e = elem_size(s.dtype);
    if (a.part * e % ROW_ALIGN) return false;
    auto fits = [&](const void* p, int64_t stride) { return !p || rows_aligned({(void*)p, stride}, s.dtype); };
    return fits(a.x, a.x_stride) && fits(a.y, a.y_stride) && (a.gate_part || fits(a.gate, a.gate_stride)) && fits(a.sum, a.sum_stride) &&
           fits(a.next, a.next_stride) && fits(a.dx, a.dx_stride) && fits(a.dy, a.dy_stride) && (a.gate_part || fits(a.dgate, a.dgate_stride));
}
template <typename E, bool AL> hipError_t residual_launch(const ResidualArgs& a, const ResidualPlan& p, bool back, hipStream_t st) {
    const double size = (double)a.rows * a.dim * sizeof(E);
    const double in = size * (!!a.x + !!a.y + (a.gate && !a.gate_part)), out = size * (!!a.sum + !!a.next);
    const ProfSlot ps = prof_slot();
    if (!back) {
        if (p.threads <= 256) PQL_LAUNCH(ps, (residual_kernel<E, AL, 256>), dim3(p.grid), dim3(p.threads), 0, st, a);
        else if (p.threads <= 512) PQL_LAUNCH(ps, (residual_kernel<E, AL, 512>), dim3(p.grid), dim3(p.threads), 0, st, a);
        else PQL_LAUNCH(ps, (residual_kernel<E, AL, 1024>), dim3(p.grid), dim3(p.threads), 0, st, a);
        prof_commit(ps, KID_RESIDUAL, 0.0, in + out);
    } else {
        if (p.threads <= 256) PQL_LAUNCH(ps, (residual_back_kernel<E, AL, 256>), dim3(p.grid), dim3(p.threads), 0, st, a);
        else if (p.threads <= 512) PQL_LAUNCH(ps, (residual_back_kernel<E, AL, 512>), dim3(p.grid), dim3(p.threads), 0, st, a);
        else PQL_LAUNCH(ps, (residual_back_kernel<E, AL, 1024>), dim3(p.grid), dim3(p.threads), 0, st, a);
        prof_commit(ps, KID_RESIDUAL_BACK, 0.0, in + out + size * (!!a.dx + !!a.dy + (a.dgate && !a.gate_part)));
    }
    return hipGetLastError();
}
hipError_t residual_run(const pql_residual_shape& s, const ResidualArgs& a, bool back, hipStream_t st) {
    const bool al = residual_aligned(s, a);
    const ResidualPlan p = residual_plan(s, back, al);
    if (s.dtype == PQL_F32) return al ? residual_launch<float, true>(a, p, back, st) : residual_launch<float, false>(a, p, back, st);
    return al ? residual_launch<bf16_t, true>(a, p, back, st) : residual_launch<bf16_t, false>(a, p, back, st);
}

}  // namespace
}  // namespace pql

using namespace pql;

extern "C" {

int32_t pql_residual_forward(pql_ctx* c, const pql_residual_shape* s, const pql_residual_input* in, const pql_rows* sum, const pql_rows* next, void* stream) {
    if (!c) return PQL_ERR_NULL;
    const int32_t rc = residual_check(c, s, in, sum, next, false);
    if (rc != PQL_OK || residual_rows(*s) == 0) return rc;
    const hipError_t e = residual_run(*s, residual_args(*s, *in, *sum, *next), false, (hipStream_t)stream);
    return e == hipSuccess ? PQL_OK : ctx_fail(c, PQL_ERR_HIP, "pql_residual_forward", e);
}

int64_t pql_residual_workspace_bytes(const pql_residual_shape* s) {
    if (!s) return PQL_ERR_NULL;
    if (!residual_ok(*s)) return PQL_ERR_INVALID_ARG;
    return (int64_t)to256((size_t)residual_plan(*s, true, true).grid * 2 * s->dim * 4);         // fewer workgroups where rows are not aligned
}

int32_t pql_residual_backward(pql_ctx* c, const pql_residual_shape* s, const pql_residual_input* in, const pql_rows* sum_grad,
                              const pql_rows* next_grad, const pql_residual_grad* g, void* workspace, void* stream) {
    if (!c) return PQL_ERR_NULL;
    if (!g) return ctx_fail(c, PQL_ERR_NULL, "pql_residual_backward: null pointer");
    const int32_t rc = residual_check(c, s, in, sum_grad, next_grad, true);
    if (rc != PQL_OK) return rc;
    const int64_t rows = residual_rows(*s);
    const size_t e = elem_size(s->dtype);
    auto bad = [&](const pql_rows& r, int cols) { return r.data && !own_rows(r, rows, cols); };
    if (bad(g->x, s->dim) || bad(g->y, s->dim) || bad(g->gate, s->gate_cols)) return ctx_fail(c, PQL_ERR_INVALID_ARG, "pql_residual_backward: bad stride");
    if (!same_place(g->x, *sum_grad, rows) || !same_place(g->y, *next_grad, rows))
        return ctx_fail(c, PQL_ERR_INVALID_ARG, "pql_residual_backward: a gradient in another's place needs its stride");
    if (rows > 0 && ((g->x.data && !in->x.data) || ((g->y.data || g->post) && !in->y.data) || (g->gate.data && (!in->y.data || s->gate_cols == 0)) ||
                     (g->pre && !next_grad->data)))
        return ctx_fail(c, PQL_ERR_INVALID_ARG, "pql_residual_backward: gradient of what is not there");
    const bool weights = g->post || g->pre;
    if (weights && rows > 0 && !workspace) return ctx_fail(c, PQL_ERR_NULL, "pql_residual_backward: null workspace");
    if (off_by(g->x.data, e) || off_by(g->y.data, e) || off_by(g->gate.data, e) || off_by(g->post, 4) || off_by(g->pre, 4) || off_by(workspace, 256))
        return ctx_fail(c, PQL_ERR_ALIGNMENT, "pql_residual_backward: misaligned pointer");
    const hipStream_t st = (hipStream_t)stream;
    hipError_t err = hipSuccess;
    unsigned parts = 0;
    if (rows > 0) {
        ResidualArgs a = residual_args(*s, *in, *sum_grad, *next_grad);
        a.dx = g->x.data; a.dx_stride = g->x.stride;
        a.dy = g->y.data; a.dy_stride = g->y.stride;
        a.dgate = g->gate.data; a.dgate_stride = g->gate.stride;
        if (weights) a.partial = (float*)workspace;
        parts = residual_plan(*s, true, residual_aligned(*s, a)).grid;
        err = residual_run(*s, a, true, st);
    }
    if (err == hipSuccess && weights) {
        const ProfSlot ps = prof_slot();
        PQL_LAUNCH(ps, residual_join_kernel, dim3((2 * s->dim + 63) / 64), dim3(1024), 0, st, (const float*)workspace,
                   (int)parts, (int)s->dim, g->post, g->pre);
        prof_commit(ps, KID_RESIDUAL_JOIN, 0.0, 8.0 * parts * s->dim);
        err = hipGetLastError();
    }
    return err == hipSuccess ? PQL_OK : ctx_fail(c, PQL_ERR_HIP, "pql_residual_backward", err);
}

}  // extern "C"
