// The gated feed-forward block of few rows (include/pql_block.h): the weights are read once and bound the call.
//
// A workgroup takes 16 outputs of a projection and all rows, or a share of them, its wavefronts each a part of the contraction;
// weights go from memory to the matrix instructions' registers without LDS between (nothing of them is used twice), 16 bytes a lane,
// the rows come from the caches.  Two launches: both projections, the activation and the product, then the last projection.  In bf16
// the product between them is kept as two bf16 terms (16 bits): a second product on weights that are there costs no time.  One token
// through a block of 4096 and 16384 in bf16 takes 84 us, 4.8 TB/s; 64 through one of 256 and 1024 in fp32 10 us, two launches.  In between
// the rows' way from the caches bounds it: they are read again for each 16 outputs.
#include "pql_ffn_internal.h"

namespace pql {
namespace {

// Wavefronts of a workgroup (one token through a block of 4096 and 16384 in bf16: 85.6 us a call, with 4 of them 89, with 16 90; twice as
// many steps ahead change nothing).
constexpr int WAVES = 8, NT = 64 * WAVES;
// Sixteens of rows share a workgroup, that reads its weights once for all of them, where that leaves FILL workgroups or the weights are
// more than CACHED bytes; others have one for each, or for two, and read weights again, from the caches (the last holds 256 MiB).  us a
// call of 64 rows in fp32, shared / by this rule / never shared: 256 and 1024 22 / 11 / 11, 1000 and 4000 67 / 37 / 47, 2048 and 8192
// 179 / 136 / 177; FILL of 96 or 384 instead: 48 or 41 and 179 or 146.  More than CACHED, 4096 and 16384: 491, never shared 768.
constexpr int FILL = 192;
constexpr double CACHED = 128 << 20;

// ---- operands: lane l holds row l % 16, and CHUNK elements of the contraction from CHUNK (l / 16) on, of 4 CHUNK a step ----
template <typename E> constexpr int M_TERMS = sizeof(E) == 2 ? 2 : 1;     // of the product between the two launches
template <typename E> struct Frag;
template <> struct Frag<bf16_t> {
    static constexpr int CHUNK = 8;
    bf16x8 v;
    __device__ __forceinline__ void zero() { v = bf16x8{}; }
    __device__ __forceinline__ void set(int i, bf16_t x) { v[i] = x; }
    __device__ __forceinline__ void load(const bf16_t* p) { v = __builtin_bit_cast(bf16x8, *(const uint4*)p); }
};
template <> struct Frag<float> {
    static constexpr int CHUNK = 4;
    floatx4 v;
    __device__ __forceinline__ void zero() { v = floatx4{}; }
    __device__ __forceinline__ void set(int i, float x) { v[i] = x; }
    __device__ __forceinline__ void load(const float* p) { v = *(const floatx4*)p; }
};
__device__ __forceinline__ void product(floatx4& c, const Frag<bf16_t>& a, const Frag<bf16_t>& b) {
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, b.v, c, 0, 0, 0);
}
__device__ __forceinline__ void product(floatx4& c, const Frag<float>& a, const Frag<float>& b) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[i], b.v[i], c, 0, 0, 0);
}
// Elements [k, k + CHUNK) of a row of `size`; nothing of a row that is not there.
template <typename E, bool AL> __device__ __forceinline__ Frag<E> fetch(const E* row, bool there, int k, int size) {
    Frag<E> f;
    f.zero();
    if constexpr (AL) {
        if (there && k < size) f.load(row + k);
    } else {
#pragma unroll
        for (int i = 0; i < Frag<E>::CHUNK; ++i)
            if (there && k + i < size) f.set(i, row[k + i]);
    }
    return f;
}

// W [outputs][size] against 16 T rows.  GATED: W and W2 are both projections.
template <typename E, int T, bool AL, bool GATED> __global__ void __launch_bounds__(NT) ffn_rows_kernel(FfnRowsArgs a) {
    constexpr int CHUNK = Frag<E>::CHUNK, STEP = 4 * CHUNK, M = GATED ? 2 : 1, AHEAD = 4;
    __shared__ floatx4 sums[WAVES][M * T][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, k0 = (lane >> 4) * CHUNK;
    const int outputs = GATED ? a.hidden : a.dim, size = GATED ? a.dim : a.hidden;
    const int o = blockIdx.x * 16 + r;
    const E* w[M];
    if constexpr (GATED) {
        w[0] = (const E*)a.gate + min(o, outputs - 1) * a.gate_stride;
        w[M - 1] = (const E*)a.up + min(o, outputs - 1) * a.up_stride;
    } else {
        w[0] = (const E*)a.down + min(o, outputs - 1) * a.down_stride;
    }
    const E* x[T];
    bool live[T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
        const int n = (blockIdx.y * T + t) * 16 + r;
        live[t] = n < a.rows && a.live(n);
        x[t] = GATED ? (const E*)a.x + (int64_t)(live[t] ? n : 0) * a.x_stride : (const E*)a.m + (int64_t)(live[t] ? n : 0) * a.m_stride;
    }
    constexpr int X = GATED ? 1 : M_TERMS<E>;
    floatx4 acc[M][T] = {};
    // the wavefronts take turns of AHEAD steps, all of whose loads go out together
    for (int k = wave * AHEAD * STEP; k < size; k += WAVES * AHEAD * STEP) {
        Frag<E> wf[AHEAD][M], xf[AHEAD][X][T];
#pragma unroll
        for (int s = 0; s < AHEAD; ++s) {
#pragma unroll
            for (int m = 0; m < M; ++m) wf[s][m] = fetch<E, AL>(w[m], true, k + s * STEP + k0, size);
#pragma unroll
            for (int q = 0; q < X; ++q)
#pragma unroll
                for (int t = 0; t < T; ++t) xf[s][q][t] = fetch<E, AL>(x[t] + q * a.m_plane, live[t], k + s * STEP + k0, size);
        }
#pragma unroll
        for (int s = 0; s < AHEAD; ++s)
#pragma unroll
            for (int m = 0; m < M; ++m)
#pragma unroll
                for (int t = 0; t < T; ++t)
#pragma unroll
                    for (int q = X - 1; q >= 0; --q) product(acc[m][t], wf[s][m], xf[s][q][t]);
    }
    settle_products();
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int t = 0; t < T; ++t) sums[wave][m * T + t][lane] = acc[m][t];
    __syncthreads();
    // results: column l % 16 is the row, outputs 4 (l / 16) .. + 3; one of them a thread
    for (int i = threadIdx.x; i < T * 256; i += NT) {
        const int t = i >> 8, l = i >> 2 & 63, e = i & 3, n = (blockIdx.y * T + t) * 16 + (l & 15), out = blockIdx.x * 16 + (l >> 4) * 4 + e;
        float s[M];
#pragma unroll
        for (int m = 0; m < M; ++m) {
            s[m] = 0.f;
#pragma unroll
            for (int v = 0; v < WAVES; ++v) s[m] += sums[v][m * T + t][l][e];
        }
        if (n >= a.rows || out >= outputs) continue;
        if constexpr (!GATED && M_TERMS<E> == 2) {
            // an infinite weight met both terms of m, the second of which is zero or of either sign: m itself decides
            if (__builtin_expect(s[0] != s[0], 0)) {
                const E *m = (const E*)a.m + (int64_t)n * a.m_stride, *down = (const E*)a.down + out * a.down_stride;
                float sum = 0.f;
                for (int k = 0; k < size && sum == sum; ++k) sum = fmaf(to_float(m[k]) + to_float(m[a.m_plane + k]), to_float(down[k]), sum);
                s[0] = sum;
            }
        }
        if constexpr (GATED) {
            float f[1] = {s[0]}, d[1];
            activate_all<E>(a.act, f, f, d);
            E* p = (E*)a.m + (int64_t)n * a.m_stride + out;
            const float m = f[0] * s[M - 1];
            const E high = from_float<E>(m);
            p[0] = high;
            // an infinite term has no rest
            if constexpr (M_TERMS<E> == 2) p[a.m_plane] = from_float<E>(fabsf(to_float(high)) < __builtin_inff() ? m - to_float(high) : 0.f);
        } else {
            ((E*)a.out)[(int64_t)n * a.out_stride + out] = from_float<E>(a.live(n) ? s[0] : 0.f);
        }
    }
}

template <typename E, int T, bool GATED> void launch(const FfnRowsArgs& a, bool al, int y, hipStream_t st) {
    const int outputs = GATED ? a.hidden : a.dim, size = GATED ? a.dim : a.hidden;
    const dim3 grid((outputs + 15) / 16, y);
    const ProfSlot ps = prof_slot();
    if (al) PQL_LAUNCH(ps, (ffn_rows_kernel<E, T, true, GATED>), grid, dim3(NT), 0, st, a);
    else PQL_LAUNCH(ps, (ffn_rows_kernel<E, T, false, GATED>), grid, dim3(NT), 0, st, a);
    prof_commit(ps, KID_FFN_ROWS, 2.0 * (GATED ? 2 : 1) * a.rows * outputs * size, (double)(GATED ? 2 : 1) * outputs * size * sizeof(E));
}
template <typename E, bool GATED> void launch_rows(const FfnRowsArgs& a, bool al, hipStream_t st) {
    const int tiles = (a.rows + 15) / 16, groups = ((GATED ? a.hidden : a.dim) + 15) / 16;
    int each = tiles == 3 ? 4 : tiles;          // sixteens of rows of a workgroup
    if ((GATED ? 2.0 : 1.0) * a.dim * a.hidden * sizeof(E) <= CACHED)
        while (each > 1 && groups * ((tiles + each - 1) / each) < FILL) each /= 2;
    const int y = (tiles + each - 1) / each;
    if (each == 1) launch<E, 1, GATED>(a, al, y, st);
    else if (each == 2) launch<E, 2, GATED>(a, al, y, st);
    else launch<E, 4, GATED>(a, al, y, st);
}
template <typename E> hipError_t rows_of(const FfnRowsArgs& a, hipStream_t st) {
    const int32_t dt = sizeof(E) == 4 ? PQL_F32 : PQL_BF16;
    const int v = VEC_OF<E>;
    auto fits = [&](const void* p, int64_t stride) { return rows_aligned({(void*)p, stride}, dt); };
    launch_rows<E, true>(a, a.dim % v == 0 && fits(a.x, a.x_stride) && fits(a.gate, a.gate_stride) && fits(a.up, a.up_stride), st);
    launch_rows<E, false>(a, a.hidden % v == 0 && fits(a.m, a.m_stride) && fits(a.down, a.down_stride), st);
    return hipGetLastError();
}

}  // namespace

hipError_t ffn_rows_launch(const FfnRowsArgs& a, int32_t dtype, hipStream_t st) {
    return dtype == PQL_F32 ? rows_of<float>(a, st) : rows_of<bf16_t>(a, st);
}

}  // namespace pql
