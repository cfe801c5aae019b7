// The gated feed-forward block (include/pql_block.h), products of row tiles:
//     a = x G^T,  b = x U^T,  m = act(a) b,  out = m D^T,
//     dm = dout D,  da = dm b act'(a),  db = dm act(a),  dx = da G + db U,  dG = da^T x,  dU = db^T x,  dD = dout^T m.
//
// All products run on the bf16 matrix instructions with sums in fp32.  fp32 values are three bf16 terms each (24 bits, exactly),
// of whose nine products the three below 2^-24 are left out: six products a pair.  Operands lie in memory as planes, one for
// each term; bf16 tensors whose rows start on 16-byte boundaries are used where they are.
//
// Rows that count are packed together first where sequences have lengths, so that no work is done for the others.
//
// A workgroup computes one tile of the result.  Tiles of both operands go from memory to LDS without registers between, one
// step ahead of the products, and are laid out there so that neither the contiguous reads (operands whose contraction runs along
// a row) nor the transposing ones (along a column) meet bank conflicts: no operand is ever transposed in memory.
#include "pql_ffn_internal.h"

namespace pql {
namespace {

typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) shortx4 lds_shortx4;

// Terms of a value, elements of the contraction a step, steps in LDS at a time.
template <typename E> struct Mode;
template <> struct Mode<bf16_t> { static constexpr int TERMS = 1, BK = 64, STAGES = 2; };
template <> struct Mode<float> { static constexpr int TERMS = 3, BK = 32, STAGES = 3; };
constexpr int BIG_TILES = 192;
constexpr int NOWHERE = 0x7fffff00;             // an offset behind every buffer: reads give zeros

// One operand: rows of a matrix, `plane` elements from one term's to the next.
struct FfnOperand { const bf16_t* p; int64_t stride, plane; };
// ROWS: the contraction runs along the rows (element (i, k) at i * stride + k); otherwise along the columns (k * stride + i).
struct FfnProblem { FfnOperand a[2], b[2]; int m, n; void* out; int64_t out_stride; };
enum Epilogue : int { EPI_GATED, EPI_BACK, EPI_OUT, EPI_PART };

struct FfnArgs {
    FfnProblem prob[3];
    int k, segments;                            // length of the contraction, of each of `segments` pairs of operands
    const int* count;                           // rows that count, NULL: all
    int count_is_k;                             // whether they are the contraction or the rows of the result
    int splits;                                 // parts of the contraction
    float* part;                                // [problem][splits][m][n] sums of the parts
    int64_t part_stride;                        // of a problem
    const int* map;                             // packed row -> row of the output, NULL: the same
    int act;
    // gated, back: [row][hidden_p]
    int hidden_p;
    float *va, *vb;                             // a and b
    bf16_t *m, *da, *db;
    int64_t m_plane;
};

// 16 bytes of every lane from the buffer to LDS, lane after lane; `lds` and the buffer are the wavefront's.  In text, so that the
// compiler does not wait for it before each transposing read of other parts of LDS, as it does behind its own instruction (there is no
// result in registers: what is in flight is counted and waited for below).
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uintx4 buffer_of(const void* p, int bytes) {
    const uint64_t at = (uint64_t)p;
    return uintx4{(unsigned)at, (unsigned)(at >> 32) & 0xffffu, (unsigned)bytes, 0x00020000u};
}
__device__ __forceinline__ void load_to_lds(uintx4 buffer, unsigned lds, int offset) {
#ifdef __HIP_DEVICE_COMPILE__
    // m0 is the compiler's own and kept; five cycles lie between an SGPR that a vector instruction has written and its use here
    unsigned m0;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 2\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds\n\ts_mov_b32 m0, %0"
                 : "=&s"(m0) : "s"(lds), "v"(offset), "s"(buffer) : "memory");
#endif
}
__device__ __forceinline__ unsigned lds_address(const char* p) { return (unsigned)(uintptr_t)(__attribute__((address_space(3))) const char*)p; }

// ---- tiles in LDS -------------------------------------------------------------------------------------
// ALONG (the contraction runs along the rows in memory): [I][BK elements], BK / 8 granules of 16 bytes a row, granule g of row i at
// place g ^ along(i).  The reads take one granule from each of 16 rows.
// ACROSS: [BK][I elements], I / 8 granules a row k, granule g at place g ^ across(k): the transposing read of 16 lanes takes 32 bytes
// from each of four rows.
template <int BK> __device__ __forceinline__ int along(int i) { return BK == 64 ? i & 7 : (i >> 1 & 3) ^ (i >> 3 & 1); }
__device__ __forceinline__ int across(int k) { return (k & 3) << 1 | (k >> 3 & 1) << 3; }
template <int I, bool ALONG, int WAVES, int BK> struct Tile {
    static constexpr int BYTES = I * BK * 2, LOADS = BYTES / 1024 / WAVES, PER_ROW = ALONG ? BK / 8 : I / 8, ROWS_A_LOAD = 64 / PER_ROW;
    static_assert(LOADS * 1024 * WAVES == BYTES, "whole loads for every wavefront");
    int at[LOADS];                              // byte offsets of this lane's granules from the tile's corner
    int first_k;                                // ALONG: the first element of its granules along the contraction

    __device__ __forceinline__ void init(int wave, int lane, int64_t stride) {
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const int row = (wave * LOADS + j) * ROWS_A_LOAD + lane / PER_ROW, place = lane % PER_ROW;
            const int g = place ^ (ALONG ? along<BK>(row) : across(row));
            at[j] = row * (int)stride * 2 + g * 16;
        }
        first_k = 8 * ((lane % PER_ROW) ^ along<BK>(lane / PER_ROW));          // the same for all loads: of 8 or 16 rows each
    }
    // From the corner p, where `bytes` bytes can be read; `left` elements of the contraction are.
    __device__ __forceinline__ void load(char* lds, int wave, const bf16_t* p, int bytes, int left) const {
        const uintx4 rs = buffer_of(p, bytes);
        const unsigned to = __builtin_amdgcn_readfirstlane(lds_address(lds)) + wave * LOADS * 1024;
#pragma unroll
        for (int j = 0; j < LOADS; ++j) load_to_lds(rs, to + j * 1024, !ALONG || first_k < left ? at[j] : NOWHERE);
    }
};
// A wavefront's operands of 16 x 16 x 32 products: lane l holds row l % 16 of 16, elements 8 (l / 16) .. + 7 of 32.
template <int I, bool ALONG, int BK> struct Reader {
    int at[ALONG ? BK / 32 : 4];
    __device__ __forceinline__ void init(int first, int lane) {         // first: the wavefront's first row, a multiple of 32
        if constexpr (ALONG) {
#pragma unroll
            for (int kk = 0; kk < BK / 32; ++kk) at[kk] = (first + (lane & 15)) * BK * 2 + (((kk * 4 + (lane >> 4)) ^ along<BK>(lane & 15)) * 16);
        } else {
            const int k = 8 * (lane >> 4) + ((lane & 15) >> 2);
#pragma unroll
            for (int i = 0; i < 4; ++i) at[i] = k * I * 2 + (((first >> 3) + 2 * i + ((lane & 3) >> 1)) ^ across(k)) * 16 + (lane & 1) * 8;
        }
    }
    // rows 16 i .. + 15, elements 32 kk .. + 31
    __device__ __forceinline__ bf16x8 get(const char* lds, int i, int kk) const {
        if constexpr (ALONG) {
            return *(const bf16x8*)(lds + at[kk] + i * 32 * BK);
        } else {
            // 64 rows on (from a multiple of 128): the granules' numbers differ in bit 3 alone, and so do their places
            const char* p = lds + (i < 4 ? at[i & 3] : at[i & 3] ^ 128) + kk * 32 * I * 2;
            const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)p);
            const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)(p + 4 * I * 2));
            return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
};

// Where an operand's next tile lies: `others` rows (or columns) of the result from `first` on, the contraction from `k` on.
template <bool ALONG, int BK> struct Corner {
    const bf16_t* p;
    int64_t step;                               // to the next tile, in elements
    int stride, fixed;                          // bytes of the other rows, or elements of the row
    __device__ __forceinline__ void set(const FfnOperand& o, int first, int others, int k) {
        stride = (int)o.stride;
        p = o.p + (ALONG ? first * o.stride + k : k * o.stride + first);
        step = ALONG ? BK : BK * o.stride;
        fixed = ALONG ? (others - 1) * stride * 2 : (others + 7) / 8 * 16;
    }
    // Rows are padded to whole granules.
    __device__ __forceinline__ int bytes(int left) const { return ALONG ? fixed + (left + 7) / 8 * 16 : (min(left, BK) - 1) * stride * 2 + fixed; }
};

// Eight values as planes of terms.
template <typename E> __device__ __forceinline__ void store_terms(bf16_t* p, int64_t plane, const float (&x)[8]) {
    if constexpr (sizeof(E) == 2) {
        *(uint4*)p = narrow(x, bf16_t{});
    } else {
        float t[3][8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const Terms s = three_terms(x[e]);
            t[0][e] = s.t[0]; t[1][e] = s.t[1]; t[2][e] = s.t[2];
        }
#pragma unroll
        for (int q = 0; q < 3; ++q) *(uint4*)(p + q * plane) = narrow(t[q], bf16_t{});
    }
}

template <typename E, Epilogue EPI> struct Output { using T = E; };
template <typename E> struct Output<E, EPI_PART> { using T = float; };

// All but the last N of this wavefront's loads to LDS are done, and every other's; all have read what they asked for.
// (The builtin and not text, so that the compiler knows what has been waited for and adds no waits of its own to the products.)
template <int N> __device__ __forceinline__ void wait_loads() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 7 << 4);        // vmcnt(N) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// ---- products -------------------------------------------------------------------------------------------
// C[m][n] = sum_k A(m, k) B(n, k).  A tile of BM x BN by WM x WN wavefronts.
template <typename E, int BM, int BN, int WM, int WN, bool A_ALONG, bool B_ALONG, Epilogue EPI>
__global__ void __launch_bounds__(64 * WM * WN) ffn_product_kernel(FfnArgs a) {
    constexpr int WAVES = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;
    constexpr int TERMS = Mode<E>::TERMS, BK = Mode<E>::BK, STAGES = Mode<E>::STAGES;
    constexpr bool GATED = EPI == EPI_GATED;
    using TA = Tile<BM, A_ALONG, WAVES, BK>;
    using TB = Tile<BN, B_ALONG, WAVES, BK>;
    constexpr int STAGE = TERMS * (TA::BYTES + TB::BYTES), LOADS = TERMS * (TA::LOADS + TB::LOADS);
    __shared__ __align__(1024) char lds[STAGES][STAGE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / WN, wn = wave % WN;
    const int which = blockIdx.y / a.splits, split = blockIdx.y % a.splits;
    const FfnProblem& pr = a.prob[which];
    const int count = a.count ? *a.count : 0;
    const int M = a.count && !a.count_is_k ? count : pr.m, N = pr.n, K = a.count && a.count_is_k ? count : a.k;
    // Tiles that share rows of A or B run on one die, whose cache then holds them: dies take consecutive stretches of the tiles that
    // rows which count make.
    const int tiles_m = (M + BM - 1) / BM, tiles_n = GATED ? (N + BN / 2 - 1) / (BN / 2) : (N + BN - 1) / BN, tiles = tiles_m * tiles_n;
    const int each = (tiles + 7) / 8, id = blockIdx.x % 8 * each + blockIdx.x / 8;
    if ((int)blockIdx.x / 8 >= each || id >= tiles) return;
    constexpr int BAND = 8;                     // rows of tiles that are worked through together
    const int band = id / (BAND * tiles_n), in_band = id - band * BAND * tiles_n, high = min(BAND, tiles_m - band * BAND);
    const int m0 = (band * BAND + in_band % high) * BM, n0 = in_band / high * (GATED ? BN / 2 : BN);

    TA ta;
    TB tb;
    ta.init(wave, lane, pr.a[0].stride);
    // gated: half of a wavefront's columns are the gate's and half the other projection's, in turn; it loads from one of them
    const int half = GATED ? wave & 1 : 0;
    static_assert(!GATED || TB::LOADS * TB::ROWS_A_LOAD == TN * 8, "a wavefront loads from one of the two projections");
    tb.init(GATED ? wave >> 1 : wave, lane, pr.b[0].stride);
    Reader<BM, A_ALONG, BK> ra;
    Reader<BN, B_ALONG, BK> rb;
    ra.init(wm * TM * 16, lane);
    rb.init(wn * TN * 16, lane);

    const int ksteps = (K + BK - 1) / BK, all = ksteps * a.segments;
    const int per_split = (all + a.splits - 1) / a.splits, from = min(split * per_split, all), n = min(from + per_split, all) - from;
    // where the next tiles to load stand
    int seg = from / max(ksteps, 1), left = K - from % max(ksteps, 1) * BK;
    Corner<A_ALONG, BK> ca;
    Corner<B_ALONG, BK> cb;
    const int64_t plane_a = pr.a[0].plane, plane_b = pr.b[0].plane;
    auto corners = [&] {
        ca.set(pr.a[seg], m0, min(M - m0, BM), K - left);
        cb.set(pr.b[GATED ? half : seg], n0, min(N - n0, BN), K - left);
    };
    corners();
    auto load = [&](int stage) {
#pragma unroll
        for (int t = 0; t < TERMS; ++t) {
            ta.load(lds[stage] + t * TA::BYTES, wave, ca.p + t * plane_a, ca.bytes(left), left);
            tb.load(lds[stage] + TERMS * TA::BYTES + t * TB::BYTES, wave, cb.p + t * plane_b, cb.bytes(left), left);
        }
        ca.p += ca.step;
        cb.p += cb.step;
        left -= BK;
        if (left <= 0 && seg + 1 < a.segments) { ++seg; left = K; corners(); }
    };
    floatx4 acc[TM][TN] = {};
    // Two sets of operands, so that one comes from LDS while the products of the other run.
    bf16x8 fa[2][TERMS][TM], fb[2][TERMS][TN];
    auto read = [&](int stage, int set, int kk) {
        const char *la = lds[stage], *lb = la + TERMS * TA::BYTES;
#pragma unroll
        for (int t = 0; t < TERMS; ++t) {
#pragma unroll
            for (int j = 0; j < TN; ++j) fb[set][t][j] = rb.get(lb + t * TB::BYTES, j, kk);
#pragma unroll
            for (int i = 0; i < TM; ++i) fa[set][t][i] = ra.get(la + t * TA::BYTES, i, kk);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // the products of terms above 2^-24, small ones first
    auto multiply = [&](int set) {
#pragma unroll
        for (int order = TERMS - 1; order >= 0; --order)
#pragma unroll
            for (int t = 0; t <= order; ++t)
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[set][order - t][j], fa[set][t][i], acc[i][j], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
    };
    if constexpr (TERMS == 1) {
        // A step is two sets.  In its middle all wavefronts have done with its tiles, so that those of the step after next are asked for.
        if (n > 0) {
            load(0);
            if (n > 1) { load(1); wait_loads<LOADS>(); } else { wait_loads<0>(); }
            read(0, 0, 0);
            for (int s = 0; s + 1 < n; ++s) {
                read(s & 1, 1, 1);
                multiply(0);
                wait_loads<0>();
                read(s + 1 & 1, 0, 0);
                if (s + 2 < n) load(s & 1);
                multiply(1);
            }
            read(n - 1 & 1, 1, 1);
            multiply(0);
            multiply(1);
        }
    } else {
        // A step is one set.  It begins with the next one's operands and the loads of the third one on, into the place of its own.
        if (n > 0) {
            load(0);
            if (n > 1) load(1);
            if (n > 2) load(2);
            if (n > 2) wait_loads<2 * LOADS>(); else if (n > 1) wait_loads<LOADS>(); else wait_loads<0>();
            read(0, 0, 0);
            int stage = 0, s = 0;               // of the step
            auto full = [&](int set) {
                const int next = stage == 2 ? 0 : stage + 1;
                wait_loads<LOADS>();
                read(next, set ^ 1, 0);
                load(stage);
                multiply(set);
                stage = next;
            };
            for (; s + 4 < n; s += 2) { full(0); full(1); }
            auto step = [&](int s, int set) {   // the last ones
                const int next = stage == 2 ? 0 : stage + 1;
                if (s + 1 < n) {
                    if (s + 2 < n) wait_loads<LOADS>(); else wait_loads<0>();
                    read(next, set ^ 1, 0);
                    if (s + 3 < n) load(stage);
                }
                multiply(set);
                stage = next;
            };
            for (; s < n; s += 2) {
                step(s, 0);
                if (s + 1 < n) step(s + 1, 1);
            }
        }
    }
    settle_products();

    // Results go through LDS, so that whole lines of memory are read and written: column l % 16 of a product is a row of C, its rows
    // 4 (l / 16) .. + 3 are columns.  Granules of four columns lie at g ^ (row & 15).  Then eight columns of a row a thread.
    constexpr int ALL = STAGES * STAGE, PASSES = (BM * BN * 4 + ALL - 1) / ALL, PM = TM / PASSES, ROWS = BM / PASSES, NT = 64 * WAVES;
    constexpr int UNITS = GATED ? BN / 16 : BN / 8, EACH = ROWS * UNITS / NT, AHEAD = EPI == EPI_BACK ? 2 : EACH;
    static_assert(PASSES * PM == TM && EACH % AHEAD == 0, "whole passes");
    char* stage = lds[0];
    auto granule = [&](int row, int g) { return (floatx4*)(stage + row * BN * 4 + ((g ^ (row & 15)) << 4)); };
#pragma unroll
    for (int pass = 0; pass < PASSES; ++pass) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < PM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
                *granule((wm * PM + i) * 16 + (lane & 15), (wn * TN + j) * 4 + (lane >> 4)) = acc[pass * PM + i][j];
        __syncthreads();
#pragma unroll 1
        for (int u0 = 0; u0 < EACH; u0 += AHEAD) {
            floatx4 va[AHEAD][2], vb[AHEAD][2];
            int row[AHEAD], col[AHEAD], local[AHEAD];
            bool on[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int unit = (u0 + u) * NT + threadIdx.x;
                local[u] = unit / UNITS;
                row[u] = m0 + (local[u] / (PM * 16) * TM + pass * PM) * 16 + local[u] % (PM * 16);
                col[u] = n0 + unit % UNITS * 8;
                on[u] = row[u] < M && col[u] < (GATED || EPI == EPI_BACK ? a.hidden_p : N);
                if constexpr (EPI == EPI_BACK) {
                    const int64_t at = on[u] ? (int64_t)row[u] * a.hidden_p + col[u] : 0;
#pragma unroll
                    for (int h = 0; h < 2; ++h) { va[u][h] = *(const floatx4*)(a.va + at + 4 * h); vb[u][h] = *(const floatx4*)(a.vb + at + 4 * h); }
                }
            }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int unit = ((u0 + u) * NT + threadIdx.x) % UNITS, g = GATED ? unit / TN * TN * 4 + unit % TN * 2 : unit * 2;
                float x[8];
                *(floatx4*)x = *granule(local[u], g);
                *(floatx4*)(x + 4) = *granule(local[u], g + 1);
                const int64_t at = (int64_t)row[u] * a.hidden_p + col[u];
                if constexpr (GATED) {
                    float y[8], f[8], d[8];
                    *(floatx4*)y = *granule(local[u], g + TN * 2);
                    *(floatx4*)(y + 4) = *granule(local[u], g + TN * 2 + 1);
                    if (!on[u]) continue;
                    if (a.va) {
                        *(floatx4*)(a.va + at) = *(floatx4*)x; *(floatx4*)(a.va + at + 4) = *(floatx4*)(x + 4);
                        *(floatx4*)(a.vb + at) = *(floatx4*)y; *(floatx4*)(a.vb + at + 4) = *(floatx4*)(y + 4);
                    }
                    if (a.m) {
                        activate_all<E>(a.act, x, f, d);
#pragma unroll
                        for (int e = 0; e < 8; ++e) f[e] *= y[e];
                        store_terms<E>(a.m + at, a.m_plane, f);
                    }
                } else if constexpr (EPI == EPI_BACK) {
                    if (!on[u]) continue;
                    float p[8], b[8], f[8], d[8];
                    *(floatx4*)p = va[u][0]; *(floatx4*)(p + 4) = va[u][1];
                    *(floatx4*)b = vb[u][0]; *(floatx4*)(b + 4) = vb[u][1];
                    activate_all<E>(a.act, p, f, d);
#pragma unroll
                    for (int e = 0; e < 8; ++e) { p[e] = x[e] * b[e] * d[e]; x[e] *= f[e]; f[e] *= b[e]; }
                    store_terms<E>(a.da + at, a.m_plane, p);
                    store_terms<E>(a.db + at, a.m_plane, x);
                    store_terms<E>(a.m + at, a.m_plane, f);
                } else {
                    if (!on[u]) continue;
                    using O = typename Output<E, EPI>::T;
                    O* p = EPI == EPI_PART ? (O*)(a.part + which * a.part_stride + ((int64_t)split * pr.m + row[u]) * pr.n)
                                           : (O*)pr.out + (int64_t)(a.map ? a.map[row[u]] : row[u]) * pr.out_stride;
                    p += col[u];
                    if (((uintptr_t)p & 15) == 0 && col[u] + 8 <= N) {
#pragma unroll
                        for (int h = 0; h < 8 / VEC_OF<O>; ++h) ((uint4*)p)[h] = narrow(x + h * VEC_OF<O>, O{});
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (col[u] + e < N) p[e] = from_float<O>(x[e]);
                    }
                }
            }
        }
    }
}

// Sums of the parts of a split contraction, in order.
template <typename E> __global__ void __launch_bounds__(256) ffn_join_kernel(FfnArgs a) {
    const FfnProblem& pr = a.prob[blockIdx.y];
    const int M = a.count && !a.count_is_k ? *a.count : pr.m;
    const int64_t all = (int64_t)M * pr.n, whole = (int64_t)pr.m * pr.n;
    for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < all; i += gridDim.x * 256ll) {
        const float* p = a.part + blockIdx.y * a.part_stride + i;
        float s = 0.f;
        for (int q = 0; q < a.splits; ++q) s += p[q * whole];
        const int row = (int)(i / pr.n), col = (int)(i - (int64_t)row * pr.n);
        ((E*)pr.out)[(int64_t)(a.map ? a.map[row] : row) * pr.out_stride + col] = from_float<E>(s);
    }
}

// ---- preparation ------------------------------------------------------------------------------------------
// Which row each packed one is, and how many there are.  A workgroup takes `per` rows of all and counts those before it itself.
__global__ void __launch_bounds__(256) ffn_map_kernel(const int* lengths, int batch, int steps, int64_t rows, int64_t per, int* map, int* count) {
    __shared__ int sums[4];
    const int64_t first = blockIdx.x * per, last = min(first + per, rows);
    auto length = [&](int b) { return min(max(lengths[b], 0), steps); };
    // rows that count before `first`: whole sequences, and the beginning of the one it lies in
    const int b0 = (int)(first / steps);
    int mine = 0;
    for (int b = threadIdx.x; b < b0; b += 256) mine += length(b);
    for (int d = 1; d < 64; d <<= 1) mine += __shfl_xor(mine, d);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = mine;
    __syncthreads();
    const int base = sums[0] + sums[1] + sums[2] + sums[3];
    // 256 rows at a time: their places follow from counts of the lanes and wavefronts before
    const int t0 = (int)(first - (int64_t)b0 * steps);
    int done = base + (t0 > 0 ? min(t0, length(b0)) : 0);
    for (int64_t r0 = first; r0 < last; r0 += 256) {
        const int64_t r = r0 + threadIdx.x;
        const int b = (int)(r / steps);
        const bool live = r < last && (int)(r - (int64_t)b * steps) < length(b);
        const uint64_t mask = __ballot(live);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = __popcll(mask);
        __syncthreads();
        int at = done + __popcll(mask & ((1ull << (threadIdx.x & 63)) - 1));
        for (int w = 0; w < (int)(threadIdx.x >> 6); ++w) at += sums[w];
        if (live) map[at] = (int)r;
        done += sums[0] + sums[1] + sums[2] + sums[3];
    }
    if (last == rows && threadIdx.x == 0) *count = done;
}

// Matrices as planes of padded rows, packed by the map where there is one.  Rows of `clear` that do not count become zeros.
struct FfnCopy { const void* from; int64_t stride; bf16_t* to; int64_t plane; int rows, cols, cols_p; const int* map; };
struct FfnCopies {
    FfnCopy c[4];
    int n;
    const int* count;
    void* clear; int64_t clear_stride; int clear_cols, clear_rows;
    Live live;
};
template <typename E> __global__ void __launch_bounds__(256) ffn_prepare_kernel(FfnCopies a) {
    if ((int)blockIdx.y == a.n) {
        for (int r = blockIdx.x; r < a.clear_rows; r += gridDim.x)
            if (!a.live(r))
                for (int i = threadIdx.x; i < a.clear_cols; i += 256) ((E*)a.clear)[(int64_t)r * a.clear_stride + i] = from_float<E>(0.f);
        return;
    }
    const FfnCopy& c = a.c[blockIdx.y];
    const int rows = c.map ? *a.count : c.rows, each = c.cols_p / 8;
    const bool al = (c.stride * sizeof(E)) % 16 == 0 && ((uintptr_t)c.from & 15) == 0;
    for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < (int64_t)rows * each; i += gridDim.x * 256ll) {
        const int row = (int)(i / each), col = (int)(i - (int64_t)row * each) * 8;
        const E* p = (const E*)c.from + (int64_t)(c.map ? c.map[row] : row) * c.stride + col;
        float x[8];
        if (al && col + 8 <= c.cols) {
#pragma unroll
            for (int g = 0; g < 8 / VEC_OF<E>; ++g) widen(((const uint4*)p)[g], x + g * VEC_OF<E>, E{});
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = col + e < c.cols ? to_float(p[e]) : 0.f;
        }
        bf16_t* to = c.to + (int64_t)row * c.cols_p + col;
        store_terms<E>(to, c.plane, x);
    }
}

// ---- host -------------------------------------------------------------------------------------------------
bool ffn_ok(const pql_ffn_shape& s) {
    return s.batch >= 0 && s.steps >= 0 && (double)s.batch * s.steps < 1073741824.0 && s.dim >= 1 && s.dim <= PQL_FFN_MAX_DIM && s.hidden >= 1 &&
           s.hidden <= PQL_FFN_MAX_DIM && (s.dtype == PQL_F32 || s.dtype == PQL_BF16) && s.act >= PQL_ACT_NONE && s.act <= PQL_ACT_RELU;
}
int ffn_rows(const pql_ffn_shape& s) { return (int)((int64_t)s.batch * s.steps); }
int up8(int x) { return (x + 7) / 8 * 8; }
int tiles_of(int x, int b) { return (x + b - 1) / b; }

// Parts of the contraction: where the tiles do not fill the card, as many as do, each of at least 8 steps.
int ffn_splits(int tiles, int at_a_time, int steps) {
    int s = tiles > 0 ? at_a_time / tiles : 1;
    if (s > steps / 8) s = steps / 8;
    return s < 1 ? 1 : s > 64 ? 64 : s;
}
// Edge of the tiles of a product of `problems` m x n results: 256 where such tiles fill the card.
int tile_edge(int32_t dtype, int64_t m, int n, int problems) { return dtype == PQL_BF16 && (int64_t)tiles_of((int)m, 256) * tiles_of(n, 256) * problems >= BIG_TILES ? 256 : 128; }

struct FfnPlan {
    int rows, terms, dim_p, hidden_p, out_splits, dx_splits, weight_splits;
    size_t map, count, x, dout, gate, up, down, m, da, db, va, vb, part, bytes;
    int64_t x_plane, gate_plane, down_plane, m_plane;
};
FfnPlan ffn_plan(const pql_ffn_shape& s, int call) {
    FfnPlan p{};
    p.rows = ffn_rows(s);
    p.terms = s.dtype == PQL_F32 ? 3 : 1;
    p.dim_p = up8(s.dim); p.hidden_p = up8(s.hidden);
    p.x_plane = (int64_t)p.rows * p.dim_p;
    p.gate_plane = (int64_t)s.hidden * p.dim_p;
    p.down_plane = (int64_t)s.dim * p.hidden_p;
    p.m_plane = (int64_t)p.rows * p.hidden_p;
    size_t o = 0;
    auto take = [&](size_t b) { const size_t at = o; o += to256(b); return at; };
    auto planes = [&](int64_t plane) { return take((size_t)plane * p.terms * 2); };
    p.map = take((size_t)p.rows * 4);
    p.count = take(4);
    p.x = planes(p.x_plane);
    p.gate = planes(p.gate_plane);
    p.up = planes(p.gate_plane);
    p.down = planes(p.down_plane);
    p.m = planes(p.m_plane);
    const int bk = s.dtype == PQL_F32 ? Mode<float>::BK : Mode<bf16_t>::BK;
    // two workgroups a compute unit with the small tiles of bf16, one otherwise
    auto splits = [&](int64_t m, int n, int problems, int steps) {
        const int e = tile_edge(s.dtype, m, n, problems);
        return ffn_splits(tiles_of((int)m, e) * tiles_of(n, e) * problems, s.dtype == PQL_BF16 && e == 128 ? 512 : 256, steps);
    };
    size_t part = 0;
    auto parts = [&](int splits, size_t floats) { if (splits > 1 && splits * floats * 4 > part) part = splits * floats * 4; };
    p.out_splits = splits(p.rows, s.dim, 1, tiles_of(s.hidden, bk));
    p.dx_splits = splits(p.rows, s.dim, 1, 2 * tiles_of(s.hidden, bk));
    p.weight_splits = splits(s.hidden, s.dim, 3, tiles_of(p.rows, bk));
    if (call == PQL_FFN_FORWARD) {
        parts(p.out_splits, (size_t)p.rows * s.dim);
    } else {
        p.dout = planes(p.x_plane);
        p.da = planes(p.m_plane);
        p.db = planes(p.m_plane);
        if (call == PQL_FFN_BACKWARD_ALONE) { p.va = take((size_t)p.m_plane * 4); p.vb = take((size_t)p.m_plane * 4); }
        parts(p.dx_splits, (size_t)p.rows * s.dim);
        parts(p.weight_splits, 3 * (size_t)s.dim * s.hidden);
    }
    p.part = take(part);
    p.bytes = o;
    return p;
}

template <typename E, bool A_ALONG, bool B_ALONG, Epilogue EPI> void launch_product(const ProfSlot& ps, int edge, dim3 grid, const FfnArgs& a, hipStream_t st) {
    if constexpr (sizeof(E) == 4) PQL_LAUNCH(ps, (ffn_product_kernel<E, 128, 128, 2, 4, A_ALONG, B_ALONG, EPI>), grid, dim3(512), 0, st, a);
    else if (edge == 256) PQL_LAUNCH(ps, (ffn_product_kernel<E, 256, 256, 2, 4, A_ALONG, B_ALONG, EPI>), grid, dim3(512), 0, st, a);
    else PQL_LAUNCH(ps, (ffn_product_kernel<E, 128, 128, 2, 2, A_ALONG, B_ALONG, EPI>), grid, dim3(256), 0, st, a);
}

struct FfnRun {
    const pql_ffn_shape& s;
    const FfnPlan& p;
    char* ws;
    hipStream_t st;
    hipError_t e = hipSuccess;
    const int *map = nullptr, *count = nullptr;
    FfnCopies copies{};
    int elem() const { return s.dtype == PQL_F32 ? 4 : 2; }

    template <typename T> T* at(size_t o) const { return (T*)(ws + o); }
    void pack(const int32_t* lengths) {
        copies.live = {lengths, (unsigned)s.steps};
        if (!lengths) return;
        const int64_t rows = p.rows;
        int64_t per = (rows + 255) / 256;
        per = per < 1024 ? 1024 : (per + 255) / 256 * 256;
        const ProfSlot ps = prof_slot();
        PQL_LAUNCH(ps, ffn_map_kernel, dim3((unsigned)((rows + per - 1) / per)), dim3(256), 0, st, lengths, s.batch, s.steps, rows, per, at<int>(p.map), at<int>(p.count));
        prof_commit(ps, KID_FFN_PREPARE, 0.0, 4.0 * rows);
        map = at<int>(p.map);
        count = at<int>(p.count);
    }
    // The matrix as an operand: where it is, or as planes at `to`.
    FfnOperand operand(const pql_rows& r, int rows, int cols, size_t to, int64_t plane, bool tokens, bool direct = true) {
        if (direct && s.dtype == PQL_BF16 && !(tokens && map) && cols % 8 == 0 && rows_aligned(r, s.dtype) && r.stride >= cols && r.stride <= 1 << 20)
            return {(const bf16_t*)r.data, r.stride, 0};
        FfnCopy& c = copies.c[copies.n++];
        c = {r.data, r.stride, at<bf16_t>(to), plane, rows, cols, up8(cols), tokens ? map : nullptr};
        return {at<bf16_t>(to), up8(cols), plane};
    }
    // Both projections' weights, alike.
    void projections(const pql_ffn_input& in, FfnOperand& gate, FfnOperand& up) {
        const bool alike = in.gate.stride == in.up.stride && rows_aligned(in.gate, s.dtype) && rows_aligned(in.up, s.dtype);
        gate = operand(in.gate, s.hidden, s.dim, p.gate, p.gate_plane, false, alike);
        up = operand(in.up, s.hidden, s.dim, p.up, p.gate_plane, false, alike);
    }
    // Rows of the output that do not count.
    void clear(const pql_rows& out) {
        if (!map) return;
        copies.clear = out.data; copies.clear_stride = out.stride; copies.clear_cols = s.dim; copies.clear_rows = p.rows;
    }
    void prepare() {
        const int y = copies.n + (copies.clear ? 1 : 0);
        if (y == 0 || e != hipSuccess) return;
        copies.count = count;
        int64_t most = copies.clear ? copies.clear_rows * 256ll : 0, bytes = 0;
        for (int i = 0; i < copies.n; ++i) {
            const int64_t n = (int64_t)copies.c[i].rows * copies.c[i].cols_p / 8;
            most = n > most ? n : most;
            bytes += n * 8 * (elem() + 2 * p.terms);
        }
        const int64_t blocks = (most + 255) / 256;
        const ProfSlot ps = prof_slot();
        const dim3 grid((unsigned)(blocks < 2048 ? blocks : 2048), y);
        if (s.dtype == PQL_F32) PQL_LAUNCH(ps, ffn_prepare_kernel<float>, grid, dim3(256), 0, st, copies);
        else PQL_LAUNCH(ps, ffn_prepare_kernel<bf16_t>, grid, dim3(256), 0, st, copies);
        prof_commit(ps, KID_FFN_PREPARE, 0.0, (double)bytes);
        e = hipGetLastError();
    }
    FfnArgs args() const {
        FfnArgs a{};
        a.segments = 1; a.splits = 1;
        a.count = count; a.map = map; a.act = s.act;
        a.hidden_p = p.hidden_p; a.m_plane = p.m_plane;
        return a;
    }
    // whole: problems of a full call, which the plan has counted with
    template <bool A_ALONG, bool B_ALONG, Epilogue EPI> void product(FfnArgs& a, int problems, int whole, int kid) {
        if (e != hipSuccess) return;
        const FfnProblem& pr = a.prob[0];
        const int edge = EPI == EPI_GATED ? tile_edge(s.dtype, pr.m, 2 * pr.n, 1) : tile_edge(s.dtype, pr.m, pr.n, whole);
        const int each = (tiles_of(pr.m, edge) * tiles_of(pr.n, EPI == EPI_GATED ? edge / 2 : edge) + 7) / 8;           // problems are alike or transposed
        const dim3 grid(each * 8, problems * a.splits);
        const ProfSlot ps = prof_slot();
        if (s.dtype == PQL_F32) launch_product<float, A_ALONG, B_ALONG, EPI>(ps, edge, grid, a, st);
        else launch_product<bf16_t, A_ALONG, B_ALONG, EPI>(ps, edge, grid, a, st);
        prof_commit(ps, kid, 2.0 * problems * (EPI == EPI_GATED ? 2 : 1) * a.segments * pr.m * pr.n * (double)a.k, 0.0);
        e = hipGetLastError();
    }
    // The product of rows or weights, in parts where that fills the card.
    template <bool A_ALONG, bool B_ALONG> void result(FfnArgs& a, int problems, int whole, int splits) {
        a.splits = splits;
        if (splits == 1) return product<A_ALONG, B_ALONG, EPI_OUT>(a, problems, whole, KID_FFN_PRODUCT);
        a.part = at<float>(p.part);
        a.part_stride = (int64_t)splits * a.prob[0].m * a.prob[0].n;
        product<A_ALONG, B_ALONG, EPI_PART>(a, problems, whole, KID_FFN_PRODUCT);
        if (e != hipSuccess) return;
        const int64_t blocks = ((int64_t)a.prob[0].m * a.prob[0].n + 255) / 256;
        const ProfSlot ps = prof_slot();
        const dim3 grid((unsigned)(blocks < 1024 ? blocks : 1024), problems);
        if (s.dtype == PQL_F32) PQL_LAUNCH(ps, ffn_join_kernel<float>, grid, dim3(256), 0, st, a);
        else PQL_LAUNCH(ps, ffn_join_kernel<bf16_t>, grid, dim3(256), 0, st, a);
        prof_commit(ps, KID_FFN_JOIN, 0.0, 4.0 * problems * splits * a.prob[0].m * a.prob[0].n);
        e = hipGetLastError();
    }
    void gated(const FfnOperand& x, const FfnOperand& gate, const FfnOperand& up, float* va, float* vb, bf16_t* m) {
        FfnArgs a = args();
        a.prob[0] = {{x, x}, {gate, up}, p.rows, s.hidden, nullptr, 0};
        a.k = s.dim;
        a.va = va; a.vb = vb; a.m = m;
        product<true, true, EPI_GATED>(a, 1, 1, KID_FFN_GATED);
    }
};

int32_t ffn_check(pql_ctx* c, const pql_ffn_shape* s, const pql_ffn_input* in, const pql_rows* out, bool back) {
    if (!s || !in || !out) return ctx_fail(c, PQL_ERR_NULL, "pql_ffn: null pointer");
    if (!ffn_ok(*s)) return ctx_fail(c, PQL_ERR_INVALID_ARG, "pql_ffn: bad shape");
    const int rows = ffn_rows(*s);
    if (!read_rows(in->x) || !read_rows(in->gate) || !read_rows(in->up) || !read_rows(in->down) || !(back ? read_rows(*out) : own_rows(*out, rows, s->dim)))
        return ctx_fail(c, PQL_ERR_INVALID_ARG, "pql_ffn: bad stride");
    if (rows == 0) return PQL_OK;
    if (!in->x.data || !in->gate.data || !in->up.data || !in->down.data || !out->data) return ctx_fail(c, PQL_ERR_NULL, "pql_ffn: null pointer");
    const size_t e = elem_size(s->dtype);
    if (off_by(in->x.data, e) || off_by(in->gate.data, e) || off_by(in->up.data, e) || off_by(in->down.data, e) || off_by(out->data, e) || off_by(in->lengths, 4))
        return ctx_fail(c, PQL_ERR_ALIGNMENT, "pql_ffn: misaligned pointer");
    return PQL_OK;
}

}  // namespace
}  // namespace pql

using namespace pql;

extern "C" {

int64_t pql_ffn_saved_bytes(const pql_ffn_shape* s) {
    if (!s) return PQL_ERR_NULL;
    if (!ffn_ok(*s)) return PQL_ERR_INVALID_ARG;
    return (int64_t)(2 * to256((size_t)ffn_rows(*s) * up8(s->hidden) * 4));
}

int64_t pql_ffn_workspace_bytes(const pql_ffn_shape* s, int32_t call) {
    if (!s) return PQL_ERR_NULL;
    if (!ffn_ok(*s) || call < PQL_FFN_FORWARD || call > PQL_FFN_BACKWARD_ALONE) return PQL_ERR_INVALID_ARG;
    return (int64_t)ffn_plan(*s, call).bytes;
}

int32_t pql_ffn_forward(pql_ctx* c, const pql_ffn_shape* s, const pql_ffn_input* in, const pql_rows* out, void* saved, void* workspace, void* stream) {
    if (!c) return PQL_ERR_NULL;
    const int32_t rc = ffn_check(c, s, in, out, false);
    if (rc != PQL_OK || ffn_rows(*s) == 0) return rc;
    if (!workspace) return ctx_fail(c, PQL_ERR_NULL, "pql_ffn_forward: null workspace");
    if (off_by(saved, 256) || off_by(workspace, 256)) return ctx_fail(c, PQL_ERR_ALIGNMENT, "pql_ffn_forward: misaligned saved or workspace");
    const FfnPlan p = ffn_plan(*s, PQL_FFN_FORWARD);
    const hipStream_t st = (hipStream_t)stream;
    hipError_t e;
    if (p.rows <= FFN_FEW_ROWS && !saved) {
        FfnRowsArgs a{{in->lengths, (unsigned)s->steps}, p.rows, s->dim, s->hidden, s->act, in->x.data, in->gate.data, in->up.data, in->down.data,
                      in->x.stride, in->gate.stride, in->up.stride, in->down.stride, (char*)workspace + p.m, p.hidden_p, out->data, out->stride};
        e = ffn_rows_launch(a, s->dtype, st);
    } else {
        FfnRun r{*s, p, (char*)workspace, st};
        r.pack(in->lengths);
        const FfnOperand x = r.operand(in->x, p.rows, s->dim, p.x, p.x_plane, true);
        FfnOperand gate, up;
        r.projections(*in, gate, up);
        const FfnOperand down = r.operand(in->down, s->dim, s->hidden, p.down, p.down_plane, false);
        r.clear(*out);
        r.prepare();
        bf16_t* m = r.at<bf16_t>(p.m);
        float* va = (float*)saved;
        r.gated(x, gate, up, va, saved ? (float*)((char*)saved + to256((size_t)p.m_plane * 4)) : nullptr, m);
        FfnArgs a = r.args();
        const FfnOperand om{m, p.hidden_p, p.m_plane};
        a.prob[0] = {{om, om}, {down, down}, p.rows, s->dim, out->data, out->stride};
        a.k = s->hidden;
        r.result<true, true>(a, 1, 1, p.out_splits);
        e = r.e;
    }
    return e == hipSuccess ? PQL_OK : ctx_fail(c, PQL_ERR_HIP, "pql_ffn_forward", e);
}

int32_t pql_ffn_backward(pql_ctx* c, const pql_ffn_shape* s, const pql_ffn_input* in, const void* saved, const pql_rows* out_grad,
                         const pql_ffn_grad* g, void* workspace, void* stream) {
    if (!c) return PQL_ERR_NULL;
    if (!g) return ctx_fail(c, PQL_ERR_NULL, "pql_ffn_backward: null pointer");
    const int32_t rc = ffn_check(c, s, in, out_grad, true);
    if (rc != PQL_OK) return rc;
    const int rows = ffn_rows(*s);
    auto bad = [&](const pql_rows& r, int64_t n, int cols) { return r.data && !own_rows(r, n, cols); };
    if (bad(g->x, rows, s->dim) || bad(g->gate, s->hidden, s->dim) || bad(g->up, s->hidden, s->dim) || bad(g->down, s->dim, s->hidden))
        return ctx_fail(c, PQL_ERR_INVALID_ARG, "pql_ffn_backward: bad stride");
    const size_t es = elem_size(s->dtype);
    if (off_by(g->x.data, es) || off_by(g->gate.data, es) || off_by(g->up.data, es) || off_by(g->down.data, es) || off_by(saved, 256) || off_by(workspace, 256))
        return ctx_fail(c, PQL_ERR_ALIGNMENT, "pql_ffn_backward: misaligned pointer");
    if (rows > 0 && !workspace) return ctx_fail(c, PQL_ERR_NULL, "pql_ffn_backward: null workspace");
    const FfnPlan p = ffn_plan(*s, saved ? PQL_FFN_BACKWARD : PQL_FFN_BACKWARD_ALONE);
    FfnRun r{*s, p, (char*)workspace, (hipStream_t)stream};
    FfnOperand x{}, dout{}, m{}, da{}, db{};
    if (rows > 0) {
        r.pack(in->lengths);
        x = r.operand(in->x, rows, s->dim, p.x, p.x_plane, true);
        dout = r.operand(*out_grad, rows, s->dim, p.dout, p.x_plane, true);
        FfnOperand gate, up;
        r.projections(*in, gate, up);
        r.prepare();
        r.copies.n = 0;
        const FfnOperand down = r.operand(in->down, s->dim, s->hidden, p.down, p.down_plane, false);
        if (g->x.data) r.clear(g->x);
        r.prepare();
        float *va = (float*)saved, *vb = (float*)((char*)saved + to256((size_t)p.m_plane * 4));
        if (!saved) {
            va = r.at<float>(p.va); vb = r.at<float>(p.vb);
            r.gated(x, gate, up, va, vb, nullptr);
        }
        m = {r.at<bf16_t>(p.m), p.hidden_p, p.m_plane};
        da = {r.at<bf16_t>(p.da), p.hidden_p, p.m_plane};
        db = {r.at<bf16_t>(p.db), p.hidden_p, p.m_plane};
        FfnArgs a = r.args();
        a.prob[0] = {{dout, dout}, {down, down}, rows, s->hidden, nullptr, 0};
        a.k = s->dim;
        a.va = va; a.vb = vb; a.m = (bf16_t*)m.p; a.da = (bf16_t*)da.p; a.db = (bf16_t*)db.p;
        r.product<true, false, EPI_BACK>(a, 1, 1, KID_FFN_BACK);
        if (g->x.data) {
            a = r.args();
            a.prob[0] = {{da, db}, {gate, up}, rows, s->dim, g->x.data, g->x.stride};
            a.k = s->hidden;
            a.segments = 2;
            r.result<true, false>(a, 1, 1, p.dx_splits);
        }
    }
    FfnArgs w = r.args();
    int n = 0;
    if (g->gate.data) w.prob[n++] = {{da, da}, {x, x}, s->hidden, s->dim, g->gate.data, g->gate.stride};
    if (g->up.data) w.prob[n++] = {{db, db}, {x, x}, s->hidden, s->dim, g->up.data, g->up.stride};
    if (g->down.data) w.prob[n++] = {{dout, dout}, {m, m}, s->dim, s->hidden, g->down.data, g->down.stride};
    w.k = rows;
    w.count_is_k = 1;
    w.map = nullptr;
    if (n > 0) r.result<false, false>(w, n, 3, p.weight_splits);
    return r.e == hipSuccess ? PQL_OK : ctx_fail(c, PQL_ERR_HIP, "pql_ffn_backward", r.e);
}

}  // extern "C"
