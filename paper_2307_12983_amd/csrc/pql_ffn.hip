// The gated feed-forward block (include/pql_block.h), products of row tiles:
//     a = x G^T,  b = x U^T,  m = act(a) b,  out = m D^T,
//     dm = dout D,  da = dm b act'(a),  db = dm act(a),  dx = da G + db U,  dG = da^T x,  dU = db^T x,  dD = dout^T m.
//
// All products run on the bf16 matrix instructions with sums in fp32.  fp32 values are three bf16 terms each (24 bits, exactly),
// of whose nine products the three below 2^-24 are left out: six products a pair.  Operands lie in memory as planes, one for each
// term; bf16 tensors whose rows start on 16-byte boundaries are used where they are, and so are fp32 weights where there are few
// rows.  bf16: m, da and db are rounded once, as operands of the next products; a and b are kept in fp32.
//
// Rows that count are packed together first where sequences have lengths, so that no work is done for the others.
//
// A workgroup computes one tile of the result.  Tiles of both operands go from memory to LDS without registers between, one
// step ahead of the products, and are laid out there so that neither the contiguous reads (operands whose contraction runs along
// a row) nor the transposing ones (along a column) meet bank conflicts: no operand is ever transposed in memory.  bf16 takes tiles of
// 256 x 256 by eight wavefronts, since what bounds it is the way from L2 to LDS, 64 KB a step of 64: 4 x 2048 rows of 2048 and 8192
// with gradients take 2.22 ms, with tiles of 128 x 128 2.71 ms, of 256 x 128 by two workgroups a compute unit 2.57 ms; three to five
// steps of 32 in LDS 2.38 ms.  Its products reach 975 (projections), 1230 (out, dx, weights' gradients) and 730 TFLOP/s (dm, da, db:
// half of its time goes to reading a and b and writing da and db, 0.8 GB at 5 TB/s); the loop without its products takes 77 % of the
// time with them.  fp32 takes 256 x 128, six products a pair, and is bound by those: 512 x 32 rows of 256 and 1024 with gradients
// take 0.41 ms.
#include <type_traits>

#include "pql_ffn_internal.h"

namespace pql {
namespace {

typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) shortx4 lds_shortx4;

// Terms of a value, elements of the contraction a step, steps in LDS at a time; the fewest steps that a part of a tile is worth, whose
// sums are written and read again (us a call with 1 / 4 / 8 / 12 of them: bf16, 65 rows of 1000 and 4000 53 / 38 / 36 / 38, 2048 rows
// of 1024 and 1024 45 / 45 / 41 / 33, 300 rows of 512 and 2048 with gradients 92 / 70 / 67 / 75; fp32, the last 144 / 138 / 140 / 167, 1665
// rows of 203 and 677 with gradients 130 / 131 / 137 / 146, 512 x 32 rows of 256 and 1024 with gradients 401 / 417).
template <typename E, int BM> struct Mode { static constexpr int TERMS = 1, BK = 64, STAGES = 2, LEAST = BM == 128 ? 8 : 4; };
template <> struct Mode<float, 128> { static constexpr int TERMS = 3, BK = 32, STAGES = 3, LEAST = 1; };
template <> struct Mode<float, 256> { static constexpr int TERMS = 3, BK = 32, STAGES = 2, LEAST = 1; };
// As many tiles of 256 rows make them worth it, fewer leave compute units without one (us a launch, 256 / 128 rows: 256 tiles, 2048 rows of
// 2048 and 2048 in fp32 162 / 193, 4096 rows in bf16 65 / 68; 128 tiles, the same calls' last product 100 with its join / 100 and 57 / 36).
constexpr int BIG_TILES = 192;
// Calls of at most so many rows read 32-bit weights as they are and make their terms in the product's kernel, for each 128 rows anew;
// others make planes of them first (us a call with gradients, as they are / planes: 128 rows, 1024 and 4096: 182 / 219, 4096 and 16384:
// 1216 / 2060; 768 rows: 454 / 457 and 5231 / 5402; 1024 rows: 529 / 494 and 6894 / 6983; 2048 rows: 953 / 842 and 13594 / 12616).
constexpr int WHOLE_ROWS = 768;
constexpr int NOWHERE = 0x7fffff00;             // an offset behind every buffer: reads give zeros

// One operand: rows of a matrix, `plane` elements from one term's to the next.
// whole: 32-bit values, the stride in halves of them.
struct FfnOperand { const bf16_t* p; int64_t stride, plane; bool whole; };
struct FfnProblem { FfnOperand a[2], b[2]; int m, n; void* out; int64_t out_stride; };
enum Epilogue : int { EPI_GATED, EPI_BACK, EPI_OUT };

struct FfnArgs {
    FfnProblem prob[3];
    int problems, k, segments;                  // length of the contraction, of each of `segments` pairs of operands
    const int* count;                           // rows that count, NULL: all
    int count_is_k;                             // whether they are the contraction or the rows of the result
    float* part;                                // [workgroups][2][tile] sums over parts of the contraction
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

// The same of 32-bit values as they are, whose terms are made here: tiles of twice as many 16-bit elements (ALONG: a row, ACROSS: I).
template <int I, bool ALONG> struct WholeReader {
    int at[ALONG ? 2 : 8];
    __device__ __forceinline__ void init(int first, int lane) {         // first: a multiple of 32; two sets of 16 rows from it on
        const int r = lane & 15, q = lane >> 4;
        if constexpr (ALONG) {
#pragma unroll
            for (int h = 0; h < 2; ++h) at[h] = (first + r) * 128 + (((2 * q + h) ^ along<64>(r)) * 16);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {                               // set i / 4, elements i % 4 and + 4 of the contraction's eight
                const int k = 8 * q + (i & 3);
                at[i] = k * I * 4 + ((((first + (i >> 2) * 16 + r) >> 2) ^ across(k)) * 16) + (r & 3) * 4;
            }
        }
    }
    __device__ __forceinline__ void get(const char* lds, int i, float (&x)[8]) const {
        if constexpr (ALONG) {
#pragma unroll
            for (int h = 0; h < 2; ++h) *(floatx4*)(x + 4 * h) = *(const floatx4*)(lds + at[h] + i * 16 * 128);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = *(const float*)(lds + at[i * 4 + (e & 3)] + (e >> 2) * 4 * I * 4);
        }
    }
};
__device__ __forceinline__ void terms_of(const float (&x)[8], bf16x8 (&t)[3]) {
    float f[3][8];
    bool odd = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        f[0][e] = (float)(bf16_t)x[e];
        odd |= !(fabsf(f[0][e]) < __builtin_inff());
        const float r = x[e] - f[0][e];
        f[1][e] = __uint_as_float(__float_as_uint(r) & 0xffff0000u);
        f[2][e] = r - f[1][e];
    }
    if (__ballot(odd)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const Terms s = three_terms(x[e]);
            f[0][e] = s.t[0]; f[1][e] = s.t[1]; f[2][e] = s.t[2];
        }
    }
#pragma unroll
    for (int q = 0; q < 3; ++q) t[q] = __builtin_bit_cast(bf16x8, narrow(f[q], bf16_t{}));
}

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

// a and b of eight columns.
__device__ __forceinline__ void read_saved(const FfnArgs& a, int64_t at, floatx4 (&va)[2], floatx4 (&vb)[2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) { va[h] = *(const floatx4*)(a.va + at + 4 * h); vb[h] = *(const floatx4*)(a.vb + at + 4 * h); }
}
// Eight columns of a row of the result from their sums; gated: those of both projections.
template <typename E, Epilogue EPI> __device__ __forceinline__ void finish(const FfnArgs& a, const FfnProblem& pr, int row, int col, float (&x)[8], float (&y)[8],
                                                                       const floatx4 (&va)[2], const floatx4 (&vb)[2]) {
    const int64_t at = (int64_t)row * a.hidden_p + col;
    if constexpr (EPI == EPI_GATED) {
        if (a.va) {
            *(floatx4*)(a.va + at) = *(floatx4*)x; *(floatx4*)(a.va + at + 4) = *(floatx4*)(x + 4);
            *(floatx4*)(a.vb + at) = *(floatx4*)y; *(floatx4*)(a.vb + at + 4) = *(floatx4*)(y + 4);
        }
        float f[8], d[8];
        activate_all<E>(a.act, x, f, d);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] *= y[e];
        store_terms<E>(a.m + at, a.m_plane, f);
    } else if constexpr (EPI == EPI_BACK) {
        float p[8], b[8], f[8], d[8];
        *(floatx4*)p = va[0]; *(floatx4*)(p + 4) = va[1];
        *(floatx4*)b = vb[0]; *(floatx4*)(b + 4) = vb[1];
        activate_all<E>(a.act, p, f, d);
#pragma unroll
        for (int e = 0; e < 8; ++e) { p[e] = x[e] * b[e] * d[e]; x[e] *= f[e]; }
        store_terms<E>(a.da + at, a.m_plane, p);
        store_terms<E>(a.db + at, a.m_plane, x);
    } else {
        E* p = (E*)pr.out + (int64_t)(a.map ? a.map[row] : row) * pr.out_stride + col;
        if (((uintptr_t)p & 15) == 0 && col + 8 <= pr.n) {
#pragma unroll
            for (int h = 0; h < 8 / VEC_OF<E>; ++h) ((uint4*)p)[h] = narrow(x + h * VEC_OF<E>, E{});
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (col + e < pr.n) p[e] = from_float<E>(x[e]);
        }
    }
}

// ---- how the tiles are shared out ------------------------------------------------------------------------
// `slots` workgroups run at a time.  As many whole rounds of tiles as there are go to a workgroup each; the `rest` tiles behind
// them are cut into steps of their contractions, of which each of `sharers` workgroups takes `per` in a row, `least` or more and at
// most a tile's.  What is not a whole tile is left as sums, joined by another launch.  Known where the rows that count are: on the device.
// Steps that the other launch takes as long as: fewer saved are not worth it, and contractions of no more never launch it (us a call with
// gradients for 6 / 7 / 8 of them: 5 x 333 rows of 203 and 677 165 / 156 / 156, 512 x 32 rows of 256 and 1024 422 / 414 / 431).
constexpr int JOIN_STEPS = 7;
struct Shares {
    int whole, rest, steps, per, sharers;
    __host__ __device__ Shares(int tiles, int slots, int steps_, int least) : steps(steps_) {
        whole = tiles / slots * slots;
        rest = tiles - whole;
        per = (int)(((int64_t)rest * steps + slots - 1) / slots);
        if (per > 0 && per < least) per = least;
        if (per > steps - JOIN_STEPS) per = steps;
        sharers = per > 0 ? (int)(((int64_t)rest * steps + per - 1) / per) : rest;
    }
    __host__ __device__ bool joins() const { return rest > 0 && per < steps; }
};
// The i-th of n things for workgroups of which every eighth runs on the same die: dies take consecutive stretches.  -1: nothing.
__device__ __forceinline__ int stretch(int i, int n) {
    const int each = (n + 7) / 8, id = i % 8 * each + i / 8;
    return i / 8 < each && id < n ? id : -1;
}
// A tile's problem and corner: in bands of BAND rows of tiles, that share what they read in one die's cache.
struct Place { int which, m0, n0; };
template <int BM, int COLS> __host__ __device__ inline int tiles_in(int m, int n) { return ((m + BM - 1) / BM) * ((n + COLS - 1) / COLS); }
template <int BM, int COLS> __device__ __forceinline__ Place place_of(const FfnArgs& a, int rows, int id) {
    constexpr int BAND = 8;
    Place p{0, 0, 0};
    int m = rows >= 0 ? rows : a.prob[0].m;
    for (; p.which + 1 < a.problems; ++p.which) {
        m = rows >= 0 ? rows : a.prob[p.which].m;
        const int t = tiles_in<BM, COLS>(m, a.prob[p.which].n);
        if (id < t) break;
        id -= t;
    }
    m = rows >= 0 ? rows : a.prob[p.which].m;
    const int tiles_m = (m + BM - 1) / BM, tiles_n = (a.prob[p.which].n + COLS - 1) / COLS;
    const int band = id / (BAND * tiles_n), in_band = id - band * BAND * tiles_n, high = min(BAND, tiles_m - band * BAND);
    p.m0 = (band * BAND + in_band % high) * BM;
    p.n0 = in_band / high * COLS;
    return p;
}
template <int BM, int COLS> __device__ __forceinline__ int all_tiles(const FfnArgs& a, int rows) {
    int t = 0;
    for (int i = 0; i < a.problems; ++i) t += tiles_in<BM, COLS>(rows >= 0 ? rows : a.prob[i].m, a.prob[i].n);
    return t;
}

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
// C[m][n] = sum_k A(m, k) B(n, k).  Tiles of BM x BN by WM x WN wavefronts; *_ALONG: the contraction runs along the operand's rows in
// memory, otherwise across them.
template <typename E, int BM, int BN, int WM, int WN, bool A_ALONG, bool B_ALONG, Epilogue EPI, bool WHOLE>
__global__ void __launch_bounds__(64 * WM * WN, 2) ffn_product_kernel(FfnArgs a, int slots) {
    constexpr int WAVES = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;
    constexpr int TERMS = Mode<E, BM>::TERMS, BK = Mode<E, BM>::BK, STAGES = Mode<E, BM>::STAGES;
    constexpr bool GATED = EPI == EPI_GATED;
    using TA = Tile<BM, A_ALONG, WAVES, BK>;
    // WHOLE: B's 32-bit values are two elements of 16 bits each to what loads them
    constexpr int BI = WHOLE && !B_ALONG ? 2 * BN : BN, BK_B = WHOLE && B_ALONG ? 2 * BK : BK, N_BY = BI / BN, K_BY = BK_B / BK;
    constexpr int B_TERMS = WHOLE ? 1 : TERMS;
    static_assert(!WHOLE || (TERMS == 3 && BM == 128 && TN == 2), "as few registers as that");
    using TB = Tile<BI, B_ALONG, WAVES, BK_B>;
    constexpr int STAGE = TERMS * TA::BYTES + B_TERMS * TB::BYTES, LOADS = TERMS * TA::LOADS + B_TERMS * TB::LOADS;
    __shared__ __align__(1024) char lds[STAGES][STAGE];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / WN, wn = wave % WN;
    constexpr int COLS = GATED ? BN / 2 : BN;
    const int count = a.count ? *a.count : 0, rows = a.count && !a.count_is_k ? count : -1, K = a.count && a.count_is_k ? count : a.k;
    const int ksteps = (K + BK - 1) / BK;
    const Shares sh(all_tiles<BM, COLS>(a, rows), slots, ksteps * a.segments, Mode<E, BM>::LEAST);
    // this workgroup's steps, of `tile` and perhaps the one behind it
    int tile, from, left_steps;
    if ((int)blockIdx.x < sh.whole) {
        tile = stretch(blockIdx.x, sh.whole);
        from = 0;
        left_steps = sh.steps;
    } else {
        const int w = stretch(blockIdx.x - sh.whole, sh.sharers);
        if (w < 0) return;
        const int64_t first = (int64_t)w * sh.per, all = (int64_t)sh.rest * sh.steps;
        tile = sh.whole + (sh.steps > 0 ? (int)(first / sh.steps) : w);
        from = sh.steps > 0 ? (int)(first % sh.steps) : 0;
        left_steps = (int)min((int64_t)sh.per, all - first);
    }
    const int sharer = blockIdx.x < sh.whole ? 0 : stretch(blockIdx.x - sh.whole, sh.sharers);
    for (;;) {
        int lane = threadIdx.x & 63;
        asm("" : "+v"(lane));                       // addresses are found anew for each tile: there are no registers to keep them in
        const int n = min(left_steps, sh.steps - from);
        const Place at = place_of<BM, COLS>(a, rows, tile);
        const int which = at.which, m0 = at.m0, n0 = at.n0;
        const FfnProblem& pr = a.prob[which];
        const int M = rows >= 0 ? rows : pr.m, N = pr.n;

        TA ta;
        TB tb;
        ta.init(wave, lane, pr.a[0].stride);
        // gated: half of a wavefront's columns are the gate's and half the other projection's, in turn; it loads from one of them
        const int half = GATED ? wave & 1 : 0;
        static_assert(!GATED || TB::LOADS * TB::ROWS_A_LOAD == TN * 8, "a wavefront loads from one of the two projections");
        tb.init(GATED ? wave >> 1 : wave, lane, pr.b[0].stride);
        Reader<BM, A_ALONG, BK> ra;
        std::conditional_t<WHOLE, WholeReader<BN, B_ALONG>, Reader<BN, B_ALONG, BK>> rb;
        ra.init(wm * TM * 16, lane);
        rb.init(wn * TN * 16, lane);

        // where the next tiles to load stand
        int seg, left;
        Corner<A_ALONG, BK> ca;
        Corner<B_ALONG, BK_B> cb;
        const int64_t plane_a = pr.a[0].plane, plane_b = pr.b[0].plane;
        auto corners = [&] {
            ca.set(pr.a[seg], m0, min(M - m0, BM), K - left);
            cb.set(pr.b[GATED ? half : seg], n0 * N_BY, min(N - n0, BN) * N_BY, (K - left) * K_BY);
        };
        auto begin = [&] {
            seg = from / max(ksteps, 1);
            left = K - from % max(ksteps, 1) * BK;
            corners();
        };
        begin();
        auto load_terms = [&](int stage, int terms) {
#pragma unroll
            for (int t = 0; t < terms; ++t) {
                ta.load(lds[stage] + t * TA::BYTES, wave, ca.p + t * plane_a, ca.bytes(left), left);
                if (t < B_TERMS) tb.load(lds[stage] + TERMS * TA::BYTES + t * TB::BYTES, wave, cb.p + t * plane_b, cb.bytes(left * K_BY), left * K_BY);
            }
            ca.p += ca.step;
            cb.p += cb.step;
            left -= BK;
            if (left <= 0 && seg + 1 < a.segments) { ++seg; left = K; corners(); }
        };
        auto load = [&](int stage) { load_terms(stage, TERMS); };
        floatx4 acc[TM][TN] = {};
        // Two sets of operands, so that one comes from LDS while the products of the other run; STREAM: of A's only 16 rows each.
        constexpr bool STREAM = TERMS == 3 && BM == 256;
        bf16x8 fa[2][TERMS][STREAM ? 1 : TM], fb[WHOLE ? 1 : 2][TERMS][TN];
        float whole[2][WHOLE ? TN : 1][8];
        auto read_a = [&](int stage, int set, int i) {
#pragma unroll
            for (int t = 0; t < TERMS; ++t) fa[set][t][0] = ra.get(lds[stage] + t * TA::BYTES, i, 0);
            __builtin_amdgcn_sched_barrier(0);
        };
        auto read_b = [&](int stage, int set) {
#pragma unroll
            for (int t = 0; t < TERMS; ++t)
#pragma unroll
                for (int j = 0; j < TN; ++j)
                    if constexpr (!WHOLE) fb[set][t][j] = rb.get(lds[stage] + TERMS * TA::BYTES + t * TB::BYTES, j, 0);
        };
        auto multiply_row = [&](int set_a, int set_b, int i) {
#pragma unroll
            for (int order = TERMS - 1; order >= 0; --order)
#pragma unroll
                for (int t = 0; t <= order; ++t)
#pragma unroll
                    for (int j = 0; j < TN; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[set_b][order - t][j], fa[set_a][t][0], acc[i][j], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        };
        auto read = [&](int stage, int set, int kk) {
            const char *la = lds[stage], *lb = la + TERMS * TA::BYTES;
#pragma unroll
            for (int t = 0; t < TERMS; ++t) {
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    if constexpr (!WHOLE) fb[set][t][j] = rb.get(lb + t * TB::BYTES, j, kk);
                    else if (t == 0) rb.get(lb, j, whole[set][j]);
                }
#pragma unroll
                for (int i = 0; i < (STREAM ? 0 : TM); ++i) fa[set][t][i] = ra.get(la + t * TA::BYTES, i, kk);
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        // the products of terms above 2^-24, small ones first
        auto multiply = [&](int set) {
            if constexpr (WHOLE) {
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    bf16x8 t[3];
                    terms_of(whole[set][j], t);
                    fb[0][0][j] = t[0]; fb[0][1][j] = t[1]; fb[0][2][j] = t[2];
                }
            }
#pragma unroll
            for (int order = TERMS - 1; order >= 0; --order)
#pragma unroll
                for (int t = 0; t <= order; ++t)
#pragma unroll
                    for (int i = 0; i < (STREAM ? 0 : TM); ++i)
#pragma unroll
                        for (int j = 0; j < TN; ++j)
                            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[WHOLE ? 0 : set][order - t][j], fa[set][t][i], acc[i][j], 0, 0, 0);
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
        } else if constexpr (STREAM) {
            // A step goes through A 16 rows at a time; with the last of them begin the next step's operands and the loads of the one after.
            static_assert(!STREAM || (TM % 2 == 0 && STAGES == 2), "sets alternate");
            if (n > 0) {
                load(0);
                if (n > 1) { load(1); wait_loads<LOADS>(); } else { wait_loads<0>(); }
                read_b(0, 0);
                read_a(0, 0, 0);
                auto rows = [&](int stage, int set) {
#pragma unroll
                    for (int i = 0; i + 1 < TM; ++i) {
                        read_a(stage, i + 1 & 1, i + 1);
                        multiply_row(i & 1, set, i);
                    }
                };
                auto next = [&](int stage, int set) {
                    wait_loads<0>();
                    read_b(stage ^ 1, set ^ 1);
                    read_a(stage ^ 1, 0, 0);
                };
                int s = 0;
                for (; s + 3 < n; s += 2) {
                    rows(0, 0);
                    next(0, 0);
                    load(0);
                    multiply_row(1, 0, TM - 1);
                    rows(1, 1);
                    next(1, 1);
                    load(1);
                    multiply_row(1, 1, TM - 1);
                }
                for (; s < n; s += 2) {
                    rows(0, 0);
                    if (s + 1 < n) next(0, 0);
                    if (s + 2 < n) load(0);
                    multiply_row(1, 0, TM - 1);
                    if (s + 1 == n) break;
                    rows(1, 1);
                    if (s + 2 < n) next(1, 1);
                    if (s + 3 < n) load(1);
                    multiply_row(1, 1, TM - 1);
                }
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
        if constexpr (TERMS == 3) {
            // An infinite value is one term, and met all terms of the other operand, of which some are zero or of the other sign; so did
            // products that overflow.  A tile with sums that are NaN takes its steps again with first terms alone: infinite or NaN as in fp32
            // arithmetic.  us for 512 x 32 rows of 256 and 1024 with gradients: 403 without the check, 408 with it, 150 more if every tile does so.
            __shared__ unsigned odd[WAVES];
            bool nan = false;
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) nan |= __builtin_isunordered(acc[i][j][0], acc[i][j][1]) | __builtin_isunordered(acc[i][j][2], acc[i][j][3]);
            const unsigned any = __ballot(nan) != 0;
            if (lane == 0) odd[wave] = any;
            __syncthreads();                            // behind all reads of the last step
            unsigned all = 0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) all |= odd[w];
            if (__builtin_expect(all, 0)) {
                if constexpr (WHOLE) {                  // no registers to keep addresses in until here
                    asm("" : "+v"(lane));
                    ta.init(wave, lane, pr.a[0].stride);
                    tb.init(GATED ? wave >> 1 : wave, lane, pr.b[0].stride);
                    ra.init(wm * TM * 16, lane);
                    rb.init(wn * TN * 16, lane);
                }
                floatx4 first[TM][TN] = {};
                begin();
#pragma unroll 1
                for (int s = 0; s < n; ++s) {
                    load_terms(0, 1);
                    wait_loads<0>();
                    bf16x8 x, y[TN];
#pragma unroll
                    for (int j = 0; j < TN; ++j) {
                        if constexpr (WHOLE) {
                            float v[8];
                            bf16x8 t[3];
                            rb.get(lds[0] + TERMS * TA::BYTES, j, v);
                            terms_of(v, t);
                            y[j] = t[0];
                        } else {
                            y[j] = rb.get(lds[0] + TERMS * TA::BYTES, j, 0);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < TM; ++i) {
                        x = ra.get(lds[0], i, 0);
#pragma unroll
                        for (int j = 0; j < TN; ++j) first[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y[j], x, first[i][j], 0, 0, 0);
                    }
                    __syncthreads();                    // the next step's loads overwrite this one's
                }
                settle_products();
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[i][j][e] = acc[i][j][e] != acc[i][j][e] ? first[i][j][e] : acc[i][j][e];
            }
        }

        // Results go through LDS, so that whole lines of memory are read and written: column l % 16 of a product is a row of C, its rows
        // 4 (l / 16) .. + 3 are columns.  Then eight columns of a row a thread: the first four of each eight lie together, then the last
        // four, both in an order that depends on the row, so that neither side meets bank conflicts.
        constexpr int ALL = STAGES * STAGE, PASSES = (BM * BN * 4 + ALL - 1) / ALL, PM = TM / PASSES, ROWS = BM / PASSES, NT = 64 * WAVES;
        constexpr int UNITS = GATED ? BN / 16 : BN / 8, EACH = ROWS * UNITS / NT, AHEAD = 2;
        static_assert(PASSES * PM == TM && EACH % AHEAD == 0, "whole passes");
        static_assert(TERMS != 3 || PASSES == 1, "the check above has been waited for");
        char* stage = lds[0];
        auto granule = [&](int row, int g) { return (floatx4*)(stage + row * BN * 4 + ((((g >> 1) + (g & 1) * (BN / 8)) ^ (row & 15)) << 4)); };
        float* part = n == sh.steps ? nullptr : a.part + ((int64_t)sharer * 2 + (from == 0)) * (BM * BN);
#pragma unroll
        for (int pass = 0; pass < PASSES; ++pass) {
            if (TERMS != 3) __syncthreads();
#pragma unroll
            for (int i = 0; i < PM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    // gated: the gate's columns, then the other projection's
                    const int g = GATED ? (wn * (TN / 2) + j % (TN / 2)) * 4 + j / (TN / 2) * (BN / 8) : (wn * TN + j) * 4;
                    *granule((wm * PM + i) * 16 + (lane & 15), g + (lane >> 4)) = acc[pass * PM + i][j];
                }
            __syncthreads();
            // What stands behind the last column is an operand of the next products, against zeros: its sums are those of zeros, and NaN in
            // a row that holds an infinite value.
            if (EPI != EPI_OUT && N % 8 != 0 && n0 + COLS > N) {
                const int from = N - n0, behind = 8 - N % 8;
                for (int i = threadIdx.x; i < ROWS * behind; i += NT) {
                    const int row = i / behind, c = from + i % behind;
#pragma unroll
                    for (int h = 0; h < (GATED ? 2 : 1); ++h) ((float*)granule(row, (c >> 2) + h * (BN / 8)))[c & 3] = 0.f;
                }
                __syncthreads();
            }
            if (part) {
                for (int i = threadIdx.x; i < ROWS * (BN / 4); i += NT) {
                    const int local = i / (BN / 4), g = i % (BN / 4), row = (local / (PM * 16) * TM + pass * PM) * 16 + local % (PM * 16);
                    *(floatx4*)(part + row * BN + g * 4) = *granule(local, g);
                }
                continue;
            }
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
                    on[u] = row[u] < M && col[u] < (EPI == EPI_OUT ? N : a.hidden_p);
                    if constexpr (EPI == EPI_BACK) read_saved(a, on[u] ? (int64_t)row[u] * a.hidden_p + col[u] : 0, va[u], vb[u]);
                }
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    const int g = ((u0 + u) * NT + threadIdx.x) % UNITS * 2;
                    float x[8], y[8];
                    *(floatx4*)x = *granule(local[u], g);
                    *(floatx4*)(x + 4) = *granule(local[u], g + 1);
                    if constexpr (GATED) {
                        *(floatx4*)y = *granule(local[u], g + BN / 8);
                        *(floatx4*)(y + 4) = *granule(local[u], g + BN / 8 + 1);
                    }
                    if (on[u]) finish<E, EPI>(a, pr, row[u], col[u], x, y, va[u], vb[u]);
                }
            }
        }
        left_steps -= n;
        if (left_steps <= 0) break;
        ++tile;
        from = 0;
        __syncthreads();                            // the next tiles overwrite the results' place
    }
}

// Tiles whose sums are in parts: those of consecutive workgroups, added in order.  Eight columns of a row a thread.
template <typename E, int BM, int BN, Epilogue EPI> __global__ void __launch_bounds__(256) ffn_join_kernel(FfnArgs a, int slots, int bk) {
    constexpr int COLS = EPI == EPI_GATED ? BN / 2 : BN, UNITS = COLS / 8;
    const int count = a.count ? *a.count : 0, rows = a.count && !a.count_is_k ? count : -1, K = a.count && a.count_is_k ? count : a.k;
    const Shares sh(all_tiles<BM, COLS>(a, rows), slots, (K + bk - 1) / bk * a.segments, Mode<E, BM>::LEAST);
    if (!sh.joins()) return;
    constexpr int BLOCKS = BM * UNITS / 256;    // of a tile
    for (int b = blockIdx.x; b < sh.rest * BLOCKS; b += gridDim.x) {
        const int j = b / BLOCKS, unit = b % BLOCKS * 256 + threadIdx.x, local = unit / UNITS, c = unit % UNITS * 8;
        const int first = (int)((int64_t)j * sh.steps / sh.per), last = (int)((((int64_t)j + 1) * sh.steps - 1) / sh.per);
        if (first == last) continue;
        const Place at = place_of<BM, COLS>(a, rows, sh.whole + j);
        const FfnProblem& pr = a.prob[at.which];
        const int row = at.m0 + local, col = at.n0 + c;
        if (row >= (rows >= 0 ? rows : pr.m) || col >= (EPI == EPI_OUT ? pr.n : a.hidden_p)) continue;
        float x[8] = {}, y[8] = {};
        for (int w = first; w <= last; ++w) {
            const float* p = a.part + ((int64_t)w * 2 + (w == first)) * (BM * BN) + local * BN + c;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const floatx4 v = *(const floatx4*)(p + 4 * h);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[4 * h + e] += v[e];
                if constexpr (EPI == EPI_GATED) {
                    const floatx4 u = *(const floatx4*)(p + COLS + 4 * h);
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[4 * h + e] += u[e];
                }
            }
        }
        floatx4 va[2], vb[2];
        if constexpr (EPI == EPI_BACK) read_saved(a, (int64_t)row * a.hidden_p + col, va, vb);
        finish<E, EPI>(a, pr, row, col, x, y, va, vb);
    }
}

// ---- preparation ------------------------------------------------------------------------------------------
// Matrices as planes of padded rows.  Rows of tokens are packed where sequences have lengths, and `clear`'s that do not count become
// zeros.  A workgroup of packed rows takes a stretch of all rows, counts those that count before it itself, and finds the places of its
// own from counts of the lanes and wavefronts before; one matrix's note which row each packed one is, and how many there are.
struct FfnCopy { const void* from; int64_t stride; bf16_t* to; int64_t plane; int rows, cols, cols_p, packed; };
struct FfnCopies {
    FfnCopy c[5];
    int n, token_blocks;
    int *map, *count;
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
    const int each = c.cols_p / 8;
    const bool al = (c.stride * sizeof(E)) % 16 == 0 && ((uintptr_t)c.from & 15) == 0;
    auto copy = [&](int64_t from, int64_t to, int col) {
        const E* p = (const E*)c.from + from * c.stride + col;
        float x[8];
        if (al && col + 8 <= c.cols) {
#pragma unroll
            for (int g = 0; g < 8 / VEC_OF<E>; ++g) widen(((const uint4*)p)[g], x + g * VEC_OF<E>, E{});
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = col + e < c.cols ? to_float(p[e]) : 0.f;
        }
        store_terms<E>(c.to + to * c.cols_p + col, c.plane, x);
    };
    if (!c.packed) {
        for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < (int64_t)c.rows * each; i += gridDim.x * 256ll) {
            const int row = (int)(i / each);
            copy(row, row, (int)(i - (int64_t)row * each) * 8);
        }
        return;
    }
    __shared__ int sums[4], places[256];
    const int per = (c.rows + a.token_blocks - 1) / a.token_blocks, steps = (int)a.live.steps;
    const int64_t first = (int64_t)blockIdx.x * per, last = min(first + per, (int64_t)c.rows);
    if ((int)blockIdx.x >= a.token_blocks || first >= last) return;
    auto length = [&](int b) { return min(max(a.live.lengths[b], 0), steps); };
    // rows that count before `first`: whole sequences, and the beginning of the one it lies in
    const int b0 = (int)(first / steps), t0 = (int)(first - (int64_t)b0 * steps);
    int mine = 0;
    for (int b = threadIdx.x; b < b0; b += 256) mine += length(b);
    for (int d = 1; d < 64; d <<= 1) mine += __shfl_xor(mine, d);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = mine;
    __syncthreads();
    int done = sums[0] + sums[1] + sums[2] + sums[3] + (t0 > 0 ? min(t0, length(b0)) : 0);
    const bool notes = c.packed == 2;
    for (int64_t r0 = first; r0 < last; r0 += 256) {
        const int64_t r = r0 + threadIdx.x;
        const bool live = r < last && a.live((unsigned)r);
        const uint64_t mask = __ballot(live);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = __popcll(mask);
        __syncthreads();
        int at = done + __popcll(mask & ((1ull << (threadIdx.x & 63)) - 1));
        for (int w = 0; w < (int)(threadIdx.x >> 6); ++w) at += sums[w];
        places[threadIdx.x] = live ? at : -1;
        if (live && notes) a.map[at] = (int)r;
        done += sums[0] + sums[1] + sums[2] + sums[3];
        __syncthreads();
        const int all = (int)min(last - r0, (int64_t)256) * each;
        for (int i = threadIdx.x; i < all; i += 256) {
            const int row = i / each;
            if (places[row] >= 0) copy(r0 + row, places[row], (i - row * each) * 8);
        }
    }
    if (notes && last == c.rows && threadIdx.x == 0) *a.count = done;
}

// ---- host -------------------------------------------------------------------------------------------------
bool ffn_ok(const pql_ffn_shape& s) {
    return s.batch >= 0 && s.steps >= 0 && (double)s.batch * s.steps < 1073741824.0 && s.dim >= 1 && s.dim <= PQL_FFN_MAX_DIM && s.hidden >= 1 &&
           s.hidden <= PQL_FFN_MAX_DIM && (s.dtype == PQL_F32 || s.dtype == PQL_BF16) && s.act >= PQL_ACT_NONE && s.act <= PQL_ACT_RELU;
}
int ffn_rows(const pql_ffn_shape& s) { return (int)((int64_t)s.batch * s.steps); }
int up8(int x) { return (x + 7) / 8 * 8; }
int tiles_of(int x, int b) { return (x + b - 1) / b; }

// Rows of the tiles of a product of `problems` m x n results, 256 where such tiles fill the card, and columns.
int tile_cols(int32_t dtype, int rows) { return dtype == PQL_BF16 ? rows : 128; }
int tile_rows(int32_t dtype, int64_t m, int n, int problems) {
    return (int64_t)tiles_of((int)m, 256) * tiles_of(n, tile_cols(dtype, 256)) * problems >= BIG_TILES ? 256 : 128;
}

// One product's tiles, workgroups at a time, and the steps of its contraction, at most.
struct FfnTiles { int rows, cols; int64_t tiles; int slots, steps; };
FfnTiles ffn_tiles(int32_t dtype, int64_t m, int n, int problems, int of, int64_t k, int segments, bool gated, bool whole = false) {
    FfnTiles t{};
    t.rows = whole ? 128 : tile_rows(dtype, m, gated ? 2 * n : n, of);
    t.cols = tile_cols(dtype, t.rows);
    t.tiles = (int64_t)tiles_of((int)m, t.rows) * tiles_of(n, gated ? t.cols / 2 : t.cols) * problems;
    t.slots = dtype == PQL_BF16 && t.rows == 128 ? 512 : 256;          // two workgroups a compute unit, one where LDS holds no more
    t.steps = tiles_of((int)k, dtype == PQL_F32 ? 32 : 64) * segments;
    return t;
}
// Bytes of the parts that as many workgroups may leave.
size_t part_bytes(const FfnTiles& t) {
    if (t.steps <= JOIN_STEPS) return 0;
    const int64_t most = t.tiles * t.steps;
    return (size_t)(most < t.slots ? most : t.slots) * 2 * t.rows * t.cols * 4;
}
struct FfnPlan {
    int rows, terms, dim_p, hidden_p;
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
    size_t o = 0, part = 0;
    auto take = [&](size_t b) { const size_t at = o; o += to256(b); return at; };
    auto planes = [&](int64_t plane) { return take((size_t)plane * p.terms * 2); };
    auto parts = [&](const FfnTiles& t) { const size_t b = part_bytes(t); part = b > part ? b : part; };
    p.map = take((size_t)p.rows * 4);
    p.count = take(4);
    p.x = planes(p.x_plane);
    p.gate = planes(p.gate_plane);
    p.up = planes(p.gate_plane);
    p.down = planes(p.down_plane);
    if (call != PQL_FFN_BACKWARD) {
        parts(ffn_tiles(s.dtype, p.rows, s.hidden, 1, 1, s.dim, 1, true));
        // the kernels for few rows keep two terms
        p.m = take((size_t)p.m_plane * 2 * (p.terms == 1 && call == PQL_FFN_FORWARD && p.rows <= FFN_FEW_ROWS ? 2 : p.terms));
    }
    if (call == PQL_FFN_FORWARD) {
        parts(ffn_tiles(s.dtype, p.rows, s.dim, 1, 1, s.hidden, 1, false));
    } else {
        p.dout = planes(p.x_plane);
        p.da = planes(p.m_plane);
        p.db = planes(p.m_plane);
        if (call == PQL_FFN_BACKWARD_ALONE) { p.va = take((size_t)p.m_plane * 4); p.vb = take((size_t)p.m_plane * 4); }
        parts(ffn_tiles(s.dtype, p.rows, s.hidden, 1, 1, s.dim, 1, false));
        parts(ffn_tiles(s.dtype, p.rows, s.dim, 1, 1, s.hidden, 2, false));
        // the weights' gradients: three products, some of them the others' transposes
        for (int i = 0; i < 2; ++i) parts(ffn_tiles(s.dtype, i ? s.dim : s.hidden, i ? s.hidden : s.dim, 3, 3, p.rows, 1, false));
    }
    p.part = take(part);
    p.bytes = o;
    return p;
}
// What a forward call saves: a, b, m.
struct FfnSaved {
    size_t b, m, bytes;
    explicit FfnSaved(const FfnPlan& p) {
        b = to256((size_t)p.m_plane * 4);
        m = 2 * b;
        bytes = m + to256((size_t)p.m_plane * p.terms * 2);
    }
};

template <typename E, int BM, int BN, int WM, int WN, bool A_ALONG, bool B_ALONG, Epilogue EPI, bool WHOLE = false>
hipError_t launch_product(const FfnTiles& t, const FfnArgs& a, int kid, double flops, hipStream_t st) {
    // A grid holds at most 2^32 - 1 threads, 2^23 workgroups of 512.  Rows are fewer than 2^30, so that two columns of tiles stay below that,
    // and m of three columns or more (64 KB a tile) would not fit the memory.
    if ((t.tiles + t.slots) * 64 * WM * WN > 0xffffffffll) return hipErrorInvalidConfiguration;
    ProfSlot ps = prof_slot();
    const Shares sh((int)t.tiles, t.slots, t.steps, Mode<E, BM>::LEAST);
    // with rows that are counted on the device, fewer tiles may be shared out otherwise
    const int grid = a.count ? (int)t.tiles / t.slots * t.slots + t.slots : sh.whole + (sh.sharers + 7) / 8 * 8;
    PQL_LAUNCH(ps, (ffn_product_kernel<E, BM, BN, WM, WN, A_ALONG, B_ALONG, EPI, WHOLE>), dim3(grid), dim3(64 * WM * WN), 0, st, a, t.slots);
    prof_commit(ps, kid, flops, 0.0);
    if (a.count ? t.steps >= JOIN_STEPS + Mode<E, BM>::LEAST : sh.joins()) {
        const int blocks = (a.count ? t.slots : sh.rest) * (BM * (EPI == EPI_GATED ? BN / 2 : BN) / 8 / 256);
        ps = prof_slot();
        PQL_LAUNCH(ps, (ffn_join_kernel<E, BM, BN, EPI>), dim3(blocks < 1024 ? blocks : 1024), dim3(256), 0, st, a, t.slots, sizeof(E) == 4 ? 32 : 64);
        prof_commit(ps, KID_FFN_JOIN, 0.0, 0.0);
    }
    return hipGetLastError();
}

// Whether 32-bit weights can be read as they are: whole granules of what becomes 16 bits, too.
bool whole_ok(const pql_ffn_shape& s, const pql_rows& r, int cols) {
    return s.dtype == PQL_F32 && ffn_rows(s) <= WHOLE_ROWS && s.dim % 8 == 0 && s.hidden % 8 == 0 && rows_aligned(r, s.dtype) && r.stride >= cols &&
           r.stride <= 1 << 20;
}

struct FfnRun {
    const pql_ffn_shape& s;
    const FfnPlan& p;
    char* ws;
    hipStream_t st;
    hipError_t e = hipSuccess;
    const int *map = nullptr, *count = nullptr;
    FfnCopies copies{};
    bool noted = false;
    int elem() const { return s.dtype == PQL_F32 ? 4 : 2; }

    template <typename T> T* at(size_t o) const { return (T*)(ws + o); }
    void pack(const int32_t* lengths) {
        copies.live = {lengths, (unsigned)s.steps};
        if (!lengths) return;
        map = copies.map = at<int>(p.map);
        count = copies.count = at<int>(p.count);
        const int blocks = (p.rows + 7) / 8;
        copies.token_blocks = blocks < 512 ? blocks : 512;
    }
    // The matrix as an operand: where it is, or as planes at `to`.
    FfnOperand operand(const pql_rows& r, int rows, int cols, size_t to, int64_t plane, bool tokens, bool direct = true) {
        if (direct && s.dtype == PQL_BF16 && !(tokens && map) && cols % 8 == 0 && rows_aligned(r, s.dtype) && r.stride >= cols && r.stride <= 1 << 20)
            return {(const bf16_t*)r.data, r.stride, 0, false};
        if (direct && !tokens && whole_ok(s, r, cols))
            return {(const bf16_t*)r.data, 2 * r.stride, 0, true};
        const int packed = tokens && map ? (noted ? 1 : 2) : 0;         // 2: with the notes, that all of them would make alike
        if (packed) noted = true;
        copies.c[copies.n++] = {r.data, r.stride, at<bf16_t>(to), plane, rows, cols, up8(cols), packed};
        return {at<bf16_t>(to), up8(cols), plane, false};
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
        int64_t most = copies.clear ? copies.clear_rows * 256ll : 0, bytes = 0;
        for (int i = 0; i < copies.n; ++i) {
            const int64_t n = (int64_t)copies.c[i].rows * copies.c[i].cols_p / 8;
            most = n > most ? n : most;
            bytes += n * 8 * (elem() + 2 * p.terms);
        }
        int64_t blocks = (most + 255) / 256;
        blocks = blocks < copies.token_blocks ? copies.token_blocks : blocks;
        const ProfSlot ps = prof_slot();
        const dim3 grid((unsigned)(blocks < 2048 ? blocks : 2048), y);
        if (s.dtype == PQL_F32) PQL_LAUNCH(ps, ffn_prepare_kernel<float>, grid, dim3(256), 0, st, copies);
        else PQL_LAUNCH(ps, ffn_prepare_kernel<bf16_t>, grid, dim3(256), 0, st, copies);
        prof_commit(ps, KID_FFN_PREPARE, 0.0, (double)bytes);
        e = hipGetLastError();
    }
    FfnArgs args() const {
        FfnArgs a{};
        a.problems = 1; a.segments = 1;
        a.count = count; a.map = map; a.act = s.act;
        a.hidden_p = p.hidden_p; a.m_plane = p.m_plane;
        a.part = at<float>(p.part);
        return a;
    }
    // of: the problems of a full call, which the plan has counted with.
    template <bool A_ALONG, bool B_ALONG, Epilogue EPI> void product(const FfnArgs& a, int of, int kid) {
        if (e != hipSuccess) return;
        const FfnProblem& pr = a.prob[0];
        const bool whole = pr.b[0].whole;
        FfnTiles t = ffn_tiles(s.dtype, pr.m, pr.n, 1, of, a.k, a.segments, EPI == EPI_GATED, whole);
        t.tiles = 0;
        for (int i = 0; i < a.problems; ++i)
            t.tiles += (int64_t)tiles_of(a.prob[i].m, t.rows) * tiles_of(a.prob[i].n, EPI == EPI_GATED ? t.cols / 2 : t.cols);
        const double flops = 2.0 * a.problems * (EPI == EPI_GATED ? 2 : 1) * a.segments * pr.m * pr.n * a.k;
        if (whole) {
            if constexpr (A_ALONG) e = launch_product<float, 128, 128, 2, 4, A_ALONG, B_ALONG, EPI, true>(t, a, kid, flops, st);
        } else if (s.dtype == PQL_F32)
            e = t.rows == 256 ? launch_product<float, 256, 128, 2, 4, A_ALONG, B_ALONG, EPI>(t, a, kid, flops, st)
                              : launch_product<float, 128, 128, 2, 4, A_ALONG, B_ALONG, EPI>(t, a, kid, flops, st);
        else
            e = t.rows == 256 ? launch_product<bf16_t, 256, 256, 2, 4, A_ALONG, B_ALONG, EPI>(t, a, kid, flops, st)
                              : launch_product<bf16_t, 128, 128, 2, 2, A_ALONG, B_ALONG, EPI>(t, a, kid, flops, st);
    }
    void gated(const FfnOperand& x, const FfnOperand& gate, const FfnOperand& up, float* va, float* vb, bf16_t* m) {
        FfnArgs a = args();
        a.prob[0] = {{x, x}, {gate, up}, p.rows, s.hidden, nullptr, 0};
        a.k = s.dim;
        a.va = va; a.vb = vb; a.m = m;
        product<true, true, EPI_GATED>(a, 1, KID_FFN_GATED);
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
    return (int64_t)FfnSaved(ffn_plan(*s, PQL_FFN_FORWARD)).bytes;
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
    const bool whole = in->gate.stride == in->up.stride && whole_ok(*s, in->gate, s->dim) && whole_ok(*s, in->up, s->dim) && whole_ok(*s, in->down, s->hidden);
    if (p.rows <= ffn_few_rows(s->dtype, (int64_t)s->dim * s->hidden, whole) && !saved) {
        FfnRowsArgs a{{in->lengths, (unsigned)s->steps}, p.rows, s->dim, s->hidden, s->act, in->x.data, in->gate.data, in->up.data, in->down.data,
                      in->x.stride, in->gate.stride, in->up.stride, in->down.stride, (char*)workspace + p.m, p.hidden_p, p.m_plane, out->data, out->stride};
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
        const FfnSaved keep(p);
        bf16_t* m = saved ? (bf16_t*)((char*)saved + keep.m) : r.at<bf16_t>(p.m);
        r.gated(x, gate, up, (float*)saved, saved ? (float*)((char*)saved + keep.b) : nullptr, m);
        FfnArgs a = r.args();
        const FfnOperand om{m, p.hidden_p, p.m_plane, false};
        a.prob[0] = {{om, om}, {down, down}, p.rows, s->dim, out->data, out->stride};
        a.k = s->hidden;
        r.product<true, true, EPI_OUT>(a, 1, KID_FFN_PRODUCT);
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
        const FfnOperand down = r.operand(in->down, s->dim, s->hidden, p.down, p.down_plane, false);
        if (g->x.data) r.clear(g->x);
        r.prepare();
        const FfnSaved keep(p);
        float *va = saved ? (float*)saved : r.at<float>(p.va), *vb = saved ? (float*)((char*)saved + keep.b) : r.at<float>(p.vb);
        m = {saved ? (const bf16_t*)((const char*)saved + keep.m) : r.at<bf16_t>(p.m), p.hidden_p, p.m_plane, false};
        if (!saved) r.gated(x, gate, up, va, vb, (bf16_t*)m.p);
        da = {r.at<bf16_t>(p.da), p.hidden_p, p.m_plane, false};
        db = {r.at<bf16_t>(p.db), p.hidden_p, p.m_plane, false};
        FfnArgs a = r.args();
        a.prob[0] = {{dout, dout}, {down, down}, rows, s->hidden, nullptr, 0};
        a.k = s->dim;
        a.va = va; a.vb = vb; a.da = (bf16_t*)da.p; a.db = (bf16_t*)db.p;
        r.product<true, false, EPI_BACK>(a, 1, KID_FFN_BACK);
        if (g->x.data) {
            a = r.args();
            a.prob[0] = {{da, db}, {gate, up}, rows, s->dim, g->x.data, g->x.stride};
            a.k = s->hidden;
            a.segments = 2;
            r.product<true, false, EPI_OUT>(a, 1, KID_FFN_PRODUCT);
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
    w.problems = n;
    if (n > 0) r.product<false, false, EPI_OUT>(w, 3, KID_FFN_PRODUCT);
    return r.e == hipSuccess ? PQL_OK : ctx_fail(c, PQL_ERR_HIP, "pql_ffn_backward", r.e);
}

}  // extern "C"
