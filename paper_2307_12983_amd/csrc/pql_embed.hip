// Embeddings (include/pql_block.h): out_n = s sum_j E[token_nj], and the gradient of the table,
// dE_v = s sum over (n, j) with token_nj = v of dOut_n.
//
// The lookup is bound by memory: a row of the output is one group of lanes, 16 bytes each.  The gradient sorts the
// places (n, j) by token, keeping their order, so that every row of the table has one run of places whose sum is taken in
// one order.  The table's rows are cleared while the list is sorted.  Then a wavefront works through a chunk of the list: runs
// that begin and end in it are written, of the others it sums its part, and a last launch joins the parts in order.  That
// bounds the work on one run, however often its token occurs.
//
// 512 x 32 rows of 256 in fp32, 20 tokens of 1020 each: the lookup takes 17 us (rows come from the caches at 21 TB/s), the gradient
// 51 us, half of it the three launches of the sort and half the sums (18 TB/s).  8192 rows of 2048 in bf16, a token of 65536 each: 19 us and
// 84 us, of which 54 us clear the table at 5 TB/s while the tokens are sorted beside.
#include "pql_block_internal.h"

namespace pql {
namespace {

struct EmbedArgs {
    const int* tokens;
    Live live;
    unsigned rows;
    int per_row, vocab, dim;
    float scale;
    const void* table; int64_t table_stride;        // the table, or its gradient
    void* out; int64_t out_stride;                  // the output, or its gradient
    // gradient
    unsigned n;                                     // places
    int chunk, chunks;                              // places of a chunk (a power of two), chunks of the list
    unsigned *key, *row, *key_to, *row_to;          // sorted tokens and the rows of their places; where a pass puts them
    unsigned *count, *total;                        // sort: [tiles][digits], [digits]
    int bits, shift, tiles;                         // of a digit
    unsigned sort_blocks;                           // the first launch's blocks behind them clear the table
    int elem;                                       // bytes of an element
    float* part;                                    // [chunks][2][dim]: a chunk's first and last run, where those cross its ends
};

// ---- lookup --------------------------------------------------------------------------------------
// `lanes` consecutive lanes (a power of two, at most 256) per row.
template <typename E, bool AL> __global__ void __launch_bounds__(256) embed_kernel(EmbedArgs a, int lanes) {
    constexpr int V = AL ? VEC_OF<E> : 1;
    const unsigned by = 256u / lanes;
    for (unsigned n = blockIdx.x * by + threadIdx.x / lanes; n < a.rows; n += gridDim.x * by) {
        const bool live = a.live(n);
        const int* tokens = a.tokens + (int64_t)n * a.per_row;
        E* out = (E*)a.out + n * a.out_stride;
        for (int at = (threadIdx.x & (lanes - 1)) * V; at < a.dim; at += lanes * V) {
            float sum[V] = {};
            if (live) {
#pragma unroll 4
                for (int j = 0; j < a.per_row; ++j) {
                    const int t = tokens[j];
                    const bool there = (unsigned)t < (unsigned)a.vocab;
                    const E* p = (const E*)a.table + (there ? t : 0) * a.table_stride + at;
                    float x[V];
                    if constexpr (AL) widen(*(const uint4*)p, x, E{}); else x[0] = to_float(*p);
#pragma unroll
                    for (int i = 0; i < V; ++i) sum[i] += there ? x[i] : 0.f;
                }
            }
#pragma unroll
            for (int i = 0; i < V; ++i) sum[i] *= a.scale;
            if constexpr (AL) *(uint4*)(out + at) = narrow(sum, E{}); else out[at] = from_float<E>(sum[0]);
        }
    }
}

// ---- sort ----------------------------------------------------------------------------------------
// A place's key: its token, or vocab for a place that counts for nothing.
__device__ __forceinline__ unsigned row_of(const EmbedArgs& a, unsigned i) { return a.per_row == 1 ? i : i / a.per_row; }
__device__ __forceinline__ unsigned key_of(const EmbedArgs& a, unsigned i) {
    const unsigned t = min((unsigned)a.tokens[i], (unsigned)a.vocab);
    return !a.live.lengths || a.live(row_of(a, i)) ? t : (unsigned)a.vocab;
}
// Zeros for rows of the table, by the blocks from sort_blocks on: 16 bytes a lane where rows allow it.
__device__ __forceinline__ void clear_table(const EmbedArgs& a) {
    const int64_t bytes = (int64_t)a.dim * a.elem, stride = a.table_stride * a.elem;
    const int unit = ((uintptr_t)a.table | bytes | stride) % 16 == 0 ? 16 : a.elem, each = (int)(bytes / unit);
    // lanes of a row, a power of two; rows of a workgroup
    int lanes = 1;
    while (lanes < (int)blockDim.x && lanes < each) lanes *= 2;
    const int by = blockDim.x / lanes, lane = threadIdx.x & (lanes - 1);
    for (int64_t v = (int64_t)(blockIdx.x - a.sort_blocks) * by + threadIdx.x / lanes; v < a.vocab; v += (int64_t)(gridDim.x - a.sort_blocks) * by) {
        char* p = (char*)a.table + v * stride;
        for (int i = lane; i < each; i += lanes) {
            if (unit == 16) *(uint4*)(p + i * 16ll) = make_uint4(0, 0, 0, 0);
            else if (unit == 4) *(unsigned*)(p + i * 4ll) = 0;
            else *(unsigned short*)(p + i * 2ll) = 0;
        }
    }
}

// Few places (at most RANK_MAX): each one's place in the sorted list is the number of smaller keys and of equal ones before it.  All
// pairs are compared, with the keys in LDS: one launch where a pass over a digit takes three.  PACKED: key and place in one number
// (vocab below 2^19), so that one comparison decides.  us for 8192 places of 65536 tokens 27 (by digits 42), of 1000 17 (17); for 4097 of 1000
// 10 (17).
constexpr int RANK_BITS = 13, RANK_MAX = 1 << RANK_BITS, RANK_WG = 256, RANK_LANES = 8;
template <bool PACKED> __global__ void __launch_bounds__(RANK_WG) embed_rank_kernel(EmbedArgs a) {
    __shared__ uint4 keys4[RANK_MAX / 4];
    unsigned* keys = (unsigned*)keys4;
    if (blockIdx.x >= a.sort_blocks) return clear_table(a);
    const unsigned padded = (a.n + 4 * RANK_LANES - 1) / (4 * RANK_LANES) * (4 * RANK_LANES);
#pragma unroll 8
    for (unsigned i = threadIdx.x; i < padded; i += RANK_WG) {
        const unsigned k = i < a.n ? key_of(a, i) : ~0u;
        keys[i] = PACKED && i < a.n ? k << RANK_BITS | i : k;
    }
    __syncthreads();
    // lane l of a place's RANK_LANES compares it with every RANK_LANES-th four of keys
    const unsigned i = blockIdx.x * (RANK_WG / RANK_LANES) + threadIdx.x / RANK_LANES, lane = threadIdx.x % RANK_LANES;
    const unsigned mine = keys[min(i, a.n - 1)];
    unsigned before = 0;
#pragma unroll 4
    for (unsigned q = lane; q < padded / 4; q += RANK_LANES) {
        const uint4 k = keys4[q];
        if constexpr (PACKED) {
            before += (k.x < mine) + (k.y < mine) + (k.z < mine) + (k.w < mine);
        } else {                                    // equal keys count where they stand before
            const unsigned j = 4 * q;
            before += (k.x < mine || (k.x == mine && j < i)) + (k.y < mine || (k.y == mine && j + 1 < i))
                    + (k.z < mine || (k.z == mine && j + 2 < i)) + (k.w < mine || (k.w == mine && j + 3 < i));
        }
    }
#pragma unroll
    for (int d = 1; d < RANK_LANES; d <<= 1) before += __shfl_xor(before, d);
    if (lane == 0 && i < a.n) { a.key_to[before] = PACKED ? mine >> RANK_BITS : mine; a.row_to[before] = row_of(a, i); }
}

// More places: passes over digits of at most DIGIT_BITS bits, from the lowest, each keeping the order of equal digits.
constexpr int DIGIT_BITS = 10, SORT_WG = 256, SORT_WAVES = SORT_WG / 64, TILE = 2048, PER_WAVE = TILE / SORT_WAVES;
template <bool FIRST> __device__ __forceinline__ unsigned sort_key(const EmbedArgs& a, unsigned i, unsigned& row) {
    if constexpr (FIRST) { row = row_of(a, i); return key_of(a, i); }
    else { row = a.row[i]; return a.key[i]; }
}
template <bool FIRST> __global__ void __launch_bounds__(SORT_WG) embed_count_kernel(EmbedArgs a) {
    __shared__ unsigned count[1 << DIGIT_BITS];
    if (FIRST && blockIdx.x >= a.sort_blocks) return clear_table(a);
    const int digits = 1 << a.bits;
    for (int d = threadIdx.x; d < digits; d += SORT_WG) count[d] = 0;
    __syncthreads();
    const unsigned from = blockIdx.x * (unsigned)TILE, to = min(from + TILE, a.n);
    for (unsigned i = from + threadIdx.x; i < to; i += SORT_WG) {
        unsigned row;
        atomicAdd(&count[sort_key<FIRST>(a, i, row) >> a.shift & (digits - 1)], 1u);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < digits; d += SORT_WG) a.count[(int64_t)blockIdx.x * digits + d] = count[d];
}
// For each digit: the counts of the tiles become those of all tiles before, their sum goes to total.  64 digits a workgroup, the
// tiles in 16 stretches.
__global__ void __launch_bounds__(1024) embed_tiles_kernel(EmbedArgs a) {
    __shared__ unsigned sums[16][64];
    const int digits = 1 << a.bits, d = blockIdx.x * 64 + (threadIdx.x & 63), part = threadIdx.x >> 6;
    const int each = (a.tiles + 15) / 16, from = part * each, to = min(from + each, a.tiles);
    unsigned sum = 0;
    if (d < digits)
        for (int t = from; t < to; ++t) sum += a.count[(int64_t)t * digits + d];
    sums[part][threadIdx.x & 63] = sum;
    __syncthreads();
    if (d >= digits) return;
    unsigned before = 0, all = 0;
    for (int p = 0; p < 16; ++p) {
        const unsigned s = sums[p][threadIdx.x & 63];
        if (p < part) before += s;
        all += s;
    }
    for (int t = from; t < to; ++t) {
        unsigned* c = a.count + (int64_t)t * digits + d;
        const unsigned x = *c;
        *c = before;
        before += x;
    }
    if (part == 0) a.total[d] = all;
}
// What lanes of a wavefront have read from and written to LDS before comes before what they read and write behind it.
__device__ __forceinline__ void lanes_meet() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}
template <bool FIRST> __global__ void __launch_bounds__(SORT_WG) embed_move_kernel(EmbedArgs a) {
    __shared__ unsigned at[SORT_WAVES][1 << DIGIT_BITS];
    __shared__ unsigned sums[SORT_WAVES];
    const int digits = 1 << a.bits, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int d = threadIdx.x; d < digits; d += SORT_WG)
#pragma unroll
        for (int w = 0; w < SORT_WAVES; ++w) at[w][d] = 0;
    __syncthreads();
    const unsigned from = blockIdx.x * (unsigned)TILE + wave * PER_WAVE, to = min(from + PER_WAVE, a.n);
    unsigned key[PER_WAVE / 64], row[PER_WAVE / 64];
#pragma unroll
    for (int r = 0; r < PER_WAVE / 64; ++r) {
        const unsigned i = from + r * 64 + lane;
        key[r] = 0;
        row[r] = 0;
        if (i < to) {
            key[r] = sort_key<FIRST>(a, i, row[r]);
            atomicAdd(&at[wave][key[r] >> a.shift & (digits - 1)], 1u);
        }
    }
    __syncthreads();
    // where each wavefront's first place of every digit goes: the digits before, the tiles before, the wavefronts before
    const int each = (digits + SORT_WG - 1) / SORT_WG, first = threadIdx.x * each;
    unsigned mine = 0;
    for (int d = first; d < min(first + each, digits); ++d) mine += a.total[d];
    unsigned up = mine;
    for (int d = 1; d < 64; d <<= 1) {
        const unsigned x = __shfl_up(up, d);
        if (lane >= d) up += x;
    }
    if (lane == 63) sums[wave] = up;
    __syncthreads();
    unsigned start = up - mine;
    for (int w = 0; w < wave; ++w) start += sums[w];
    for (int d = first; d < min(first + each, digits); ++d) {
        unsigned go = start + a.count[(int64_t)blockIdx.x * digits + d];
        start += a.total[d];
#pragma unroll
        for (int w = 0; w < SORT_WAVES; ++w) { const unsigned c = at[w][d]; at[w][d] = go; go += c; }
    }
    __syncthreads();
    // 64 places at a time: lanes of one digit in order
#pragma unroll
    for (int r = 0; r < PER_WAVE / 64; ++r) {
        const unsigned i = from + r * 64 + lane;
        const unsigned d = key[r] >> a.shift & (digits - 1);
        uint64_t same = __ballot(i < to);
        for (int b = 0; b < a.bits; ++b) {
            const uint64_t set = __ballot(d >> b & 1);
            same &= d >> b & 1 ? set : ~set;
        }
        if (i < to) {
            const int before = __popcll(same & ((1ull << lane) - 1));
            const unsigned go = at[wave][d] + before;
            a.key_to[go] = key[r];
            a.row_to[go] = row[r];
            // the last lane of a digit counts on, when the others have read, and for those of the next 64 places
            lanes_meet();
            if (same >> lane == 1) at[wave][d] = go + 1;
        }
        lanes_meet();
    }
}

// ---- sums over runs ------------------------------------------------------------------------------
// The first place whose key is at least v, by 64 lanes at a time.
__device__ __forceinline__ unsigned first_place(const EmbedArgs& a, unsigned v) {
    unsigned from = 0, to = a.n;                // the answer lies in [from, to]
    const int lane = threadIdx.x & 63;
    while (to > from) {
        const unsigned step = (to - from + 63) / 64, i = from + lane * step;
        const uint64_t less = __ballot(i < to && a.key[i] < v);         // the lower lanes
        const int count = __popcll(less);
        if (count == 0) return from;
        const unsigned low = from + (count - 1) * step + 1;
        to = min(to, from + count * step);
        from = low;
    }
    return from;
}

// A wavefront a chunk, NV granules of V columns a lane.
template <typename E, bool AL, int NV> __global__ void __launch_bounds__(256) embed_sum_kernel(EmbedArgs a) {
    constexpr int V = AL ? VEC_OF<E> : 1, AHEAD = 8;
    const unsigned c = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    if (c >= (unsigned)a.chunks) return;
    const int lane = threadIdx.x & 63, col = blockIdx.y * 64 * NV * V;
    const unsigned from = c * a.chunk, to = min(from + a.chunk, a.n);
    const unsigned previous = from > 0 ? a.key[from - 1] : ~0u, next = to < a.n ? a.key[to] : ~0u;
    unsigned run = a.key[from];
    float sum[NV * V] = {};
    // the run's sum goes to its row of the table, or to the chunk's parts if it begins before it (slot 0) or goes on behind it
    auto put = [&](bool last) {
        if (run >= (unsigned)a.vocab) return;
        const bool before = run == previous, behind = last && run == next;
        if (before || behind) {
            float* p = a.part + ((int64_t)c * 2 + (before ? 0 : 1)) * a.dim;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int at = col + (v * 64 + lane) * V;
                if (at >= a.dim) continue;
#pragma unroll
                for (int k = 0; k < V; ++k) p[at + k] = sum[v * V + k];
            }
            return;
        }
        E* p = (E*)a.table + run * a.table_stride;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int at = col + (v * 64 + lane) * V;
            if (at >= a.dim) continue;
            float x[V];
#pragma unroll
            for (int k = 0; k < V; ++k) x[k] = a.scale * sum[v * V + k];
            if constexpr (AL) *(uint4*)(p + at) = narrow(x, E{}); else p[at] = from_float<E>(x[0]);
        }
    };
    bool end = false;
    for (unsigned w = from; w < to && !end; w += 64) {
        const unsigned keys = a.key[min(w + lane, to - 1)], rows = a.row[min(w + lane, to - 1)];
        // places that count for nothing lie at the end
        const int here = __popcll(__ballot(w + lane < to && keys < (unsigned)a.vocab));
        end = here < 64;
        for (int j = 0; j < here; j += AHEAD) {
            uint4 g[AHEAD][NV];
            float one[AHEAD][NV];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const unsigned n = __builtin_amdgcn_readlane(rows, min(j + u, here - 1));
                const E* p = (const E*)a.out + n * a.out_stride;
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    const int at = min(col + (v * 64 + lane) * V, a.dim - V);
                    if constexpr (AL) g[u][v] = *(const uint4*)(p + at); else one[u][v] = to_float(p[at]);
                }
            }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                if (j + u >= here) break;
                const unsigned k = __builtin_amdgcn_readlane(keys, j + u);
                if (k != run) {
                    put(false);
                    run = k;
#pragma unroll
                    for (int i = 0; i < NV * V; ++i) sum[i] = 0.f;
                }
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    float x[V];
                    if constexpr (AL) widen(g[u][v], x, E{}); else x[0] = one[u][v];
#pragma unroll
                    for (int i = 0; i < V; ++i) sum[v * V + i] += x[i];
                }
            }
        }
    }
    put(true);
}
// Runs that cross a chunk's end: the workgroup of the chunk where one begins adds its parts, a wavefront a quarter of them.
template <typename E> __global__ void __launch_bounds__(256) embed_join_kernel(EmbedArgs a) {
    __shared__ float sums[4][256];
    const unsigned c = blockIdx.x, from = c * a.chunk, to = min(from + a.chunk, a.n);
    if (to >= a.n) return;
    const unsigned v = a.key[to - 1], next = a.key[to], first = a.key[from], previous = a.key[from > 0 ? from - 1 : 0];
    if (v >= (unsigned)a.vocab || next != v) return;
    if (first == v && from > 0 && previous == v) return;                        // begins before
    const unsigned lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const unsigned end = first_place(a, v + 1), last = (end - 1) / a.chunk, parts = last - c + 1;
    const unsigned each = (parts + 3) / 4, p0 = min(wave * each, parts), p1 = min(p0 + each, parts);
    const int col = blockIdx.y * 256 + lane * 4;
    float sum[4] = {};
#pragma unroll 4
    for (unsigned p = p0; p < p1; ++p) {
        const float* x = a.part + ((int64_t)(c + p) * 2 + (p == 0)) * a.dim;
#pragma unroll
        for (int k = 0; k < 4; ++k) sum[k] += col + k < a.dim ? x[col + k] : 0.f;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) sums[wave][lane * 4 + k] = sum[k];
    __syncthreads();
    const int at = blockIdx.y * 256 + threadIdx.x;
    if (at >= a.dim) return;
    const float s = ((sums[0][threadIdx.x] + sums[1][threadIdx.x]) + sums[2][threadIdx.x]) + sums[3][threadIdx.x];
    ((E*)a.table)[v * a.table_stride + at] = from_float<E>(a.scale * s);
}

// ---- host ----------------------------------------------------------------------------------------
bool embed_ok(const pql_embed_shape& s) {
    return s.batch >= 0 && s.steps >= 0 && s.per_row >= 1 && s.vocab >= 1 && s.vocab < 0x7fffffff && s.dim >= 1 && s.dim <= 1 << 24 &&
           (s.dtype == PQL_F32 || s.dtype == PQL_BF16) && s.scale - s.scale == 0.f &&
           (double)s.batch * s.steps * s.per_row < 2147483648.0;
}
unsigned embed_rows(const pql_embed_shape& s) { return (unsigned)((int64_t)s.batch * s.steps); }

struct EmbedPlan {
    unsigned n;
    int chunk, chunks, bits, passes, tiles;
    size_t key[2], row[2], count, total, part, bytes;
};
EmbedPlan embed_plan(const pql_embed_shape& s) {
    EmbedPlan p{};
    p.n = embed_rows(s) * (unsigned)s.per_row;
    // as many chunks as fill the card, then longer ones, which leave fewer parts to join (us for sums and joins: 4096 places of 1000 tokens
    // 10, with chunks of 256 42; 327680 of 1020 47, with chunks of 16 63, of 256 46)
    p.chunk = 16;
    while (p.chunk < 256 && p.n / p.chunk > 8192) p.chunk *= 2;
    p.chunks = (int)((p.n + (unsigned)p.chunk - 1) / p.chunk);
    size_t o = 0;
    auto take = [&](size_t b) { const size_t at = o; o += to256(b); return at; };
    p.key[0] = take((size_t)p.n * 4);
    p.row[0] = take((size_t)p.n * 4);
    if (p.n > RANK_MAX) {
        int need = 0;                                   // bits of the largest key, vocab itself
        while ((uint64_t)s.vocab >> need) ++need;
        p.passes = (need + DIGIT_BITS - 1) / DIGIT_BITS;
        p.bits = (need + p.passes - 1) / p.passes;
        p.tiles = (int)((p.n + TILE - 1u) / TILE);
        if (p.passes > 1) { p.key[1] = take((size_t)p.n * 4); p.row[1] = take((size_t)p.n * 4); }
        p.count = take((size_t)p.tiles << (p.bits + 2));
        p.total = take((size_t)4 << p.bits);
    }
    p.part = take((size_t)p.chunks * 2 * s.dim * 4);
    p.bytes = o;
    return p;
}
EmbedArgs embed_args(const pql_embed_shape& s, const int32_t* tokens, const int32_t* lengths, const pql_rows& table, const pql_rows& out) {
    EmbedArgs a{};
    a.tokens = tokens;
    a.live = {lengths, (unsigned)s.steps};
    a.rows = embed_rows(s);
    a.elem = elem_size(s.dtype);
    a.per_row = s.per_row; a.vocab = s.vocab; a.dim = s.dim; a.scale = s.scale;
    a.table = table.data; a.table_stride = table.stride;
    a.out = out.data; a.out_stride = out.stride;
    return a;
}
bool embed_aligned(const pql_embed_shape& s, const pql_rows& table, const pql_rows& out) {
    return s.dim * elem_size(s.dtype) % ROW_ALIGN == 0 && rows_aligned(table, s.dtype) && rows_aligned(out, s.dtype);
}
// A grid holds at most 2^32 - 1 threads.
constexpr unsigned MOST_BLOCKS = 1 << 22;
template <typename E, bool AL> hipError_t embed_launch(const EmbedArgs& a, hipStream_t st) {
    const int granules = AL ? a.dim / VEC_OF<E> : a.dim;
    int lanes = 1;
    while (lanes < 256 && lanes < granules) lanes *= 2;
    const unsigned by = 256 / lanes, blocks = (a.rows + by - 1) / by;
    const ProfSlot ps = prof_slot();
    PQL_LAUNCH(ps, (embed_kernel<E, AL>), dim3(blocks < MOST_BLOCKS ? blocks : MOST_BLOCKS), dim3(256), 0, st, a, lanes);
    prof_commit(ps, KID_EMBED, 0.0, (double)a.rows * (a.per_row * (4.0 + a.dim * sizeof(E)) + a.dim * sizeof(E)));
    return hipGetLastError();
}
hipError_t embed_sort(EmbedArgs& a, const EmbedPlan& p, char* ws, hipStream_t st) {
    // workgroups that clear the table: four 16-byte stores a lane, at most four workgroups a CU
    const double stores = (double)a.vocab * a.dim * a.elem / (4 * 16 * 256);
    const unsigned clear = stores < 1 ? 1 : stores < 1024 ? (unsigned)stores + 1 : 1024;
    unsigned* key[2] = {(unsigned*)(ws + p.key[0]), (unsigned*)(ws + p.key[1])};
    unsigned* row[2] = {(unsigned*)(ws + p.row[0]), (unsigned*)(ws + p.row[1])};
    if (p.n <= RANK_MAX) {
        a.key_to = key[0]; a.row_to = row[0];
        const ProfSlot ps = prof_slot();
        a.sort_blocks = (a.n * RANK_LANES + RANK_WG - 1) / RANK_WG;
        const dim3 grid(a.sort_blocks + clear);
        if (a.vocab < 1 << (32 - RANK_BITS)) PQL_LAUNCH(ps, embed_rank_kernel<true>, grid, dim3(RANK_WG), 0, st, a);
        else PQL_LAUNCH(ps, embed_rank_kernel<false>, grid, dim3(RANK_WG), 0, st, a);
        prof_commit(ps, KID_EMBED_SORT, 0.0, 12.0 * a.n);
    } else {
        a.count = (unsigned*)(ws + p.count); a.total = (unsigned*)(ws + p.total);
        a.bits = p.bits; a.tiles = p.tiles;
        a.sort_blocks = p.tiles;
        int to = (p.passes - 1) & 1;                    // the last pass ends in the first pair
        for (int i = 0; i < p.passes; ++i, to ^= 1) {
            a.shift = i * p.bits;
            a.key = key[to ^ 1]; a.row = row[to ^ 1]; a.key_to = key[to]; a.row_to = row[to];
            ProfSlot ps = prof_slot();
            if (i == 0) PQL_LAUNCH(ps, embed_count_kernel<true>, dim3(p.tiles + clear), dim3(SORT_WG), 0, st, a);
            else PQL_LAUNCH(ps, embed_count_kernel<false>, dim3(p.tiles), dim3(SORT_WG), 0, st, a);
            prof_commit(ps, KID_EMBED_SORT, 0.0, 4.0 * a.n);
            ps = prof_slot();
            PQL_LAUNCH(ps, embed_tiles_kernel, dim3(((1 << p.bits) + 63) / 64), dim3(1024), 0, st, a);
            prof_commit(ps, KID_EMBED_SORT, 0.0, 8.0 * p.tiles * (1 << p.bits));
            ps = prof_slot();
            if (i == 0) PQL_LAUNCH(ps, embed_move_kernel<true>, dim3(p.tiles), dim3(SORT_WG), 0, st, a);
            else PQL_LAUNCH(ps, embed_move_kernel<false>, dim3(p.tiles), dim3(SORT_WG), 0, st, a);
            prof_commit(ps, KID_EMBED_SORT, 0.0, 16.0 * a.n);
        }
    }
    a.key = key[0]; a.row = row[0];
    return hipGetLastError();
}
template <typename E, bool AL, int NV> void embed_sum_launch(const EmbedArgs& a, hipStream_t st) {
    constexpr int COLS = 64 * NV * (AL ? VEC_OF<E> : 1);
    const ProfSlot ps = prof_slot();
    PQL_LAUNCH(ps, (embed_sum_kernel<E, AL, NV>), dim3((a.chunks + 3) / 4, (a.dim + COLS - 1) / COLS), dim3(256), 0, st, a);
    prof_commit(ps, KID_EMBED_SUM, 0.0, (double)a.n * a.dim * sizeof(E));
}
template <typename E> hipError_t embed_back_launch(const EmbedArgs& a, bool aligned, hipStream_t st) {
    if (aligned) {
        if (a.dim <= 64 * VEC_OF<E>) embed_sum_launch<E, true, 1>(a, st);
        else embed_sum_launch<E, true, 2>(a, st);
    } else {
        if (a.dim <= 64) embed_sum_launch<E, false, 1>(a, st);
        else embed_sum_launch<E, false, 4>(a, st);
    }
    if (a.chunks > 1) {
        const ProfSlot ps = prof_slot();
        PQL_LAUNCH(ps, embed_join_kernel<E>, dim3(a.chunks, (a.dim + 255) / 256), dim3(256), 0, st, a);
        prof_commit(ps, KID_EMBED_JOIN, 0.0, 0.0);
    }
    return hipGetLastError();
}
int32_t embed_check(pql_ctx* c, const pql_embed_shape* s, const int32_t* tokens, const int32_t* lengths, const pql_rows* table,
                    const pql_rows* out, bool back) {
    if (!s || !table || !out) return ctx_fail(c, PQL_ERR_NULL, "pql_embed: null pointer");
    if (!embed_ok(*s)) return ctx_fail(c, PQL_ERR_INVALID_ARG, "pql_embed: bad shape");
    const int64_t rows = embed_rows(*s);
    const pql_rows& read = back ? *out : *table;
    const pql_rows& write = back ? *table : *out;
    if (!read_rows(read) || !own_rows(write, back ? s->vocab : rows, s->dim)) return ctx_fail(c, PQL_ERR_INVALID_ARG, "pql_embed: bad stride");
    if (rows == 0 && !back) return PQL_OK;
    if (!write.data || (rows > 0 && (!tokens || !read.data))) return ctx_fail(c, PQL_ERR_NULL, "pql_embed: null pointer");
    const size_t e = elem_size(s->dtype);
    if (off_by(tokens, 4) || off_by(lengths, 4) || off_by(table->data, e) || off_by(out->data, e))
        return ctx_fail(c, PQL_ERR_ALIGNMENT, "pql_embed: misaligned pointer");
    return PQL_OK;
}

}  // namespace
}  // namespace pql

using namespace pql;

extern "C" {

int32_t pql_embed_forward(pql_ctx* c, const pql_embed_shape* s, const int32_t* tokens, const int32_t* lengths, const pql_rows* table,
                          const pql_rows* out, void* stream) {
    if (!c) return PQL_ERR_NULL;
    const int32_t rc = embed_check(c, s, tokens, lengths, table, out, false);
    if (rc != PQL_OK || embed_rows(*s) == 0) return rc;
    const EmbedArgs a = embed_args(*s, tokens, lengths, *table, *out);
    const bool al = embed_aligned(*s, *table, *out);
    const hipStream_t st = (hipStream_t)stream;
    const hipError_t e = s->dtype == PQL_F32 ? (al ? embed_launch<float, true>(a, st) : embed_launch<float, false>(a, st))
                                             : (al ? embed_launch<bf16_t, true>(a, st) : embed_launch<bf16_t, false>(a, st));
    return e == hipSuccess ? PQL_OK : ctx_fail(c, PQL_ERR_HIP, "pql_embed_forward", e);
}

int64_t pql_embed_workspace_bytes(const pql_embed_shape* s) {
    if (!s) return PQL_ERR_NULL;
    if (!embed_ok(*s)) return PQL_ERR_INVALID_ARG;
    return (int64_t)embed_plan(*s).bytes;
}

int32_t pql_embed_backward(pql_ctx* c, const pql_embed_shape* s, const int32_t* tokens, const int32_t* lengths, const pql_rows* out_grad,
                           const pql_rows* table_grad, void* workspace, void* stream) {
    if (!c) return PQL_ERR_NULL;
    const int32_t rc = embed_check(c, s, tokens, lengths, table_grad, out_grad, true);
    if (rc != PQL_OK) return rc;
    const EmbedPlan p = embed_plan(*s);
    if (p.n > 0 && !workspace) return ctx_fail(c, PQL_ERR_NULL, "pql_embed_backward: null workspace");
    if (off_by(workspace, 256)) return ctx_fail(c, PQL_ERR_ALIGNMENT, "pql_embed_backward: misaligned workspace");
    EmbedArgs a = embed_args(*s, tokens, lengths, *table_grad, *out_grad);
    const hipStream_t st = (hipStream_t)stream;
    hipError_t e = hipSuccess;
    a.n = p.n;
    e = embed_sort(a, p, (char*)workspace, st);
    a.chunk = p.chunk; a.chunks = p.chunks;
    a.part = (float*)((char*)workspace + p.part);
    const bool al = embed_aligned(*s, *table_grad, *out_grad);
    if (e == hipSuccess && p.n > 0) e = s->dtype == PQL_F32 ? embed_back_launch<float>(a, al, st) : embed_back_launch<bf16_t>(a, al, st);
    return e == hipSuccess ? PQL_OK : ctx_fail(c, PQL_ERR_HIP, "pql_embed_backward", e);
}

}  // extern "C"
