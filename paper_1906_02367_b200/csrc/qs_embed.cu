// Embedding rows and their gradient.
//
//   forward    out[r, n, :] = scale * table[r][tok[r, n], :]
//   gradient   grad[r][v, :] = scale * sum over the places n with tok[r, n] = v of g[r, n, :]
//
// for R workers at once, each with its own table (a stretch of its row of the R x d batch) or a
// shared one.  Both are bound by memory: the forward pass by the rows it reads and writes, the
// gradient by g and by the whole table that it writes, most of it zeros.
//
// The gradient is formed without atomic additions.  The places are sorted by token (a stable radix
// sort, so equal tokens stay in the order of their places), the sorted list is cut into chunks of
// equal length whatever the lengths of the runs, and a warp sums a chunk's runs for 256 columns.  A
// run that crosses chunks (a frequent token's) leaves one partial sum per chunk, and these are
// joined in order.  The rows that no token names are known after the first look at the tokens (a byte
// per row); they are set to zero by blocks beside those that sum, so that reads and writes share the
// memory, and, as far as there is time, beside those that sort.  At 8 workers x 4096 tokens, tables of
// 32000 x 1024, bf16 in: 187 us, 6.0 TB/s of what has to be read and written; 65536 tokens, 128000 x
// 2048: 249 us, 5.3 TB/s.  Added to what is there (29 us' worth of bytes in the first case), nothing hides the sort and
// the joins: 88 us.
#include "qs_lm.cuh"

namespace {

using namespace qs;

constexpr int COLS = 256;                  // columns a warp handles at a time, 8 per lane

// columns of lane `lane` in a 256-column tile: WIDE, 16 bytes at a time (8 of a 2-byte type side by side, twice 4 of a
// 4-byte type); else 32 apart, so that a warp's single-element accesses lie side by side
template <int SIZE, bool WIDE>
__device__ __forceinline__ int col_of(int lane, int j) {
    if (!WIDE) return lane + 32 * j;
    return SIZE == 2 ? lane * 8 + j : (j >> 2) * 128 + lane * 4 + (j & 3);
}

__device__ __forceinline__ void widen(const uint4& q, float* f, __nv_bfloat16) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void widen(const uint4& q, float* f, __half) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
        f[2 * i] = p.x;
        f[2 * i + 1] = p.y;
    }
}

// ------------------------------------------------------------------ forward
struct EmbedArgs {
    long long N, V, D;
    Ids tok;
    const void* table;
    long long worker_stride, row_stride;   // of the table, in elements
    float scale;
    void* out;
    long long out_stride;
    int* status;
    long long rows;                        // R x N
    uint32_t units;                        // 256-column tiles per row
    int lanes;                             // log2 of the lanes that share a row (wide)
};

// where a place's row comes from; null: it names none
template <class TW>
__device__ __forceinline__ const TW* source_row(const EmbedArgs& a, long long row, long long t) {
    const long long r = a.rows == a.N ? 0 : row / a.N;
    return t >= 0 && t < a.V ? static_cast<const TW*>(a.table) + r * a.worker_stride + t * a.row_stride : nullptr;
}

template <class T> struct Eight {              // eight neighbours of a type
    uint4 q[sizeof(T) / 2];
};
template <class T> __device__ __forceinline__ void eight_to_float(const Eight<T>& e, float* f) { widen(e.q[0], f, T()); }
template <> __device__ __forceinline__ void eight_to_float<float>(const Eight<float>& e, float* f) {
    const uint32_t w[8] = {e.q[0].x, e.q[0].y, e.q[0].z, e.q[0].w, e.q[1].x, e.q[1].y, e.q[1].z, e.q[1].w};
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(w[i]);
}
__device__ __forceinline__ uint32_t two(float a, float b, __nv_bfloat16) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t two(float a, float b, __half) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <class T> __device__ __forceinline__ void store_eight(T* p, const float* f) {
    __stcs(reinterpret_cast<uint4*>(p), make_uint4(two(f[0], f[1], T()), two(f[2], f[3], T()), two(f[4], f[5], T()), two(f[6], f[7], T())));
}
template <> __device__ __forceinline__ void store_eight<float>(float* p, const float* f) {
    __stcs(reinterpret_cast<float4*>(p), make_float4(f[0], f[1], f[2], f[3]));
    __stcs(reinterpret_cast<float4*>(p) + 1, make_float4(f[4], f[5], f[6], f[7]));
}

constexpr int UNITS = 4;                       // 8-column units per lane in flight together

// Rows 16-byte aligned on both sides.  1 << a.lanes lanes share a row, so that a warp takes a long row or several short
// ones: one token and one address per lane, 64 (2-byte types) or 128 bytes of table in flight per lane.  8 x 4096 rows of 1024
// fp32 to bf16: 25 us; rows of any alignment, by the kernel after this one, 39
template <class TW, class TO>
__global__ void __launch_bounds__(256) embed_wide_kernel(const EmbedArgs a) {
    const int lane = (int)(threadIdx.x & ((1u << a.lanes) - 1u));
    const long long row = ((long long)blockIdx.x * 256 + threadIdx.x) >> a.lanes;
    if (row >= a.rows) return;
    const long long t = a.tok.at(row);
    const TW* src = source_row<TW>(a, row, t);
    TO* out = static_cast<TO*>(a.out) + row * a.out_stride;
    const float none = t < 0 ? 0.0f : quiet_nan();
    if (t >= a.V && lane == 0) flag_status(a.status, QS_INVALID_ARG);
    const int step = 8 << a.lanes, D = (int)a.D;
    for (int c0 = lane * 8; c0 < D; c0 += UNITS * step) {
        Eight<TW> e[UNITS];
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int c = c0 + i * step;
            if (!src || c + 8 > D) continue;
            const uint4* p = reinterpret_cast<const uint4*>(src + c);
#pragma unroll
            for (int w = 0; w < (int)sizeof(TW) / 2; ++w) e[i].q[w] = __ldg(p + w);
        }
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int c = c0 + i * step;
            if (c + 8 <= D) {
                float f[8];
                eight_to_float<TW>(e[i], f);
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = src ? f[j] * a.scale : none;
                store_eight<TO>(out + c, f);
            } else {
                for (int x = c; x < D; ++x) out[x] = from_float<TO>(src ? to_float(src[x]) * a.scale : none);
            }
        }
    }
}

// rows of any alignment: a warp per row and 256 columns
template <class TW, class TO>
__global__ void __launch_bounds__(256) embed_kernel(const EmbedArgs a) {
    const int lane = threadIdx.x & 31;
    const unsigned long long total = (unsigned long long)a.rows * a.units, id = (unsigned long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (id >= total) return;
    const long long row = (long long)(id / a.units), c0 = (long long)(id - (unsigned long long)row * a.units) * COLS, t = a.tok.at(row);
    const TW* src = source_row<TW>(a, row, t);
    const float none = t < 0 ? 0.0f : quiet_nan();
    if (t >= a.V && c0 == 0 && lane == 0) flag_status(a.status, QS_INVALID_ARG);
    TO* out = static_cast<TO*>(a.out) + row * a.out_stride;
    float f[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const long long c = c0 + lane + 32 * j;
        f[j] = c < a.D && src ? to_float(src[c]) * a.scale : none;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const long long c = c0 + lane + 32 * j;
        if (c < a.D) out[c] = from_float<TO>(f[j]);
    }
}

template <class TW, class TO>
cudaError_t launch_embed(EmbedArgs a, bool wide, cudaStream_t st) {
    if (wide) {
        while (a.lanes < 5 && (8ll << a.lanes) < a.D) ++a.lanes;
        return launch(false, embed_wide_kernel<TW, TO>, (unsigned)(((a.rows << a.lanes) + 255) / 256), 256, 0, st, a);
    }
    a.units = (uint32_t)((a.D + COLS - 1) / COLS);
    return launch(false, embed_kernel<TW, TO>, (unsigned)((a.rows * a.units + 7) / 8), 256, 0, st, a);
}

// ------------------------------------------------------------------ gradient: sort by token
// The kernels of one call follow one another without a gap: each is launched while the one before still runs, and waits
// here for its end before it reads or writes anything
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void next_may_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

constexpr int SORT_THREADS = 1024;
constexpr int SORT_MAX_BITS = 9;
constexpr int SORT_ITEMS = 8;              // places per thread and tile, as long as a worker's tiles are no more than
constexpr int MOST_TILES = 2048;           // (each tile reads the counts of all: 131072 of them for 2^30 tokens would be 30 TB)
constexpr int ONE_TILE = 1024;             // places per worker that one block sorts in its shared memory
constexpr int WARPS = SORT_THREADS / 32;

struct GradArgs {
    int R;
    long long N, V, D;
    Ids tok;
    const void* g;
    long long g_stride;
    float scale;
    int accumulate;
    float* grad;
    long long worker_stride, row_stride;
    int* status;
    // workspace
    uint32_t* key[2];                      // sorted tokens and their places, two of each for the passes
    uint32_t* pos[2];
    uint32_t* count[4];                    // per pass: R x tiles x bins
    uint8_t* named;                        // R x padded: 1 for a row that some token names
    long long padded;                      // V up to a multiple of 32
    uint32_t* turns;                       // pieces of the tables handed out
    uint32_t* joins;                       // [0] runs that cross chunks, then the chunk each of them starts in
    float* part;                           // R x chunks x 2 x padded D: partial sums of such runs
    int passes, bits, tiles, items, tile;  // bits per digit, tiles per worker, places per thread, places per tile
    int chunk, chunks;                     // places per chunk, chunks per worker
    int col_tiles;
    int side;                              // where the sorted list ends up
    int unit;                              // rows a warp sets to zero at a time
    int pieces;                            // or: rows side by side, in pieces (1), of whole 16-byte units (2)
};

__device__ __forceinline__ uint32_t key_of(const GradArgs& a, long long i) {
    const long long t = a.tok.at(i);
    if (t >= a.V) flag_status(a.status, QS_INVALID_ARG);
    return (uint32_t)(t < 0 || t >= a.V ? a.V : t);      // places that name no row sort behind all rows
}
// a byte per row: a plain store, which frequent tokens may repeat (an atomic on a bit made them wait in line: 22 us for
// 65536 tokens, 6 us this way)
__device__ __forceinline__ void mark_row(const GradArgs& a, int r, uint32_t k) {
    if (k < a.V) a.named[r * a.padded + k] = 1;
}

// `n` floats of zeros, a warp's work; dst on a 4-byte boundary
__device__ __forceinline__ void warp_zero(float* dst, long long n) {
    const int lane = threadIdx.x & 31;
    const long long head = min((long long)((16 - (reinterpret_cast<uintptr_t>(dst) & 15)) & 15) / 4, n), quads = (n - head) / 4;
    float4* p = reinterpret_cast<float4*>(dst + head);
#pragma unroll 4
    for (long long i = lane; i < quads; i += 32) __stcs(p + i, make_float4(0.0f, 0.0f, 0.0f, 0.0f));
    if (lane < head) dst[lane] = 0.0f;
    const long long tail = head + quads * 4;
    if (tail + lane < n) dst[tail + lane] = 0.0f;
}

// Rows that no token names become zero.  Rows side by side: the table is cut into 16-byte units, and pieces of 32 KB are
// handed out in order (`most` at most to a block), so that the writes go through memory in order and no block is left with
// more than its share: 7.2 TB/s, where a warp on 8 KB of its own writes 5.9.  Rows that are no whole units (EVEN false)
// have the units counted from the 16-byte boundary at or before the table, `lead` floats off; one that two rows share is
// written by elements unless both become zero, by a mask of its elements (16384 tokens, 50000 x 257: 33.0 us, 35.3 with a
// second look at the names of such units only; where such units are few that is the faster one: 8 x 4096 tokens,
// 32000 x 1024 at an odd place, 197 us against 208)
constexpr int PIECE = 2048;                // 16-byte units
template <int NT, bool EVEN>
__device__ void zero_pieces(const GradArgs& a, int most) {
    constexpr int U = PIECE / NT;
    __shared__ uint32_t turn;
    // places in a table: units, or floats
    constexpr uint32_t STEP = EVEN ? 1 : 4;
    const uint32_t D = (uint32_t)(EVEN ? a.D / 4 : a.D), all = (uint32_t)a.V * D;
    const uint32_t per = ((EVEN ? all : (all + 6) / 4) + PIECE - 1) / PIECE;
    const unsigned long long pieces = (unsigned long long)per * a.R;
    const uint32_t rows = STEP * NT / D, rest = STEP * NT - rows * D;
    uint32_t mine = threadIdx.x == 0 ? atomicAdd(a.turns, 1u) : 0u;
    for (int done = 1;; ++done) {
        if (threadIdx.x == 0) turn = mine;
        __syncthreads();
        const uint32_t piece = turn;
        __syncthreads();
        if (piece >= pieces) return;
        if (done < most && threadIdx.x == 0) mine = atomicAdd(a.turns, 1u);            // known by the time it is needed
        const uint32_t r = piece / per;
        const uint8_t* named = a.named + r * a.padded;
        float* table = a.grad + r * a.worker_stride;
        const uint32_t lead = EVEN ? 0u : (uint32_t)(reinterpret_cast<uintptr_t>(table) & 15u) / 4;
        const uint32_t first = ((piece - r * per) * PIECE + threadIdx.x) * STEP;
        float4* units = reinterpret_cast<float4*>(table - lead) + first / STEP;
        uint32_t zero[U];                              // a bit per element (EVEN: for the unit)
        if (EVEN || (first >= lead && first + STEP * NT * (U - 1) + 4 <= all + lead)) {
            uint32_t row = (first - lead) / D, in = first - lead - row * D;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (EVEN) zero[u] = first + u * NT < all && !named[row];
                else {
                    const uint32_t here = in + 3 < D ? 15u : (1u << (D - in)) - 1u;
                    const uint8_t one = named[row], other = named[here == 15u ? row : row + 1];        // (no branch between the loads)
                    zero[u] = (one ? 0u : here) | (other ? 0u : 15u ^ here);
                }
                row += rows;
                in += rest;
                if (in >= D) { in -= D; ++row; }
            }
        } else if constexpr (!EVEN) {                  // a table's first or last units are among the thread's
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t f = first + u * STEP * NT, off = f < lead ? lead - f : 0u;          // `off` elements lie before the table
                zero[u] = 0;
                if (f >= all + lead) continue;
                const uint32_t row = (f + off - lead) / D, end = off + D - (f + off - lead - row * D);
                const uint32_t there = f + 4 <= all + lead ? 15u : (1u << (all + lead - f)) - 1u, here = end < 4 ? (1u << end) - 1u : 15u;
                zero[u] = named[row] ? 0u : here & there;
                if ((there & ~here) && !named[row + 1]) zero[u] |= there & ~here;
                zero[u] &= 15u << off;
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (zero[u] == (EVEN ? 1u : 15u)) __stcs(units + u * NT, make_float4(0.0f, 0.0f, 0.0f, 0.0f));
            else if (!EVEN && zero[u]) {
                float* p = reinterpret_cast<float*>(units + u * NT);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (zero[u] >> e & 1u) p[e] = 0.0f;
            }
        }
        if (done == most) return;
    }
}

// Other tables, by `blocks` blocks of which this is number `block`: a warp takes `unit` rows at a time (a power of two up to
// 32, about 8 KB); neighbours without a name are one stretch where rows lie side by side
__device__ void zero_rows(const GradArgs& a, long long block, long long blocks) {
    const int unit = a.unit, lane = threadIdx.x & 31;
    const long long per = a.padded / unit, all = per * a.R, warps = blocks * (blockDim.x >> 5);
    const bool side_by_side = a.row_stride == a.D;
    for (long long i = block * (blockDim.x >> 5) + (threadIdx.x >> 5); i < all; i += warps) {
        const long long r = i / per, v0 = (i - r * per) * unit;
        uint32_t left = ~__ballot_sync(~0u, lane < unit && a.named[r * a.padded + v0 + lane]);
        const long long rows = min((long long)unit, a.V - v0);
        if (rows <= 0) continue;
        if (rows < 32) left &= (1u << rows) - 1u;
        float* base = a.grad + r * a.worker_stride + v0 * a.row_stride;
        while (left) {
            const int b = __ffs(left) - 1;
            const uint32_t up = ~(left >> b);              // zeros where the stretch goes on
            const int len = !side_by_side ? 1 : up ? __ffs(up) - 1 : 32;
            warp_zero(base + b * a.row_stride, len * a.D);
            left &= b + len >= 32 ? 0u : ~0u << (b + len);
        }
    }
}
template <int NT>
__device__ __forceinline__ void zero_all(const GradArgs& a, long long block, long long blocks) {
    if (a.pieces == 2) zero_pieces<NT, true>(a, 0x7fffffff);
    else if (a.pieces) zero_pieces<NT, false>(a, 0x7fffffff);
    else zero_rows(a, block, blocks);
}

constexpr int SEEN = 2048;

// counts of the first digit per tile; which rows are named
__global__ void __launch_bounds__(SORT_THREADS) sort_count_kernel(const GradArgs a) {
    __shared__ uint32_t hist[1 << SORT_MAX_BITS];
    __shared__ uint32_t seen[SEEN];                      // tokens the block has marked, by their low bits
    const int r = blockIdx.y, bins = 1 << a.bits;
    next_may_start();
    for (int b = threadIdx.x; b < bins; b += SORT_THREADS) hist[b] = 0;
    for (int b = threadIdx.x; b < SEEN; b += SORT_THREADS) seen[b] = 0;
    __syncthreads();
    for (int i = 0; i < a.items; ++i) {
        const long long n = (long long)blockIdx.x * a.tile + i * SORT_THREADS + threadIdx.x;
        if (n >= a.N) break;
        const uint32_t k = key_of(a, r * a.N + n);
        atomicAdd(&hist[k & (bins - 1)], 1u);
        if (!a.accumulate && atomicExch(&seen[k % SEEN], k + 1) != k + 1) mark_row(a, r, k);
    }
    __syncthreads();
    uint32_t* out = a.count[0] + ((long long)r * a.tiles + blockIdx.x) * bins;
    for (int b = threadIdx.x; b < bins; b += SORT_THREADS) out[b] = hist[b];
}

struct SortShared {
    uint16_t warp_count[WARPS << SORT_MAX_BITS];
    uint32_t base[1 << SORT_MAX_BITS], total[1 << SORT_MAX_BITS];
    uint32_t sums[WARPS];
};

// exclusive sums of v over the block's threads
__device__ uint32_t block_scan(uint32_t v, uint32_t* sums) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(~0u, x, o);
        if (lane >= o) x += y;
    }
    if (lane == 31) sums[warp] = x;
    __syncthreads();
    if (warp == 0) {
        uint32_t s = lane < WARPS ? sums[lane] : 0u;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t y = __shfl_up_sync(~0u, s, o);
            if (lane >= o) s += y;
        }
        if (lane < WARPS) sums[lane] = s;
    }
    __syncthreads();
    return x - v + (warp ? sums[warp - 1] : 0u);
}

// Rank of this thread's element among the block's elements of digit d (bins: none), in thread order, past what base
// says; base then moves on past the block's elements
__device__ uint32_t stable_place(SortShared& s, uint32_t d, int bins) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int b = threadIdx.x; b < WARPS * bins / 2; b += SORT_THREADS) reinterpret_cast<uint32_t*>(s.warp_count)[b] = 0;
    __syncthreads();
    const uint32_t same = __match_any_sync(0xffffffffu, d);
    const int rank = __popc(same & ((1u << lane) - 1u));
    if (d < (uint32_t)bins && rank == 0) s.warp_count[warp * bins + d] = (uint16_t)__popc(same);
    __syncthreads();
    for (int b = threadIdx.x; b < bins; b += SORT_THREADS) {
        uint32_t run = 0;
        for (int w = 0; w < WARPS; ++w) {
            const uint32_t v = s.warp_count[w * bins + b];
            s.warp_count[w * bins + b] = (uint16_t)run;
            run += v;
        }
        s.total[b] = run;
    }
    __syncthreads();
    const uint32_t to = d < (uint32_t)bins ? s.base[d] + s.warp_count[warp * bins + d] + rank : 0u;
    __syncthreads();
    for (int b = threadIdx.x; b < bins; b += SORT_THREADS) s.base[b] += s.total[b];
    return to;
}

// One pass of the sort: blocks [0, R x tiles) scatter a tile each, the others meanwhile set as many pieces to zero as the
// sorting, bound by latency, leaves time for (65536 tokens, 128000 rows of 2048: 251 us with 1 piece each, 248 with 4, 258
// with 16)
constexpr int BESIDE = 4;
__global__ void __launch_bounds__(SORT_THREADS, 2) sort_scatter_kernel(const GradArgs a, int pass) {
    __shared__ SortShared s;
    wait_for_previous();
    next_may_start();
    const int sorters = a.R * a.tiles;
    if ((int)blockIdx.x >= sorters) {
        if (a.pieces == 2) zero_pieces<SORT_THREADS, true>(a, BESIDE);
        else zero_pieces<SORT_THREADS, false>(a, BESIDE);
        return;
    }
    const int r = blockIdx.x / a.tiles, tile = blockIdx.x % a.tiles, bins = 1 << a.bits, shift = pass * a.bits;
    const uint32_t* count = a.count[pass] + (long long)r * a.tiles * bins;
    // places before this tile's elements of a digit: all smaller digits, and the same digit in earlier tiles
    uint32_t all = 0, before = 0;
    if ((int)threadIdx.x < bins) {
#pragma unroll 8
        for (int i = 0; i < a.tiles; ++i) {
            const uint32_t c = count[(long long)i * bins + threadIdx.x];
            all += c;
            before += i < tile ? c : 0u;
        }
    }
    const uint32_t smaller = block_scan(all, s.sums);
    if ((int)threadIdx.x < bins) s.base[threadIdx.x] = smaller + before;
    const uint32_t* key = a.key[pass & 1] + r * a.N;
    const uint32_t* pos = a.pos[pass & 1] + r * a.N;
    uint32_t* key_to = a.key[(pass + 1) & 1] + r * a.N;
    uint32_t* pos_to = a.pos[(pass + 1) & 1] + r * a.N;
    for (int i = 0; i < a.items; ++i) {
        const long long n = (long long)tile * a.tile + i * SORT_THREADS + threadIdx.x;
        const bool in = n < a.N;
        uint32_t k = 0, p = 0;
        if (in) {
            k = pass == 0 ? key_of(a, r * a.N + n) : key[n];
            p = pass == 0 ? (uint32_t)n : pos[n];
        }
        const uint32_t to = stable_place(s, in ? (k >> shift) & (bins - 1) : (uint32_t)bins, bins);
        if (!in) continue;
        key_to[to] = k;
        pos_to[to] = p;
        if (pass + 1 < a.passes)
            atomicAdd(a.count[pass + 1] + ((long long)r * a.tiles + to / a.tile) * bins + ((k >> (shift + a.bits)) & (bins - 1)), 1u);
    }
}

// A worker's whole sort in one block
__global__ void __launch_bounds__(SORT_THREADS) sort_one_tile_kernel(const GradArgs a) {
    __shared__ uint32_t key[ONE_TILE], pos[ONE_TILE];
    __shared__ SortShared s;
    const int r = blockIdx.x, bins = 1 << a.bits, i = threadIdx.x;
    const bool in = i < a.N;
    uint32_t k = 0, p = i;
    if (in) k = key_of(a, r * a.N + i);
    if (r == 0 && i == 0) a.joins[0] = a.turns[0] = 0;
    if (!a.accumulate) {
        uint32_t* marks = reinterpret_cast<uint32_t*>(a.named + r * a.padded);
        for (long long w = i; w < a.padded / 4; w += SORT_THREADS) marks[w] = 0;
        __syncthreads();
        if (in) mark_row(a, r, k);
    }
    next_may_start();
    for (int pass = 0; pass < a.passes; ++pass) {
        const uint32_t d = in ? (k >> (pass * a.bits)) & (bins - 1) : (uint32_t)bins;
        for (int b = i; b < bins; b += SORT_THREADS) s.total[b] = 0;
        __syncthreads();
        if (in) atomicAdd(&s.total[d], 1u);
        __syncthreads();
        const uint32_t base = block_scan(i < bins ? s.total[i] : 0u, s.sums);
        if (i < bins) s.base[i] = base;
        const uint32_t to = stable_place(s, d, bins);
        if (in) {
            key[to] = k;
            pos[to] = p;
        }
        __syncthreads();
        if (in) {
            k = key[i];
            p = pos[i];
        }
    }
    if (in) {
        a.key[a.side][r * a.N + i] = k;
        a.pos[a.side][r * a.N + i] = p;
    }
}
static_assert(ONE_TILE <= SORT_THREADS, "one place per thread");

// ------------------------------------------------------------------ gradient: sums of the runs
// A lane's 8 sums into the table's row.  IN: the sums' columns are those of 16-byte loads; OUT: rows 16-byte aligned.  Where
// only the first holds (a worker's table at an odd place of the batch), the sums change lanes through the warp's 256
// floats of shared memory, so that single-element stores lie side by side: 211 us for the 8 workers' tables above from a
// place that is odd (188 from an aligned one), 331 with single-element loads as well
template <bool IN, bool OUT, int SIZE>
__device__ __forceinline__ void write_sum(const GradArgs& a, float* dst, int c0, const float (&sum)[8], float* swap) {
    const int lane = threadIdx.x & 31;
    if (IN && OUT) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int c = c0 + col_of<SIZE, true>(lane, 4 * h);
            if (c + 4 <= a.D) {
                float4* p = reinterpret_cast<float4*>(dst + c);
                float4 v = make_float4(a.scale * sum[4 * h], a.scale * sum[4 * h + 1], a.scale * sum[4 * h + 2], a.scale * sum[4 * h + 3]);
                if (a.accumulate) {
                    const float4 o = *p;
                    v = make_float4(fmaf(a.scale, sum[4 * h], o.x), fmaf(a.scale, sum[4 * h + 1], o.y), fmaf(a.scale, sum[4 * h + 2], o.z),
                                    fmaf(a.scale, sum[4 * h + 3], o.w));
                }
                __stcs(p, v);
            } else {
#pragma unroll
                for (int j = 4 * h; j < 4 * h + 4; ++j) {
                    const int x = c0 + col_of<SIZE, true>(lane, j);
                    if (x < a.D) dst[x] = a.accumulate ? fmaf(a.scale, sum[j], dst[x]) : a.scale * sum[j];
                }
            }
        }
        return;
    }
    float x[8];
    if (IN) {
        __syncwarp();
#pragma unroll
        for (int h = 0; h < 2; ++h)
            *reinterpret_cast<float4*>(swap + col_of<SIZE, true>(lane, 4 * h)) = make_float4(sum[4 * h], sum[4 * h + 1], sum[4 * h + 2], sum[4 * h + 3]);
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = swap[lane + 32 * j];
        __syncwarp();
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = sum[j];
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int c = c0 + lane + 32 * j;
        if (c < a.D) dst[c] = a.accumulate ? fmaf(a.scale, x[j], dst[c]) : a.scale * x[j];
    }
}

// A warp's chunk of the sorted places and 256 columns of it
struct Chunk {
    long long ch, r, i0;                   // chunk, worker, first place
    int c0, n;                             // first column, places
    const uint32_t* key;
    const uint32_t* pos;
    uint32_t prev, next;                   // tokens beside the chunk
    bool there;

    __device__ __forceinline__ Chunk(const GradArgs& a, long long id) {
        there = id < (long long)a.R * a.chunks * a.col_tiles;
        if (!there) return;
        ch = id / a.col_tiles;
        c0 = (int)(id - ch * a.col_tiles) * COLS;
        r = ch / a.chunks;
        i0 = (ch - r * a.chunks) * a.chunk;
        n = (int)min((long long)a.chunk, a.N - i0);
        key = a.key[a.side] + r * a.N + i0;
        pos = a.pos[a.side] + r * a.N + i0;
        prev = i0 > 0 ? key[-1] : 0xffffffffu;
        next = i0 + n < a.N ? key[n] : 0xffffffffu;
    }
};

// the run being summed
template <bool IN, bool OUT, int SIZE>
struct Run {
    uint32_t cur;
    bool first;                            // of its chunk
    float sum[8];
    float* swap;                           // see write_sum

    __device__ __forceinline__ void start(uint32_t k) {
        cur = k;
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] = 0.0f;
    }
    // on: it goes on in the next chunk
    __device__ __forceinline__ void flush(const GradArgs& a, const Chunk& c, bool on) {
        if (cur >= (uint32_t)a.V) return;
        const int lane = threadIdx.x & 31;
        const bool from = first && cur == c.prev;
        if (!from && !on) {
            write_sum<IN, OUT, SIZE>(a, a.grad + c.r * a.worker_stride + (long long)cur * a.row_stride, c.c0, sum, swap);
        } else {                                   // part of a run that crosses chunks
            float4* p = reinterpret_cast<float4*>(a.part + (c.ch * 2 + (from ? 0 : 1)) * ((long long)a.col_tiles * COLS) + c.c0 + lane * 8);
            p[0] = make_float4(sum[0], sum[1], sum[2], sum[3]);
            p[1] = make_float4(sum[4], sum[5], sum[6], sum[7]);
            if (!from && c.c0 == 0 && lane == 0) a.joins[1 + atomicAdd(a.joins, 1u)] = (uint32_t)c.ch;
        }
    }
    __device__ __forceinline__ void meet(const GradArgs& a, const Chunk& c, uint32_t k) {
        if (k == cur) return;
        flush(a, c, false);
        first = false;
        start(k);
    }
};

// adds a lane's 8 columns of a row
__device__ __forceinline__ void add_pieces(const uint4* q, float (&sum)[8], float) {
    const uint32_t w[8] = {q[0].x, q[0].y, q[0].z, q[0].w, q[1].x, q[1].y, q[1].z, q[1].w};
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] += __uint_as_float(w[j]);
}
template <class T>
__device__ __forceinline__ void add_pieces(const uint4* q, float (&sum)[8], T type) {
    float x[8];
    widen(q[0], x, type);
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] += x[j];
}

// Wide rows: a warp per chunk and 256 columns, its rows on their way through a ring of its own in shared memory, 16 (or 8
// of fp32) ahead of the sums: each lane copies and reads its own 16 bytes, so that no barrier is needed
constexpr int RING_WARPS = 8, RING_BYTES = 8192;           // per warp

__device__ __forceinline__ void copy16(uint4* dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <class T, bool OUT>
__global__ void __launch_bounds__(RING_WARPS * 32, 3) run_sum_wide_kernel(const GradArgs a, unsigned sum_blocks) {
    constexpr int E = 16 / sizeof(T), PIECES = sizeof(T) / 2, DEPTH = RING_BYTES / (512 * PIECES);
    extern __shared__ __align__(16) uint4 ring_of_all[];
    __shared__ __align__(16) float swap[RING_WARPS][OUT ? 4 : COLS];
    wait_for_previous();
    next_may_start();
    if (blockIdx.x >= sum_blocks) {
        zero_all<RING_WARPS * 32>(a, blockIdx.x - sum_blocks, gridDim.x - sum_blocks);
        return;
    }
    const int lane = threadIdx.x & 31;
    uint4* ring = ring_of_all + (threadIdx.x >> 5) * (RING_BYTES / 16) + lane;         // slot s, piece h: ring[(s * PIECES + h) * 32]
    const Chunk c(a, (long long)blockIdx.x * RING_WARPS + (threadIdx.x >> 5));
    if (!c.there) return;
    const uint32_t none = 0xffffffffu, V = (uint32_t)a.V;
    const uint32_t k0 = lane < c.n ? c.key[lane] : none, k1 = lane + 32 < c.n ? c.key[lane + 32] : none;
    const uint32_t p0 = lane < c.n ? c.pos[lane] : 0u, p1 = lane + 32 < c.n ? c.pos[lane + 32] : 0u;
    const int n = __popc(__ballot_sync(~0u, k0 < V)) + __popc(__ballot_sync(~0u, k1 < V));     // places past these name no row
    if (n == 0) return;
    const T* g = static_cast<const T*>(a.g) + c.r * a.N * a.g_stride;
    int col[PIECES];
#pragma unroll
    for (int h = 0; h < PIECES; ++h) col[h] = c.c0 + col_of<sizeof(T), true>(lane, h * E);
    auto issue = [&](int i) {
        if (i < n) {
            const uint32_t at = __shfl_sync(~0u, i < 32 ? p0 : p1, i & 31);
            const T* row = g + (long long)at * a.g_stride;
            uint4* slot = ring + (i % DEPTH) * PIECES * 32;
#pragma unroll
            for (int h = 0; h < PIECES; ++h) {
                if (col[h] + E <= a.D) copy16(slot + h * 32, row + col[h]);
                else if (col[h] < a.D) {                   // the last columns
                    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
                    for (int j = 0; j < E; ++j) {
                        if (col[h] + j >= a.D) continue;
                        if (sizeof(T) == 4) w[j] = reinterpret_cast<const uint32_t*>(row)[col[h] + j];
                        else w[j / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(row)[col[h] + j] << (16 * (j & 1));
                    }
                    slot[h * 32] = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
        }
        copy_commit();
    };
#pragma unroll 1
    for (int i = 0; i < DEPTH; ++i) issue(i);
    Run<true, OUT, sizeof(T)> run;
    run.first = true;
    run.swap = swap[threadIdx.x >> 5];
    run.start(__shfl_sync(~0u, k0, 0));
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
        copy_wait<DEPTH - 1>();
        run.meet(a, c, __shfl_sync(~0u, i < 32 ? k0 : k1, i & 31));
        uint4 q[PIECES];
#pragma unroll
        for (int h = 0; h < PIECES; ++h) q[h] = ring[((i % DEPTH) * PIECES + h) * 32];
        add_pieces(q, run.sum, T());
        issue(i + DEPTH);
    }
    run.flush(a, c, n == c.n && run.cur == c.next);
}

// Rows of any alignment: the same with single-element loads, side by side across the warp.  Blocks past the chunks set rows
// to zero (one-tile sorts: nothing ran beside them)
constexpr int SUM_THREADS = 128;

template <class T>
__global__ void __launch_bounds__(SUM_THREADS, 5) run_sum_kernel(const GradArgs a, unsigned sum_blocks) {
    constexpr int AHEAD = 4;                       // rows in flight
    wait_for_previous();
    next_may_start();
    if (blockIdx.x >= sum_blocks) {
        zero_all<SUM_THREADS>(a, blockIdx.x - sum_blocks, gridDim.x - sum_blocks);
        return;
    }
    const int lane = threadIdx.x & 31;
    const Chunk c(a, (long long)blockIdx.x * (SUM_THREADS / 32) + (threadIdx.x >> 5));
    if (!c.there) return;
    const T* g = static_cast<const T*>(a.g) + c.r * a.N * a.g_stride + c.c0 + lane;
    const int cols = (int)min(a.D - c.c0 - lane, (long long)COLS);     // the lane's columns are 32 apart below it
    Run<false, false, sizeof(T)> run;
    run.first = true;
    run.swap = nullptr;
    run.start(c.key[0]);
    for (int i = 0; i < c.n; i += AHEAD) {
        float f[AHEAD][8];
        uint32_t k[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            k[u] = i + u < c.n ? c.key[i + u] : 0xffffffffu;
            const T* row = g + (long long)(k[u] < (uint32_t)a.V ? c.pos[i + u] : 0u) * a.g_stride;
#pragma unroll
            for (int j = 0; j < 8; ++j) f[u][j] = k[u] < (uint32_t)a.V && 32 * j < cols ? to_float(row[32 * j]) : 0.0f;
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if (i + u >= c.n) break;
            run.meet(a, c, k[u]);
#pragma unroll
            for (int j = 0; j < 8; ++j) run.sum[j] += f[u][j];
        }
        if (run.cur >= (uint32_t)a.V) return;      // only places that name no row are left
    }
    run.flush(a, c, run.cur == c.next);
}

// Runs that cross chunks: their partial sums are added in order.  A warp per run and 256 columns; a run of more than
// JOIN_ALONE chunks takes the whole block, each warp a stretch of it
constexpr int JOIN_ALONE = 12;

// adds partial sums [lo, hi) of the run that starts in chunk ch: the first chunk left its sum in slot 1, the others in 0
__device__ __forceinline__ void add_parts(const GradArgs& a, long long ch, int c0, long long lo, long long hi, float (&sum)[8]) {
    const long long width = (long long)a.col_tiles * COLS;
    const float* base = a.part + ch * 2 * width + c0 + (threadIdx.x & 31) * 8;
#pragma unroll 4
    for (long long i = lo; i < hi; ++i) {
        const float4* p = reinterpret_cast<const float4*>(base + (i * 2 + (i == 0)) * width);
        const float4 x = p[0], y = p[1];
        sum[0] += x.x; sum[1] += x.y; sum[2] += x.z; sum[3] += x.w;
        sum[4] += y.x; sum[5] += y.y; sum[6] += y.z; sum[7] += y.w;
    }
}

template <int SIZE, bool IN, bool OUT>
__global__ void __launch_bounds__(256) run_join_kernel(const GradArgs a) {
    __shared__ __align__(16) float sums[8][COLS];
    __shared__ long long length[8];                // chunks of the long runs met in this round
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    wait_for_previous();
    const long long all = (long long)a.joins[0] * a.col_tiles;
    // a run's column tiles follow one another: neighbours go to different blocks, so that a long run's do not queue up in one
    for (long long id0 = blockIdx.x; id0 < all; id0 += (long long)gridDim.x * 8) {
        const long long id = id0 + (long long)warp * gridDim.x;
        float sum[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] = 0.0f;
        long long n = 0;
        if (id < all) {
            const long long at = id / a.col_tiles, ch = a.joins[1 + at], r = ch / a.chunks, c = ch - r * a.chunks;
            const uint32_t* key = a.key[a.side] + r * a.N;
            const uint32_t cur = key[(c + 1) * a.chunk - 1];
            n = 1;
            for (;;) {                             // chunks the run goes on in
                const long long j = c + n + lane;
                const uint32_t same = __ballot_sync(~0u, j < a.chunks && key[j * a.chunk] == cur);
                n += same == ~0u ? 32 : __ffs(~same) - 1;
                if (same != ~0u) break;
            }
            if (n <= JOIN_ALONE) {
                const int c0 = (int)(id - at * a.col_tiles) * COLS;
                add_parts(a, ch, c0, 0, n, sum);
                write_sum<IN, OUT, SIZE>(a, a.grad + r * a.worker_stride + (long long)cur * a.row_stride, c0, sum, sums[warp]);
                n = 0;
            }
        }
        if (lane == 0) length[warp] = n;
        __syncthreads();
        for (int w = 0; w < 8; ++w) {
            const long long m = length[w];
            if (m == 0) continue;
            const long long of = id0 + (long long)w * gridDim.x, at = of / a.col_tiles, ch = a.joins[1 + at], r = ch / a.chunks, c = ch - r * a.chunks;
            const int c0 = (int)(of - at * a.col_tiles) * COLS;
            const long long per = (m + 7) / 8, lo = min(warp * per, m), hi = min(lo + per, m);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] = 0.0f;
            add_parts(a, ch, c0, lo, hi, sum);
#pragma unroll
            for (int j = 0; j < 8; ++j) sums[warp][lane + 32 * j] = sum[j];
            __syncthreads();
            if (warp == 0) {
                for (int x = 1; x < 8; ++x)
#pragma unroll
                    for (int j = 0; j < 8; ++j) sum[j] += sums[x][lane + 32 * j];
                const uint32_t cur = a.key[a.side][r * a.N + (c + 1) * a.chunk - 1];
                write_sum<IN, OUT, SIZE>(a, a.grad + r * a.worker_stride + (long long)cur * a.row_stride, c0, sum, sums[warp]);
            }
            __syncthreads();
        }
        __syncthreads();                           // `length` is written again
    }
}

// rows of zeros alone (no tokens)
__global__ void __launch_bounds__(256) zero_all_kernel(const GradArgs a) { zero_all<256>(a, blockIdx.x, gridDim.x); }

// IN, OUT: the rows of g, of the table on 16-byte boundaries
template <class T, bool IN, bool OUT>
cudaError_t launch_sums(const GradArgs& a, bool zero, int sms, cudaStream_t st) {
    const int warps = IN ? RING_WARPS : SUM_THREADS / 32;
    const unsigned blocks = (unsigned)(((long long)a.R * a.chunks * a.col_tiles + warps - 1) / warps);
    cudaError_t e;
    if (IN) {
        e = cudaFuncSetAttribute(run_sum_wide_kernel<T, OUT>, cudaFuncAttributeMaxDynamicSharedMemorySize, RING_WARPS * RING_BYTES);
        if (e == cudaSuccess) e = launch(true, run_sum_wide_kernel<T, OUT>, blocks + (zero ? sms * 3 : 0), RING_WARPS * 32, RING_WARPS * RING_BYTES, st, a, blocks);
    } else {
        e = launch(true, run_sum_kernel<T>, blocks + (zero ? sms * 8 : 0), SUM_THREADS, 0, st, a, blocks);
    }
    return e != cudaSuccess ? e : launch(true, run_join_kernel<sizeof(T), IN, OUT>, sms * 4, 256, 0, st, a);
}
template <class T>
cudaError_t launch_sums(const GradArgs& a, bool zero, bool in, bool out, int sms, cudaStream_t st) {
    if (in && out) return launch_sums<T, true, true>(a, zero, sms, st);
    if (in) return launch_sums<T, true, false>(a, zero, sms, st);
    return launch_sums<T, false, false>(a, zero, sms, st);
}

int bits_for(long long v) {
    int b = 1;
    while ((1ll << b) < v) ++b;
    return b;
}

// Sizes and the places of the workspace's parts, in 32-bit words
struct SortPlan {
    int passes, bits, tiles, items, chunk, chunks, col_tiles;
    bool one_tile;
    int64_t count, named, turns, joins, zeroed, part, words;    // first words; [count, zeroed) starts at zero
};
SortPlan sort_plan(int R, int64_t N, int64_t V, int64_t D) {
    SortPlan s;
    const int total = bits_for(V + 1);                   // keys 0 .. V
    s.passes = (total + SORT_MAX_BITS - 1) / SORT_MAX_BITS;
    s.bits = (total + s.passes - 1) / s.passes;
    s.one_tile = N <= ONE_TILE;
    s.items = 1;                                         // tiles of 1024 places while 64 of them cover the list: every block reads all tiles' counts
    while (N > 64ll * SORT_THREADS * s.items && (s.items < SORT_ITEMS || N > (long long)MOST_TILES * SORT_THREADS * s.items)) s.items *= 2;
    const int64_t tile = (int64_t)s.items * SORT_THREADS;
    s.tiles = (int)((N + tile - 1) / tile);
    s.col_tiles = (int)((D + COLS - 1) / COLS);
    // chunks as long as 64 places while they give every SM of a B200 some 16 warps (the size of the workspace asks no device)
    s.chunk = 8;
    while (s.chunk < 64 && R * N / (2 * s.chunk) * s.col_tiles >= 148 * 16) s.chunk *= 2;
    s.chunks = (int)((N + s.chunk - 1) / s.chunk);
    s.count = 4 * R * N;
    s.named = s.count + (s.one_tile ? 0 : (int64_t)s.passes * R * s.tiles << s.bits);
    s.turns = s.named + R * ((V + 31) / 32 * 32) / 4;
    s.joins = s.turns + 1;
    s.zeroed = s.joins + 1;
    s.part = (s.zeroed + (int64_t)R * s.chunks + 3) / 4 * 4;
    s.words = s.part + (int64_t)R * s.chunks * 2 * s.col_tiles * COLS;
    return s;
}

template <class TW>
cudaError_t launch_embed_to(const EmbedArgs& a, int out_type, cudaStream_t st) {
    const int out_size = out_type == QS_F32 ? 4 : 2, size = (int)sizeof(TW);
    // 16-byte accesses need every row on a 16-byte boundary
    const bool wide = aligned_to(a.table, 16) && a.row_stride * size % 16 == 0 && a.worker_stride * size % 16 == 0 && aligned_to(a.out, 16) &&
                      a.out_stride * out_size % 16 == 0;
    if (out_type == QS_F32) return launch_embed<TW, float>(a, wide, st);
    return out_type == QS_BF16 ? launch_embed<TW, __nv_bfloat16>(a, wide, st) : launch_embed<TW, __half>(a, wide, st);
}

bool bad_shape(int R, int64_t N, int64_t V, int64_t D) { return R < 1 || R > 32 || N < 0 || V < 1 || D < 1; }
bool too_large(int R, int64_t N, int64_t V, int64_t D) {
    // (the last: what a grid can count)
    return V > (1ll << 30) || N > (1ll << 30) / R || D > (1ll << 30) || R * N * ((D + 255) / 256) > (1ll << 33);
}

}  // namespace

extern "C" {

int qs_embed(int R, int64_t N, int64_t V, int64_t D, const void* tokens, int token_type, const void* table, int table_type,
             int64_t worker_stride, int64_t row_stride, float scale, void* out, int out_type, int64_t out_stride, int* status,
             void* cuda_stream) {
    if (bad_shape(R, N, V, D) || !is_id_type(token_type) || !size_of_type(table_type) || !size_of_type(out_type)) return QS_INVALID_ARG;
    if (too_large(R, N, V, D)) return QS_TOO_LARGE;
    if (worker_stride < 0 || row_stride < D || out_stride < D) return QS_INVALID_ARG;
    if (N == 0) return QS_OK;
    if (!tokens || !table || !out || !aligned_to(tokens, token_type == QS_I64 ? 8 : 4) || !aligned_to(table, size_of_type(table_type)) ||
        !aligned_to(out, size_of_type(out_type)) || !aligned_to(status, 4)) return QS_INVALID_ARG;
    EmbedArgs a{N, V, D, Ids{tokens, token_type == QS_I64}, table, worker_stride, row_stride, scale, out, out_stride, status, R * N, 0, 0};
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    return status_of(table_type == QS_F32 ? launch_embed_to<float>(a, out_type, st) : table_type == QS_BF16 ? launch_embed_to<__nv_bfloat16>(a, out_type, st)
                                                                                                            : launch_embed_to<__half>(a, out_type, st));
}

int64_t qs_embed_grad_bytes(int R, int64_t N, int64_t V, int64_t D) {
    if (bad_shape(R, N, V, D)) return QS_INVALID_ARG;
    if (too_large(R, N, V, D)) return QS_TOO_LARGE;
    return 4 * sort_plan(R, N, V, D).words;
}

int qs_embed_grad(int R, int64_t N, int64_t V, int64_t D, const void* tokens, int token_type, const void* grad_out, int grad_type,
                  int64_t grad_stride, float scale, int accumulate, float* grad_table, int64_t worker_stride, int64_t row_stride,
                  void* work, int64_t work_bytes, int* status, void* cuda_stream) {
    if (bad_shape(R, N, V, D) || !is_id_type(token_type) || !size_of_type(grad_type)) return QS_INVALID_ARG;
    if (too_large(R, N, V, D)) return QS_TOO_LARGE;
    // the workers' tables must not overlap: one after the other, or row by row
    if (grad_stride < D || row_stride < D || (R > 1 && worker_stride < (V - 1) * row_stride + D &&
                                              (worker_stride < D || row_stride < (R - 1) * worker_stride + D))) return QS_INVALID_ARG;
    if (!grad_table || !aligned_to(grad_table, 4) || !aligned_to(status, 4)) return QS_INVALID_ARG;
    const SortPlan p = sort_plan(R, N, V, D);
    if (!work || !aligned_to(work, 16)) return QS_INVALID_ARG;
    if (N > 0 && (!tokens || !grad_out || !aligned_to(tokens, token_type == QS_I64 ? 8 : 4) || !aligned_to(grad_out, size_of_type(grad_type))))
        return QS_INVALID_ARG;
    if (work_bytes < 4 * p.words) return QS_CAPACITY;
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
        cudaGetLastError();
        return QS_CUDA;
    }
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    uint32_t* w = static_cast<uint32_t*>(work);
    const int64_t m = R * N;
    GradArgs a{};
    a.R = R; a.N = N; a.V = V; a.D = D; a.tok = Ids{tokens, token_type == QS_I64};
    a.g = grad_out; a.g_stride = grad_stride; a.scale = scale; a.accumulate = accumulate; a.grad = grad_table;
    a.worker_stride = worker_stride; a.row_stride = row_stride; a.status = status;
    a.key[0] = w; a.key[1] = w + m; a.pos[0] = w + 2 * m; a.pos[1] = w + 3 * m;
    for (int i = 0; i < p.passes; ++i) a.count[i] = w + p.count + ((int64_t)i * R * p.tiles << p.bits);
    a.named = reinterpret_cast<uint8_t*>(w + p.named); a.padded = (V + 31) / 32 * 32; a.turns = w + p.turns; a.joins = w + p.joins; a.part = reinterpret_cast<float*>(w + p.part);
    a.passes = p.passes; a.bits = p.bits; a.tiles = p.tiles; a.items = p.items; a.tile = p.items * SORT_THREADS;
    a.chunk = p.chunk; a.chunks = p.chunks; a.col_tiles = p.col_tiles; a.side = p.passes & 1;
    a.unit = 32;
    while (a.unit > 1 && a.unit * D > 2048) a.unit /= 2;
    // (counters of 32 bits, with a piece to spare)
    a.pieces = row_stride == D && D >= 4 && V * D < (1ll << 32) - (1ll << 16);
    if (a.pieces && aligned_to(grad_table, 16) && D % 4 == 0 && worker_stride % 4 == 0) a.pieces = 2;
    // (without whole units, where there is no longer sort to be beside, the pieces' start costs more than their order gains in
    // small tables.  509 tokens, fp32, rows of 1025, us in pieces and by rows: 32 MB 20.6, 18.5; 128 MB 35.1, 34.7; 192 MB 45.1,
    // 46.7; 800 MB 139, 169.  Of 257 columns: 128 MB 38.3, 37.1; 256 MB 60.1, 59.9; 800 MB 155, 165)
    else if (a.pieces && p.one_tile && R * V * D < 1ll << 25) a.pieces = 0;
    if (N == 0 && accumulate) return QS_OK;
    // (the one-tile sort sets its own marks to zero)
    cudaError_t e = cudaSuccess;
    if (N == 0 || !p.one_tile) e = cudaMemsetAsync(w + p.count, 0, 4 * (p.zeroed - p.count), st);
    if (N == 0) return status_of(e != cudaSuccess ? e : launch(false, zero_all_kernel, sms * 8, 256, 0, st, a));
    if (p.one_tile) {
        e = launch(false, sort_one_tile_kernel, R, SORT_THREADS, 0, st, a);
    } else {
        if (e == cudaSuccess) e = launch(false, sort_count_kernel, dim3(p.tiles, R), SORT_THREADS, 0, st, a);
        const int sorters = R * p.tiles, beside = accumulate || !a.pieces || sorters > 2 * sms ? 0 : 2 * sms - sorters;
        for (int pass = 0; pass < p.passes && e == cudaSuccess; ++pass)
            e = launch(true, sort_scatter_kernel, (unsigned)(sorters + beside), SORT_THREADS, 0, st, a, pass);
    }
    if (e != cudaSuccess) return status_of(e);
    const int size = size_of_type(grad_type);
    const bool in = aligned_to(grad_out, 16) && grad_stride * size % 16 == 0;
    const bool out = aligned_to(grad_table, 16) && row_stride % 4 == 0 && worker_stride % 4 == 0;
    return status_of(grad_type == QS_F32 ? launch_sums<float>(a, !accumulate, in, out, sms, st)
                     : grad_type == QS_BF16 ? launch_sums<__nv_bfloat16>(a, !accumulate, in, out, sms, st) : launch_sums<__half>(a, !accumulate, in, out, sms, st));
}

}  // extern "C"
