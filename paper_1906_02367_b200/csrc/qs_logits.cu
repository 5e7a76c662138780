// Rows of logits: log probabilities of given tokens with the entropy and the top alternatives, and
// distillation from a teacher's top logits, with their gradients.
//
// With y = scale * z over a row of V logits, m = max y, s = sum exp(y - m), lse = m + log s and
// p = exp(y - lse):
//   logp     = y_t - lse,   entropy = log s - sum p (y - m),   alternatives: the K largest z
//   d/dz_v   = scale [ g (1[v = t] - p_v) - h p_v (log p_v + entropy) ]
//   distill  = sum_k q_k (log q_k - log p_k) (+ q_T (log q_T - log p_T) for the mass outside the ids)
//   d/dz_v   = weight scale [ p_v (Q + q_T - (q_T / p_T outside the ids)) - q_v ]
// A column at -inf has p = 0 and adds nothing; a row without any other column has lse = -inf.
//
// All of these are bound by the memory that holds the logits: each must read the row, and the gradients write
// one.  So a row is read once.  Statistics and alternatives are taken as the vectors come by, with plain loads of
// many resident warps (48 an SM of 40 registers, 40 of 48 with alternatives; the same loop behind a ring of bulk copies and
// 24 warps took 480 us where this took 363).  The loss that also gives its gradient keeps the row in the shared memory of a
// cluster's blocks, one bulk copy each, until the statistics are joined.  The backward calls, which start from a saved
// lse, are one pass per vector.  bf16 rows of 128000: statistics alone 389 us for 8192 rows (5.4 TB/s), the loss and its
// gradient 692 us for 6144 (4.5 TB/s; a block reads, computes and writes in turn, and only other blocks fill the gaps);
// 64 alternatives, 4096 rows of 50003: 133 us (3.1 TB/s; finding and ranking them takes as long as reading).
#include <algorithm>
#include <cstdlib>

#include "qs_rows.cuh"

namespace {

using namespace qs;

constexpr int MAX_BLOCKS = 8;              // blocks of a row's cluster
constexpr int MAX_THREADS = 256;
constexpr int MAX_WARPS = MAX_THREADS / 32;
constexpr int PARTS = MAX_BLOCKS * MAX_WARPS;
constexpr int VPT = 4;                     // vectors per thread and batch
constexpr int VK = 8;                      // the same where the row is kept: 128 threads and 8 vectors take a tenth less than 256 and 4
constexpr int SLOTS = 16;                  // stretches of a thread's share whose largest elements are kept apart
constexpr int PAIRS = 512;                 // such stretches that are looked through again
constexpr int MOST = QS_MAX_TOP + QS_MAX_TOP / 4 + 16;      // candidates ranked against one another
constexpr int CANDS = 1024;                // candidates a block keeps, and a row's blocks send in all (>= MAX_BLOCKS QS_MAX_TOP)

struct RowArgs {
    long long N, V, row0;
    const void* logits;
    long long stride;
    float scale;
    Ids tok;                       // given tokens (N) or the teacher's ids (N x K)
    int K;                         // alternatives, or ids per row
    float* logp; float* lse; float* entropy;
    void* top_ids; float* top_logp;
    const void* teacher; int teacher_type;
    float teacher_scale;
    float* loss; float* log_tail;
    // gradients
    const float* in_lse; const float* in_entropy; const float* in_log_tail;
    const float* g1; const float* g2;      // of logp and of the entropy; g1: of the loss
    float g_all;                           // where g1 is null
    void* grad; long long grad_stride;
    int wide;                              // the gradient's rows lie like the logits' rows within 16 bytes
    int parts;                             // log2 of the blocks per row
    int per;                               // batches per stretch whose maximum is kept
    int rows;                              // backward calls: which rows this launch is for
    unsigned long long wait_ns;            // limit of a wait
    int* status;
};

// ------------------------------------------------------------------ log probabilities
// Places that a cut takes: key above the cut's, or equal to it with a column at or below the cut's
struct Cut { uint32_t key, idx; };
__device__ __forceinline__ bool takes(Cut c, uint32_t key, uint32_t idx) { return key > c.key || (key == c.key && idx <= c.idx); }

__device__ __forceinline__ bool takes(Cut c, unsigned long long e) { return takes(c, (uint32_t)(e >> 32), ~(uint32_t)e); }

// a sum over the block's threads
__device__ __forceinline__ int block_count(int mine, int* sums) {
    const int w = __reduce_add_sync(~0u, mine), warps = blockDim.x >> 5;
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = w;
    __syncthreads();
    int total = 0;
    for (int i = 0; i < warps; ++i) total += sums[i];
    return total;
}

// A cut that takes between K and `most` places, by bisection over the keys in [lo, hi) and then, where equal keys alone
// are more than that, over the columns.  `count(cut)` is the number of places a cut takes, the same in all threads;
// Cut{lo, ~0} takes more than `most`, Cut{hi, ~0} none
template <class Count>
__device__ __forceinline__ Cut find_cut(int K, int most, uint32_t lo, uint32_t hi, uint32_t columns, Count count) {
    while (hi - lo > 1) {
        const uint32_t mid = lo + (hi - lo) / 2;
        const int c = count(Cut{mid, 0xffffffffu});
        if (c >= K) {
            lo = mid;
            if (c <= most) return Cut{mid, 0xffffffffu};
        } else {
            hi = mid;
        }
    }
    uint32_t a = 0, b = columns - 1;               // the smallest column that makes it K, or an earlier stop
    while (a < b) {
        const uint32_t mid = a + (b - a) / 2;
        const int c = count(Cut{lo, mid});
        if (c >= K) {
            if (c <= most) return Cut{lo, mid};
            b = mid;
        } else {
            a = mid + 1;
        }
    }
    return Cut{lo, b};
}

struct TopShared {
    unsigned long long list[CANDS];        // candidates (key, ~column) of the block's share, then of the cluster's
    int count[MAX_BLOCKS];
    unsigned long long last[MOST];         // what is left of the list for the ranking
    int n, left, sums[MAX_WARPS];          // candidates in the list; entries in `last`
    int pairs;                             // (slot, thread) pairs whose largest element reaches the bound
    uint16_t pair[PAIRS];
    uint32_t low[MAX_WARPS], high[MAX_WARPS];
};

// smallest and largest key of the block's threads
__device__ __forceinline__ uint2 block_range(uint32_t low, uint32_t high, TopShared& t) {
    const uint32_t a = __reduce_min_sync(~0u, low), b = __reduce_max_sync(~0u, high);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) {
        t.low[threadIdx.x >> 5] = a;
        t.high[threadIdx.x >> 5] = b;
    }
    __syncthreads();
    uint2 r = make_uint2(t.low[0], t.high[0]);
    for (int i = 1; i < (int)(blockDim.x >> 5); ++i) r = make_uint2(min(r.x, t.low[i]), max(r.y, t.high[i]));
    return r;
}

// The largest key found that at least K of the threads' maxima reach (a few more may), 0 if fewer are above -inf
__device__ uint32_t maxima_bound(uint32_t mine, int K, TopShared& t) {
    const int live = __syncthreads_count(mine >= KEY_LOWEST);
    if (live < K) return 0;
    const uint2 range = block_range(mine >= KEY_LOWEST ? mine : 0xffffffffu, mine, t);
    uint32_t lo = range.x, hi = range.y + 1;
    while (hi - lo > 1) {
        const uint32_t mid = lo + (hi - lo) / 2;
        const int c = __syncthreads_count(mine >= mid);
        if (c >= K) {
            lo = mid;
            if (c <= K + K / 8 + 1) break;
        } else {
            hi = mid;
        }
    }
    return lo;
}

// Between K and `most` (<= MOST) of the list's n entries, the largest, into `last`; all if there are no more than that
__device__ void shrink_list(TopShared& t, int n, int K, int most, uint32_t columns) {
    const int nt = blockDim.x;
    Cut cut{0, 0xffffffffu};
    if (n > most) {
        uint32_t low = 0xffffffffu, high = 0;
        for (int i = threadIdx.x; i < n; i += nt) {
            low = min(low, (uint32_t)(t.list[i] >> 32));
            high = max(high, (uint32_t)(t.list[i] >> 32));
        }
        const uint2 range = block_range(low, high, t);
        cut = find_cut(K, most, range.x, range.y + 1, columns, [&](Cut c) {
            int k = 0;
            for (int i = threadIdx.x; i - (int)threadIdx.x < n; i += nt) k += __syncthreads_count(i < n && takes(c, t.list[i]));
            return k;
        });
    }
    __syncthreads();
    if (threadIdx.x == 0) t.left = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += nt)
        if (takes(cut, t.list[i])) t.last[atomicAdd(&t.left, 1)] = t.list[i];
    __syncthreads();
}

// calls f(z, column) for the elements of a vector that reach `bound`
template <class T, class F>
__device__ __forceinline__ void each_above(const uint4& q, int e0, float bound, F f) {
    if (!(Vec<T>::top(max_of_words<T>(q)) >= bound)) return;
#pragma unroll
    for (int i = 0; i < Vec<T>::E / 2; ++i) {
        const float2 p = parts(Vec<T>::pair(q, i));
        if (p.x >= bound) f(p.x, (uint32_t)(e0 + 2 * i));
        if (p.y >= bound) f(p.y, (uint32_t)(e0 + 2 * i + 1));
    }
}
// the same for the vectors [v0, v1) of a row, read anew
template <class T, class F>
__device__ __forceinline__ void each_of_row(const Share<T>& r, int v0, int v1, float bound, F f) {
    for (int vec = v0 + (int)threadIdx.x; vec < v1; vec += blockDim.x)
        each_above<T>(vec >= r.w0 && vec < r.w1 ? r.vectors()[vec] : r.edge(vec), r.first(vec), bound, f);
}

__device__ __forceinline__ unsigned long long entry_of(float z, uint32_t col) { return ((unsigned long long)key_of(z) << 32) | (uint32_t)~col; }

__device__ __forceinline__ void put_candidate(TopShared& t, float z, uint32_t col) {
    const int at = atomicAdd(&t.n, 1);
    if (at < CANDS) t.list[at] = entry_of(z, col);
}

// The elements of the share that reach the bound, from the stretches whose largest does; false (and no list) if there are
// too many.  All threads
template <class T>
__device__ bool collect(TopShared& t, const Share<T>& r, const float* slot_max, int slots, int per, float bound) {
    const int nt = blockDim.x;
    __syncthreads();
    if (threadIdx.x == 0) t.n = t.pairs = 0;
    __syncthreads();
    for (int i = 0; i < slots; ++i)
        if (slot_max[i * nt + threadIdx.x] >= bound) {
            const int at = atomicAdd(&t.pairs, 1);
            if (at < PAIRS) t.pair[at] = (uint16_t)(i * nt + threadIdx.x);
        }
    __syncthreads();
    if (t.pairs > PAIRS) return false;
    auto put = [&](float z, uint32_t col) { put_candidate(t, z, col); };
    const int each = per * VPT, all = t.pairs * each;
    for (int i = threadIdx.x; i < all; i += nt) {
        const int pair = t.pair[i / each], vec = r.w0 + (pair / nt * each + i % each) * nt + pair % nt;
        if (vec < r.w1) each_above<T>(r.vectors()[vec], r.first(vec), bound, put);
    }
    if (threadIdx.x == 0 && r.w0 > r.v0) each_above<T>(r.edge(r.v0), r.first(r.v0), bound, put);
    if ((int)threadIdx.x == nt - 1 && r.w1 < r.v1) each_above<T>(r.edge(r.w1), r.first(r.w1), bound, put);
    __syncthreads();
    return t.n <= CANDS;
}

// Too many elements reach the bound: equal ones, as a rule (a mask of the lowest value).  What lies above it, and of the
// equal ones the first that make it K, stretch of columns by stretch; an order that defeats the bound itself
// is cut exactly, reading the row once per step of a bisection
template <class T>
__device__ __noinline__ void collect_hard(TopShared& t, const Share<T>& r, const float* slot_max, int slots, int per, int K, uint32_t bound) {
    const int nt = blockDim.x;
    if (!collect<T>(t, r, slot_max, slots, per, value_of(bound + 1))) {
        const Cut cut = find_cut(K, CANDS / 2, bound - 1, 0xff800001u, (uint32_t)r.V, [&](Cut c) {
            int k = 0;
            each_of_row<T>(r, r.v0, r.v1, value_of(bound), [&](float z, uint32_t col) { k += takes(c, key_of(z), col); });
            return block_count(k, t.sums);
        });
        __syncthreads();
        if (threadIdx.x == 0) t.n = 0;
        __syncthreads();
        each_of_row<T>(r, r.v0, r.v1, value_of(bound), [&](float z, uint32_t col) {
            if (takes(cut, key_of(z), col)) put_candidate(t, z, col);
        });
        __syncthreads();
        return;
    }
    const float tie = value_of(bound);
    int have = t.n;
    for (int v0 = r.v0; v0 < r.v1 && have < K; v0 += nt * VPT) {
        const int v1 = min(v0 + nt * VPT, r.v1);
        auto count = [&](uint32_t col_most) {
            int k = 0;
            each_of_row<T>(r, v0, v1, tie, [&](float z, uint32_t col) { k += key_of(z) == bound && col <= col_most; });
            return block_count(k, t.sums);
        };
        uint32_t to = 0xffffffffu;
        if (count(to) > CANDS - have) {            // a column that leaves enough of them, and few enough
            uint32_t a = (uint32_t)max(r.first(v0), 0), b = (uint32_t)r.first(v1);
            while (a < b) {
                const uint32_t mid = a + (b - a) / 2;
                const int c = count(mid);
                if (c >= K - have) {
                    b = mid;
                    if (c <= CANDS - have) break;
                } else {
                    a = mid + 1;
                }
            }
            to = b;
        }
        __syncthreads();
        each_of_row<T>(r, v0, v1, tie, [&](float z, uint32_t col) {
            if (key_of(z) == bound && col <= to) put_candidate(t, z, col);
        });
        __syncthreads();
        have = t.n;
        __syncthreads();
    }
}

// Statistics of the row, and with TOP its alternatives.  While the row comes by, each thread keeps the largest element of
// each of up to 16 stretches of its share; the K-th largest of the threads' maxima is a bound below which no alternative
// can lie, and the few stretches that reach it (about K) are read again, from the L2.
template <class T, bool TOP>
__global__ void __launch_bounds__(MAX_THREADS, TOP ? 5 : 6) token_logp_kernel(const RowArgs a) {
    __shared__ float4 part[PARTS];
    __shared__ float row_m, row_ls, row_lse;
    __shared__ TopShared top[1];                   // (no room where it is not used)
    // TOP: the stretches' maxima (slots x threads), and what a cluster's blocks have left, block b's at b * CANDS / blocks
    extern __shared__ unsigned long long merged[];
    const int nt = blockDim.x, warps = nt >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, blocks = 1 << a.parts;
    const int rank = blocks == 1 ? 0 : (int)cluster_rank();
    const long long n = a.row0 + (blockIdx.x >> a.parts);
    const float c2 = a.scale * LOG2E;
    if (blocks > 1) cluster_arrive();              // the blocks have started: their shared memory may be written
    const Share<T> r(a.logits, a.stride, n, a.V, rank, a.parts);
    Stat st{neg_inf(), 0.0f, 0.0f};
    float mine = neg_inf();                        // the thread's largest
    float* slot_max = reinterpret_cast<float*>(merged + (blocks > 1 ? CANDS : 0)) + threadIdx.x;
    float stretch = neg_inf();
    int batch = 0, slot = 0;
    each_batch<T, VPT, TOP>(r, [&](auto& q, int vec, auto more) {
        constexpr int P = sizeof(q) / sizeof(uint4);
        const float m = thread_max_of<T, P>(q);
        take<T, P, true, decltype(more)::value>(st, q, m, c2);
        mine = fmaxf(mine, m);
        if (TOP) {
            if (vec < r.w0 || vec >= r.w1) return; // (vectors that are not whole are looked through in any case)
            stretch = fmaxf(stretch, m);
            slot_max[slot * nt] = stretch;
            if (++batch == a.per) {
                batch = 0;
                ++slot;
                stretch = neg_inf();
            }
        }
    });
    if (TOP) {
        if (batch == 0) slot_max[slot * nt] = neg_inf();       // (a thread without a vector in the last batch)
        const int slots = (r.w1 - r.w0 + nt * VPT * a.per - 1) / (nt * VPT * a.per);
        const uint32_t key = max(maxima_bound(key_of(mine), a.K, *top), KEY_LOWEST);
        if (!collect<T>(*top, r, slot_max - threadIdx.x, slots, a.per, value_of(key)))
            collect_hard<T>(*top, r, slot_max - threadIdx.x, slots, a.per, a.K, key);
    }
    long long t = -1;
    float zt = 0.0f;
    if (rank == 0 && (int)threadIdx.x == nt - 1 && a.logp) {
        t = a.tok.at(n);
        if (t >= a.V) flag_status(a.status, QS_INVALID_ARG);
        else if (t >= 0) zt = to_float(r.z[t]);
    }
    const int most = min(max(a.K + a.K / 4 + 16, 96), nt);       // candidates that are ranked, a thread or more each
    const Stat w = join_warp<true>(st, mine, c2);
    const float4 sent = make_float4(w.m, w.s, w.u, 0.0f);
    if (blocks == 1) {
        if (lane == 0) part[warp] = sent;
        __syncthreads();
    } else {
        cluster_wait();
        if (TOP) {
            shrink_list(*top, top->n, a.K, min(most, CANDS / blocks), (uint32_t)a.V);
            for (int i = threadIdx.x; i < top->left; i += nt) remote_store(remote_addr(&merged[rank * (CANDS / blocks) + i], 0), top->last[i]);
            if (threadIdx.x == 0) remote_store(remote_addr(&top->count[rank], 0), (uint32_t)top->left);
        }
        if (lane == 0) remote_store(remote_addr(&part[rank * warps + warp], 0), sent);
        cluster_arrive();
        if (rank != 0) return;                     // nothing is written into this block's memory
        cluster_wait();
    }
    if (warp == warps - 1) {
        const Stat v = final_stat(join_parts(part, warps * blocks, c2), c2);
        const bool empty = is_empty(v);
        const float ls = logf(v.s), lse = lse_of(v, a.scale, ls);
        if (lane == 31) {                          // the thread that holds the token
            if (a.lse) a.lse[n] = lse;
            if (a.entropy) a.entropy[n] = empty ? 0.0f : ls - LN2 * (v.u / v.s);
            if (a.logp) a.logp[n] = t >= a.V ? quiet_nan() : t < 0 ? 0.0f : empty ? neg_inf() : fmaf(zt - v.m, a.scale, -ls);
            row_m = v.m; row_ls = ls; row_lse = lse;
        }
    }
    if (!TOP) return;
    int n_list = top->n;
    if (blocks > 1) {
        n_list = 0;
        for (int b = 0; b < blocks; ++b) {
            for (int i = threadIdx.x; i < top->count[b]; i += nt) top->list[n_list + i] = merged[b * (CANDS / blocks) + i];
            n_list += top->count[b];
        }
        __syncthreads();
    }
    shrink_list(*top, n_list, a.K, most, (uint32_t)a.V);         // (its barriers publish row_m and the others, too)
    const float lse = row_lse, ls = row_ls, m = row_m;
    const bool broken = !(lse == lse);
    auto put = [&](int at, long long id, float lp) {
        if (a.tok.wide) static_cast<long long*>(a.top_ids)[n * a.K + at] = id;
        else static_cast<int*>(a.top_ids)[n * a.K + at] = (int)id;
        a.top_logp[n * a.K + at] = lp;
    };
    // places by comparison with all others, each entry by as many threads of a warp as there are
    const int left = top->left;
    int split = 1;
    while (split < 32 && left * split * 2 <= nt) split *= 2;
    const int of = (int)threadIdx.x / split, share = (int)threadIdx.x % split;
    const unsigned long long v = of < left ? top->last[of] : 0ull;
    int place = 0;
    for (int x = share; x < left; x += split) place += top->last[x] > v;
    for (int o = 1; o < split; o <<= 1) place += __shfl_xor_sync(~0u, place, o);
    if (of < left && share == 0 && place < a.K && !broken) put(place, ~(uint32_t)v, fmaf(value_of((uint32_t)(v >> 32)) - m, a.scale, -ls));
    for (int k = (broken ? 0 : left) + (int)threadIdx.x; k < a.K; k += nt) put(k, -1, broken ? lse : neg_inf());
}

// One pass over the row: f(q) turns a vector of logits into its gradient.  Four loads in flight; each vector is read and
// written by one thread, so that the gradient may take the logits' place.  `skip`: this row is not for it (false is
// returned).  That depends on a number from memory, and the first loads do not wait for it (40000 rows of 1000 fp32: 64 us
// where they do, 58 so)
__device__ __forceinline__ uint4 read_now(const uint4* p) {
    uint4 q;
    asm volatile("ld.global.cs.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "l"(p));
    return q;
}
template <class T, bool WIDE, class F>
__device__ __forceinline__ bool map_row(const Share<T>& r, T* out, bool skip, F f) {
    const int nt = blockDim.x;
    const uint4* p = r.vectors();
    auto put = [&](int vec, const uint4& g) {
        if (WIDE) __stcs(reinterpret_cast<uint4*>(out - r.head) + vec, g);
        else store_whole(out + r.first(vec), g);
    };
    int vec = r.w0 + (int)threadIdx.x;
    uint4 q[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (vec + j * nt < r.w1) q[j] = read_now(p + vec + j * nt);
    if (skip) return false;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (vec + j * nt < r.w1) put(vec + j * nt, f(q[j], vec + j * nt));
    for (vec += 4 * nt; vec + 3 * nt < r.w1; vec += 4 * nt) {
#pragma unroll
        for (int j = 0; j < 4; ++j) q[j] = __ldcs(p + vec + j * nt);
#pragma unroll
        for (int j = 0; j < 4; ++j) put(vec + j * nt, f(q[j], vec + j * nt));
    }
    for (; vec < r.w1; vec += nt) put(vec, f(__ldcs(p + vec), vec));
    if (threadIdx.x == 0 && r.w0 > r.v0) store_edge(r, out, r.v0, f(r.edge(r.v0), r.v0));
    if ((int)threadIdx.x == nt - 1 && r.w1 < r.v1) store_edge(r, out, r.w1, f(r.edge(r.w1), r.w1));
    return true;
}
template <class T, class F>
__device__ __forceinline__ bool map_row(const Share<T>& r, T* out, bool wide, bool skip, F f) {
    return wide ? map_row<T, true>(r, out, skip, f) : map_row<T, false>(r, out, skip, f);
}

// the same, one vector at a time: rows that are rare
template <class T, class F>
__device__ __forceinline__ void map_row_again(const Share<T>& r, T* out, bool wide, F f) {
    uint4* to = reinterpret_cast<uint4*>(out - r.head);
#pragma unroll 1
    for (int vec = r.v0 + (int)threadIdx.x; vec < r.v1; vec += blockDim.x) {
        const bool whole = vec >= r.w0 && vec < r.w1;
        const uint4 g = f(whole ? __ldcs(r.vectors() + vec) : r.edge(vec), vec);
        if (wide && whole) __stcs(to + vec, g);
        else store_edge(r, out, vec, g);
    }
}

// ------------------------------------------------------------------ gradients from a saved lse
constexpr uint32_t NO_ID = 0xffffffffu;

struct TeacherShared {
    float q[QS_MAX_TOP], logq[QS_MAX_TOP], z[QS_MAX_TOP];
    uint32_t id[QS_MAX_TOP];
    float Q, rest;                         // sum of q, mass left to the other columns (tail)
    float w;                               // weight * scale
    int bad;                               // an id past the last column
};

// the statistics of the ids that lie in the block's share, by one warp (an id given twice is one column)
template <class T>
__device__ __forceinline__ float4 ids_stat(const RowArgs& a, const TeacherShared& t, const Share<T>& r, float c2) {
    constexpr int PER = QS_MAX_TOP / 32;
    const int lane = threadIdx.x & 31;
    float z[PER], m = neg_inf(), s = 0.0f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int k = lane + 32 * i;
        z[i] = neg_inf();
        if (k >= a.K || t.id[k] == NO_ID || !r.holds((int)t.id[k])) continue;
        bool first = true;
        for (int j = 0; j < k; ++j) first &= t.id[j] != t.id[k];
        if (first) z[i] = t.z[k];
        m = fmaxf(m, z[i]);
    }
    m = warp_max(m);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const float at = shift_of(m);
        s += ex2(in_range(at, c2) ? fmaf(z[i], c2, -(at * c2)) : (z[i] - at) * c2);
    }
    return make_float4(m, warp_sum(s), 0.0f, 0.0f);
}
// vectors that an id may name, by their low bits; and those places of a vector dropped
__device__ __forceinline__ void mark_id(uint32_t* marks, int vec) { atomicOr(&marks[(vec & 8191) >> 5], 1u << (vec & 31)); }
template <class T>
__device__ __forceinline__ void drop_ids(uint4& q, int vec, const uint32_t* marks, const TeacherShared& t, int K, int head) {
    constexpr int E = Vec<T>::E;
    if (!(marks[(vec & 8191) >> 5] >> (vec & 31) & 1)) return;
    for (int k = 0; k < K; ++k)
        if (t.id[k] != NO_ID && ((int)t.id[k] + head) / E == vec) drop<T>(q, ((int)t.id[k] + head) % E);
}

// An lse of 32 bits is off by half its last place, and so is every p by that factor: 2^-17 at 256, all of it where the log of
// the sum is lost beside a maximum of -1e9.  Rows beyond that, and rows whose share outside the ids needs the statistics there,
// take them again, in a cluster that first reads all of the row (the gradient may lie in the logits' place).  A row of
// more blocks than a cluster holds is left out by the launch that has them (SAVED), and a second launch, of clusters, takes
// such rows alone (AGAIN): in most calls none.  The clusters cost the other rows up to 1.5 % (4096 rows of 50003: 76.0 us
// and 76.9), a second launch in place of them some 3 us a call
constexpr float LSE_RANGE = 256.0f;
enum { ROWS_ALL = 0, ROWS_SAVED = 1, ROWS_AGAIN = 2 };
__device__ __forceinline__ bool lse_far(float lse) { return fabsf(lse) > LSE_RANGE && lse != neg_inf(); }

constexpr int AGAIN_BLOCKS = 16;               // of such a row's cluster
struct Again {
    float4 part[AGAIN_BLOCKS * MAX_WARPS], in_part[AGAIN_BLOCKS];
    uint32_t marks[256];
};
struct RowStats { Stat all, out; };            // of the row, and (TAIL) of its columns outside the ids
// All threads of the row's blocks.  TAIL: t.z holds the logits at the share's ids
template <class T, bool TAIL>
__device__ __forceinline__ RowStats stats_again(const RowArgs& a, const Share<T>& r, const TeacherShared* t, Again& sh, int rank) {
    const int nt = blockDim.x, warps = nt >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, blocks = 1 << a.parts;
    const float c2 = a.scale * LOG2E;
    if (blocks > 1) cluster_arrive();              // the blocks have started: their shared memory may be written
    if (TAIL) {
        for (int i = threadIdx.x; i < 256; i += nt) sh.marks[i] = 0;
        __syncthreads();
        for (int k = threadIdx.x; k < a.K; k += nt)
            if (t->id[k] != NO_ID && r.holds((int)t->id[k])) mark_id(sh.marks, ((int)t->id[k] + r.head) / Vec<T>::E);
        __syncthreads();
    }
    Stat st{neg_inf(), 0.0f, 0.0f};
    float largest = neg_inf();
    for (int base = r.v0; base < r.v1; base += nt * VPT) {
        uint4 q[VPT];
        load_share<T, VPT>(r, base, nt, q);
        if (TAIL) {
#pragma unroll
            for (int j = 0; j < VPT; ++j)
                if (base + j * nt + (int)threadIdx.x < r.v1) drop_ids<T>(q[j], base + j * nt + (int)threadIdx.x, sh.marks, *t, a.K, r.head);
        }
        const float most = thread_max_of<T, VPT>(q);
        take<T, VPT, false, false>(st, q, most, c2);
        largest = fmaxf(largest, most);
    }
    const Stat w = join_warp<false>(st, largest, c2);
    const float4 sent = make_float4(w.m, w.s, 0.0f, 0.0f), in = TAIL && warp == 0 ? ids_stat<T>(a, *t, r, c2) : sent;
    if (blocks == 1) {
        if (lane == 0) {
            sh.part[warp] = sent;
            if (TAIL && warp == 0) sh.in_part[0] = in;
        }
        __syncthreads();
    } else {
        cluster_wait();
        if (lane < blocks) {
            remote_store(remote_addr(&sh.part[rank * warps + warp], lane), sent);
            if (TAIL && warp == 0) remote_store(remote_addr(&sh.in_part[rank], lane), in);
        }
        cluster_arrive();
        cluster_wait();                            // all of the row has been read; nothing is written to another block after this
    }
    const Stat v = join_parts(sh.part, warps * blocks, c2);
    RowStats x{final_stat(v, c2), Stat{}};
    if (TAIL) {
        const Stat y = join_parts(sh.in_part, blocks, c2);
        const float m = fmaxf(v.m, y.m);
        x.out = x.all;
        x.all = final_stat(Stat{m, rescale(v, m, c2).s + rescale(y, m, c2).s, 0.0f}, c2);
    }
    return x;
}

// What turns a row's log p into its gradient: p times minus (g + h (log p + entropy)), and g at the token
template <class T, bool ENT>
struct LogpSlope {
    long long t;
    int hot;                               // the token's vector
    float hot_g, shift;                    // g scale; minus lse
    f2 scale, slope, offset;

    __device__ __forceinline__ LogpSlope(const RowArgs& a, const Share<T>& r, long long n, float lse, bool tell) {
        t = a.tok.p ? a.tok.at(n) : -1;
        float g = t < 0 ? 0.0f : t >= a.V ? quiet_nan() : a.g1 ? a.g1[n] : a.g_all, h = ENT ? a.g2[n] : 0.0f;
        shift = -lse;
        if (t >= a.V && tell) flag_status(a.status, QS_INVALID_ARG);
        if (lse == neg_inf()) {                    // an empty row: zeros, unless the token makes it NaN
            h = 0.0f;
            if (t < a.V) g = 0.0f;
            shift = LOW_EXP;
        }
        const float at_one = (g + h * (ENT ? a.in_entropy[n] : 0.0f)) * a.scale;
        scale = make_f2(a.scale, a.scale);
        slope = make_f2(-h * a.scale, -h * a.scale);
        offset = make_f2(-at_one, -at_one);
        hot = t >= 0 && t < a.V ? (int)((t + r.head) / Vec<T>::E) : -1;
        hot_g = g * a.scale;
    }
    // log_p: of a pair of logits
    template <class F>
    __device__ __forceinline__ uint4 vec_of(const uint4& q, int vec, int head, F log_p) const {
        const f2 l2e = make_f2(LOG2E, LOG2E);
        f2 d[Vec<T>::E / 2];
#pragma unroll
        for (int i = 0; i < Vec<T>::E / 2; ++i) {
            f2 lp = log_p(Vec<T>::pair(q, i));
            if (ENT) lp = floor2(lp);
            d[i] = mul2(ex2_2(mul2(lp, l2e)), ENT ? fma2(lp, slope, offset) : offset);
        }
        if (vec == hot) {
            const int e = (int)t + head - vec * Vec<T>::E;
#pragma unroll
            for (int i = 0; i < Vec<T>::E / 2; ++i) {
                const float2 p = parts(d[i]);
                d[i] = make_f2(2 * i == e ? p.x + hot_g : p.x, 2 * i + 1 == e ? p.y + hot_g : p.y);
            }
        }
        return Vec<T>::pack(d);
    }
};
template <class T, bool ENT>
__device__ __noinline__ void token_logp_grad_again(const RowArgs& a, Again& sh) {
    const int rank = (int)(blockIdx.x & ((1u << a.parts) - 1u));
    const long long n = a.row0 + (blockIdx.x >> a.parts);
    const Share<T> r(a.logits, a.stride, n, a.V, rank, a.parts);
    const LogpSlope<T, ENT> s(a, r, n, a.in_lse[n], false);
    const Stat v = stats_again<T, false>(a, r, nullptr, sh, rank).all;
    const float m = -shift_of(v.m), ls = -logf(v.s);
    const f2 mm = make_f2(m, m), mls = make_f2(ls, ls);
    map_row_again<T>(r, static_cast<T*>(a.grad) + n * a.grad_stride, a.wide, [&](const uint4& q, int vec) {
        return s.vec_of(q, vec, r.head, [&](f2 z) { return fma2(add2(z, mm), s.scale, mls); });
    });
}

// (six blocks of 40 registers an SM; without the bound the path of rows taken again would have 64 for itself and all others)
template <class T, bool ENT>
__global__ void __launch_bounds__(MAX_THREADS, 6) token_logp_grad_kernel(const __grid_constant__ RowArgs a) {
    __shared__ Again sh;
    const long long n = a.row0 + (blockIdx.x >> a.parts);
    const Share<T> r(a.logits, a.stride, n, a.V, (int)(blockIdx.x & ((1u << a.parts) - 1u)), a.parts);
    const float lse = a.in_lse[n];
    const LogpSlope<T, ENT> s(a, r, n, lse, threadIdx.x == 0);
    const f2 minus = make_f2(s.shift, s.shift);
    if (!map_row<T>(r, static_cast<T*>(a.grad) + n * a.grad_stride, a.wide, lse_far(lse) || a.rows == ROWS_AGAIN, [&](const uint4& q, int vec) {
            return s.vec_of(q, vec, r.head, [&](f2 z) { return fma2(z, s.scale, minus); });
        })) {
        if (lse_far(lse) && a.rows != ROWS_SAVED) token_logp_grad_again<T, ENT>(a, sh);
    }
}

// ------------------------------------------------------------------ distillation
__device__ __forceinline__ float teacher_at(const RowArgs& a, long long i) {
    return a.teacher_type == QS_F32 ? static_cast<const float*>(a.teacher)[i]
         : a.teacher_type == QS_BF16 ? to_float(static_cast<const __nv_bfloat16*>(a.teacher)[i])
                                     : to_float(static_cast<const __half*>(a.teacher)[i]);
}

// One warp's view of a row's entries, as they come from memory: entry lane + 32 i
struct Entries {
    static constexpr int PER = QS_MAX_TOP / 32;
    long long id[PER];
    float u[PER], w;

    __device__ __forceinline__ void load(const RowArgs& a, long long n) {
        w = n < a.N && a.g1 ? a.g1[n] : a.g_all;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int k = (int)(threadIdx.x & 31) + 32 * i;
            id[i] = -1;
            u[i] = 0.0f;
            if (k >= a.K || n >= a.N) continue;
            id[i] = a.tok.at(n * a.K + k);
            u[i] = teacher_at(a, n * a.K + k);
        }
    }
    // the row's probabilities into shared memory
    // (how many of them name a column)
    template <bool TAIL>
    __device__ int finish(const RowArgs& a, TeacherShared& s, bool tell) {
        const int lane = threadIdx.x & 31;
        bool bad = false;
        int entries = 0;
        float m = neg_inf();
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int k = lane + 32 * i;
            const bool named = id[i] >= 0 && id[i] < a.V;
            bad |= id[i] >= a.V;
            entries += __popc(__ballot_sync(~0u, named));
            u[i] = named ? u[i] * a.teacher_scale : neg_inf();
            if (k < a.K) s.id[k] = named ? (uint32_t)id[i] : NO_ID;
            m = fmaxf(m, u[i]);
        }
        bad = __any_sync(~0u, bad);
        m = TAIL ? 0.0f : shift_of(warp_max(m));
        float e[PER], total = 0.0f;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            e[i] = ex2((u[i] - m) * LOG2E);
            total += e[i];
        }
        total = warp_sum(total);
        const float lt = TAIL || total == 0.0f ? 0.0f : logf(total), by = TAIL || total == 0.0f ? 1.0f : 1.0f / total;
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int k = lane + 32 * i;
            const float q = e[i] * by;
            if (k < a.K) {
                s.q[k] = q;
                s.logq[k] = u[i] - m - lt;
            }
            sum += q;
        }
        sum = warp_sum(sum);
        if (lane == 0) {
            s.w = w * a.scale;
            s.Q = sum;
            s.rest = !TAIL ? 0.0f : sum == sum ? fmaxf(0.0f, 1.0f - sum) : sum;
            s.bad = bad;
            if (bad && tell) flag_status(a.status, QS_INVALID_ARG);
        }
        __syncwarp();
        return entries;
    }
};

// What turns a row's probabilities into its gradient: outside the ids f p with f = w (Q + q_T - q_T / p_T), or, where
// p_T is too small for the quotient, w p (Q + q_T) - w q_T share with the column's share of p_T.  That share is taken from
// the statistics of the columns outside: log p - log p_T would be the difference of two large numbers.  At the bound, e^-60,
// a p below the smallest normal number, which counts as 0, would have had 1e-12 of the weight
struct Slope {
    float w, in, out;                      // weight * scale, Q + q_T, and out = f / w
    float rest;
    int thin, empty;
};
// with what the shares take: the largest logit outside the ids; one over the sum relative to it, 0 if there is none
struct Shares : Slope {
    float out_m, out_by;

    __device__ __forceinline__ Shares(const Slope& s, Stat out) : Slope(s), out_m(shift_of(out.m)), out_by(out.s == 0.0f ? 0.0f : 1.0f / out.s) {}
};
template <bool TAIL>
__device__ __forceinline__ Slope slope_of(float w, const TeacherShared& t, bool empty, float log_tail) {
    Slope s;
    s.w = w;
    s.in = t.bad ? quiet_nan() : t.Q + t.rest;
    s.rest = t.rest;
    s.thin = TAIL && t.rest > 0.0f && log_tail < -60.0f;
    s.out = !TAIL ? s.in : s.thin ? s.in : s.in - (t.rest > 0.0f ? t.rest * ex2(-log_tail * LOG2E) : t.rest);
    s.empty = empty;
    return s;
}

// the gradient at an id of the row: all entries that name it count
__device__ __forceinline__ float at_id(const TeacherShared& t, int K, int k, const Slope& s, float p) {
    float q = 0.0f;
    for (int j = 0; j < K; ++j) q += t.id[j] == t.id[k] ? t.q[j] : 0.0f;
    return s.empty ? (t.bad ? s.in : 0.0f) : s.w * fmaf(p, s.in, -q);
}

// The factor that turns 2^d into the gradient outside the ids; norm: 1 over the sum of the row's 2^d
__device__ __forceinline__ float factor(const Slope& s, float norm) {
    return s.empty ? (s.in == s.in ? 0.0f : s.in) : s.w * s.out * norm;
}
// rows whose p_T is too small for the quotient: the shares instead
template <class T>
__device__ __noinline__ uint4 share_vec(uint4 q, const f2* d, const Shares& s, float norm, float c2) {
    constexpr int P = Vec<T>::E / 2;
    f2 g[P];
    const float f = factor(s, norm), c = s.out_by > 0.0f ? -s.w * s.rest * s.out_by : 0.0f;
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const float2 x = parts(d[i]), z = parts(Vec<T>::pair(q, i));
        const float a = c == 0.0f ? 0.0f : c * ex2((z.x - s.out_m) * c2), b = c == 0.0f ? 0.0f : c * ex2((z.y - s.out_m) * c2);
        g[i] = make_f2(fmaf(f, ex2(x.x), a), fmaf(f, ex2(x.y), b));
    }
    return Vec<T>::pack(g);
}
// the gradient of one vector outside the ids, from d = log2 of p times the sum
template <class T>
__device__ __forceinline__ uint4 slope_vec(const f2* d, float f) {
    f2 g[Vec<T>::E / 2];
    const f2 ff = make_f2(f, f);
#pragma unroll
    for (int i = 0; i < Vec<T>::E / 2; ++i) g[i] = mul2(ex2_2(d[i]), ff);
    return Vec<T>::pack(g);
}

// vectors base + j nt + t of the share, from where it is kept or from memory
template <class T, bool KEEP>
__device__ __forceinline__ void load_kept(const Share<T>& r, const uint4* kept, int base, uint4 (&q)[VK]) {
    if (!KEEP) {
        load_share<T, VK>(r, base, blockDim.x, q);
    } else {
#pragma unroll
        for (int j = 0; j < VK; ++j) {
            const int vec = base + j * (int)blockDim.x + (int)threadIdx.x;
            q[j] = all_lowest<T>();
            if (vec < r.v1) q[j] = kept[vec - r.v0];
        }
    }
}

// Loss and, with a.grad, its gradient.  KEEP: the share lies in shared memory from one bulk copy until its gradient is
// written; otherwise (rows beyond a cluster's shared memory) it is read twice
template <class T, bool KEEP, bool TAIL>
__global__ void __launch_bounds__(MAX_THREADS, 4) distill_kernel(const RowArgs a) {
    constexpr int E = Vec<T>::E, PER = (QS_MAX_TOP + 31) / 32;
    extern __shared__ __align__(128) uint4 kept[];
    __shared__ uint64_t landed, met;               // the share's copy; what the row's blocks send to one another
    __shared__ float4 part[PARTS];
    __shared__ float4 in_part[MAX_BLOCKS];         // tail: the statistics of the ids' own columns, block by block
    __shared__ float z_at[QS_MAX_TOP];             // first block: logits at the ids
    __shared__ TeacherShared t;
    __shared__ float row_m, row_by;                // maximum, one over the sum
    __shared__ Slope row;
    __shared__ uint32_t marks[KEEP || !TAIL ? 1 : 256];        // vectors that an id may name, by their low bits
    const int nt = blockDim.x, warps = nt >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, blocks = 1 << a.parts;
    const int rank = blocks == 1 ? 0 : (int)cluster_rank();
    const long long n = a.row0 + (blockIdx.x >> a.parts);
    const float c2 = a.scale * LOG2E;
    if (threadIdx.x == 0) {
        mbar_init(&landed, 1);
        mbar_init(&met, 1);
        fence_async_smem();
        if (blocks > 1) fence_barrier_init();
    }
    if (blocks > 1) cluster_arrive();              // the blocks have started: their shared memory may be written
    const Share<T> r(a.logits, a.stride, n, a.V, rank, a.parts);
    if (KEEP) {
        if (threadIdx.x == 0) {
            const uint32_t bytes = r.w1 > r.w0 ? (uint32_t)(r.w1 - r.w0) * 16u : 0u;
            mbar_expect(&landed, bytes);
            if (bytes) bulk_load(kept + (r.w0 - r.v0), r.vectors() + r.w0, bytes, &landed);
        }
        if ((int)threadIdx.x == nt - 1 && r.w0 > r.v0) kept[0] = r.edge(r.v0);
        if ((int)threadIdx.x == nt - 2 && r.w1 < r.v1) kept[r.w1 - r.v0] = r.edge(r.w1);
    }
    if (!KEEP && TAIL)
        for (int i = threadIdx.x; i < 256; i += nt) marks[i] = 0;
    const int readers = a.grad ? blocks : 1;       // blocks that need the row's statistics
    if (warp == 0) {
        Entries e;
        e.load(a, n);
        const int entries = e.finish<TAIL>(a, t, rank == 0);
        if (lane == 0 && blocks > 1 && rank < readers)
            mbar_expect(&met, blocks * (warps + (TAIL ? 1 : 0)) * (uint32_t)sizeof(float4) + (rank == 0 ? entries * (uint32_t)sizeof(float) : 0u));
    }
    __syncthreads();
    if (blocks > 1) cluster_wait();
    bool ok = true;
    if (KEEP) ok = mbar_wait(&landed, 0, a.wait_ns);
    // logits at the ids of the share
    T* flat = reinterpret_cast<T*>(kept);
    bool named[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int k = (int)threadIdx.x + i * nt;
        named[i] = k < a.K && t.id[k] != NO_ID && r.holds((int)t.id[k]);
        if (!named[i]) continue;
        const int place = (int)t.id[k] + r.head;
        const float z = to_float(KEEP ? flat[place - r.v0 * E] : r.z[t.id[k]]);
        t.z[k] = z;
        if (blocks == 1) z_at[k] = z;
        else send(remote_addr(&z_at[k], 0), z, remote_addr(&met, 0));
        if (!KEEP && TAIL) mark_id(marks, place / E);
    }
    if (TAIL) {                                    // these places leave the sum; their own statistics join later
        __syncthreads();                           // (an id given twice is read twice)
        if (KEEP) {
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (named[i]) flat[(int)t.id[threadIdx.x + i * nt] + r.head - r.v0 * E] = from_float<T>(neg_inf());
            __syncthreads();
        }
    }
    // a share that has not come (see below) makes the row's sums NaN, and so all of its results in every block
    Stat st{neg_inf(), ok ? 0.0f : quiet_nan(), 0.0f};
    float largest = neg_inf();
    // (one loop for all vectors: a second copy of its body for the rest costs more in instruction misses than it saves)
    for (int base = r.v0; base < r.v1; base += nt * VK) {
        uint4 q[VK];
        load_kept<T, KEEP>(r, kept, base, q);
        if (!KEEP && TAIL) {
#pragma unroll
            for (int j = 0; j < VK; ++j) {
                const int vec = base + j * nt + (int)threadIdx.x;
                if (vec < r.v1) drop_ids<T>(q[j], vec, marks, t, a.K, r.head);
            }
        }
        const float most = thread_max_of<T, VK>(q);
        take<T, VK, false, false>(st, q, most, c2);
        largest = fmaxf(largest, most);
    }
    const Stat w = join_warp<false>(st, largest, c2);
    const float4 sent = make_float4(w.m, w.s, 0.0f, 0.0f);
    if (blocks == 1) {
        if (lane == 0) part[warp] = sent;
    } else if (lane < readers) {
        send(remote_addr(&part[rank * warps + warp], lane), sent, remote_addr(&met, lane));
    }
    if (TAIL && warp == 0) {
        const float4 v = ids_stat<T>(a, t, r, c2);
        if (blocks == 1) {
            if (lane == 0) in_part[0] = v;
        } else if (lane < readers) {
            send(remote_addr(&in_part[rank], lane), v, remote_addr(&met, lane));
        }
    }
    if (blocks == 1) __syncthreads();
    else if (rank < readers) ok &= mbar_wait(&met, 0, a.wait_ns);
    if (!ok) {                                     // a copy or a block's sums did not come in time: the row's results are NaN
        if (a.status) atomicExch(a.status, QS_TIMEOUT);
        if (KEEP) mbar_wait(&landed, 0);           // once more, before the memory goes to another block
        if (rank < readers && blocks > 1) mbar_wait(&met, 0);
    }
    if (rank >= readers) return;                   // nothing is sent to this block
    Stat v{};
    float log_tail = 0.0f, out_gap = 0.0f;
    bool empty = false;
    if (warp == 0) {
        v = join_parts(part, warps * blocks, c2);
        if (!ok) v.s = quiet_nan();
        if (TAIL) {
            const Stat in = join_parts(in_part, blocks, c2);
            const float m = fmaxf(v.m, in.m);
            const Stat x = rescale(v, m, c2), y = rescale(in, m, c2);
            const float s = x.s + y.s;
            // log of the share outside: near 1 the difference of two logs would cancel
            const float out_s = final_stat(v, c2).s;
            const bool none = is_empty(v);
            out_gap = v.m - m;
            v = final_stat(Stat{m, s, 0.0f}, c2);
            log_tail = none ? neg_inf() : fmaf(out_gap, a.scale, logf(out_s) - logf(v.s));
            if (!none && log_tail == neg_inf()) log_tail = -FLT_MAX;           // as for lse
            if (log_tail > -0.5f) log_tail = -log1pf(y.s / x.s);
        } else {
            v = final_stat(v, c2);
        }
        empty = is_empty(v);
        const Slope s = slope_of<TAIL>(t.w, t, empty, log_tail);
        if (lane == 0) {
            row_m = shift_of(v.m);
            row_by = empty ? 0.0f : 1.0f / v.s;
            row = s;
        }
    }
    if (a.grad) __syncthreads();
    if (warp == 0 && rank == 0) {                  // while the other warps go on
        const float ls = logf(v.s);
        float loss = 0.0f;
        bool beyond = false, masked = false;       // an entry whose log p is no number; where the student has no mass at all
        for (int k = lane; k < a.K; k += 32) {
            if (t.id[k] == NO_ID || t.q[k] == 0.0f) continue;
            const float lp = empty ? neg_inf() : fmaf(z_at[k] - v.m, a.scale, -ls);
            beyond |= lp == neg_inf();
            loss = fmaf(t.q[k], t.logq[k] - lp, loss);
        }
        if (__any_sync(~0u, beyond)) {             // a log p beyond the largest number, of a column at a lowest value: its product with q need not be
            loss = 0.0f;
            for (int k = lane; k < a.K; k += 32) {
                if (t.id[k] == NO_ID || t.q[k] == 0.0f) continue;
                const float gap = z_at[k] - v.m, lp = fmaf(gap, a.scale, -ls);
                masked |= empty || z_at[k] == neg_inf();
                loss = !empty && lp == neg_inf() && gap > lp ? fmaf(-t.q[k] * a.scale, gap, loss) : fmaf(t.q[k], t.logq[k] - (empty ? neg_inf() : lp), loss);
            }
            masked = __any_sync(~0u, masked);
        }
        loss = warp_sum(loss);
        // a mean of log p at masks of the lowest value that passes the largest number is that number
        if (!masked && loss == -neg_inf()) loss = FLT_MAX;
        if (TAIL && t.rest != 0.0f) {
            loss = log_tail == -FLT_MAX ? fmaf(-t.rest * a.scale, out_gap, loss) : fmaf(t.rest, logf(t.rest) - log_tail, loss);
            if (!masked && log_tail > neg_inf() && loss == -neg_inf()) loss = FLT_MAX;
        }
        if (lane == 0) {
            if (a.loss) a.loss[n] = t.bad || !ok ? quiet_nan() : loss;
            if (a.lse) a.lse[n] = lse_of(v, a.scale, ls);
            if (TAIL && a.log_tail) a.log_tail[n] = log_tail;
        }
    }
    if (!a.grad) return;
    const Slope s = row;
    const float m = row_m, by = row_by;
    T* out = static_cast<T*>(a.grad) + n * a.grad_stride;
    uint4* to = reinterpret_cast<uint4*>(out - r.head);
    // exponents as in the sums: one multiply-add where the reference allows it
    const bool far = !in_range(m, c2), thin = TAIL && s.thin && !s.empty;
    const float ref = m * c2, norm = far ? by : by * ex2(-fmaf(m, c2, -ref)), f = factor(s, norm);
    const f2 c2s = make_f2(c2, c2);
    if (KEEP && a.wide && !far && !thin) {
        const f2 minus = make_f2(-ref, -ref);
        auto grad_of = [&](const uint4& q) {
            f2 d[E / 2];
#pragma unroll
            for (int i = 0; i < E / 2; ++i) d[i] = fma2(Vec<T>::pair(q, i), c2s, minus);
            return slope_vec<T>(d, f);
        };
#pragma unroll 4
        for (int vec = r.w0 + (int)threadIdx.x; vec < r.w1; vec += nt) __stcs(to + vec, grad_of(kept[vec - r.v0]));
        if ((int)threadIdx.x == nt - 1 && r.w0 > r.v0) store_edge(r, out, r.v0, grad_of(kept[0]));
        if ((int)threadIdx.x == nt - 2 && r.w1 < r.v1) store_edge(r, out, r.w1, grad_of(kept[r.w1 - r.v0]));
    } else {
        const f2 minus = far ? make_f2(-m, -m) : make_f2(-ref, -ref);
        auto each = [&](auto grad_of) {
#pragma unroll 1
            for (int vec = r.v0 + (int)threadIdx.x; vec < r.v1; vec += nt) {
                const bool whole = vec >= r.w0 && vec < r.w1;
                const uint4 q = KEEP ? kept[vec - r.v0] : whole ? __ldcs(r.vectors() + vec) : r.edge(vec);
                f2 d[E / 2];
#pragma unroll
                for (int i = 0; i < E / 2; ++i) {
                    const f2 z = Vec<T>::pair(q, i);
                    d[i] = far ? mul2(add2(z, minus), c2s) : fma2(z, c2s, minus);
                }
                const uint4 g = grad_of(q, d);
                if (a.wide && whole) __stcs(to + vec, g);
                else store_edge(r, out, vec, g);
            }
        };
        if (thin) {
            const Shares by_share(s, final_stat(join_parts(part, warps * blocks, c2), c2));
            each([&](const uint4& q, const f2* d) { return share_vec<T>(q, d, by_share, norm, c2); });
        } else each([&](const uint4&, const f2* d) { return slope_vec<T>(d, f); });
    }
    __syncthreads();                               // the ids' places are written last
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int k = (int)threadIdx.x + i * nt;
        if (named[i]) out[t.id[k]] = from_float<T>(at_id(t, a.K, k, s, ex2((t.z[k] - m) * c2) * by));
    }
}

template <class T, bool TAIL>
__device__ __noinline__ void distill_grad_again(const RowArgs& a, const TeacherShared& t, Again& sh) {
    constexpr int E = Vec<T>::E;
    const int rank = (int)(blockIdx.x & ((1u << a.parts) - 1u));
    const long long n = a.row0 + (blockIdx.x >> a.parts);
    const Share<T> r(a.logits, a.stride, n, a.V, rank, a.parts);
    T* out = static_cast<T*>(a.grad) + n * a.grad_stride;
    const RowStats x = stats_again<T, TAIL>(a, r, &t, sh, rank);
    const Shares s(slope_of<TAIL>(t.w, t, is_empty(x.all), TAIL ? a.in_log_tail[n] : 0.0f), x.out);
    const bool thin = TAIL && s.thin && !s.empty;
    const float m = shift_of(x.all.m), ls = s.empty ? -LOW_EXP : logf(x.all.s), f = factor(s, 1.0f), c2 = a.scale * LOG2E;
    const f2 scale = make_f2(a.scale, a.scale), l2e = make_f2(LOG2E, LOG2E), mm = make_f2(-m, -m), mls = make_f2(-ls, -ls);
    map_row_again<T>(r, out, a.wide, [&](const uint4& q, int) {
        f2 d[E / 2];
#pragma unroll
        for (int i = 0; i < E / 2; ++i) d[i] = mul2(fma2(add2(Vec<T>::pair(q, i), mm), scale, mls), l2e);
        return thin ? share_vec<T>(q, d, s, 1.0f, c2) : slope_vec<T>(d, f);
    });
    __syncthreads();
    for (int k = threadIdx.x; k < a.K; k += blockDim.x)
        if (t.id[k] != NO_ID && r.holds((int)t.id[k])) out[t.id[k]] = from_float<T>(at_id(t, a.K, k, s, ex2(fmaf(t.z[k] - m, a.scale, -ls) * LOG2E)));
}

template <class T, bool TAIL>
__global__ void __launch_bounds__(MAX_THREADS, 6) distill_grad_kernel(const __grid_constant__ RowArgs a) {
    constexpr int E = Vec<T>::E;
    __shared__ TeacherShared t;
    __shared__ Again sh;
    const int nt = blockDim.x;
    const long long n = a.row0 + (blockIdx.x >> a.parts);
    const Share<T> r(a.logits, a.stride, n, a.V, (int)(blockIdx.x & ((1u << a.parts) - 1u)), a.parts);
    const float lse = a.in_lse[n], log_tail = TAIL ? a.in_log_tail[n] : 0.0f;
    if (threadIdx.x < 32) {
        Entries e;
        e.load(a, n);
        e.finish<TAIL>(a, t, r.v0 == 0);
    }
    __syncthreads();
    for (int k = threadIdx.x; k < a.K; k += nt)
        if (t.id[k] != NO_ID && r.holds((int)t.id[k])) t.z[k] = to_float(r.z[t.id[k]]);
    __syncthreads();                               // the gradient may take the logits' place
    const Slope s = slope_of<TAIL>(t.w, t, lse == neg_inf(), log_tail);
    T* out = static_cast<T*>(a.grad) + n * a.grad_stride;
    const bool again = lse_far(lse) || (TAIL && s.thin && !s.empty);
    const float shift = s.empty ? LOW_EXP : -lse, f = factor(s, 1.0f);
    const f2 scale = make_f2(a.scale, a.scale), minus = make_f2(shift, shift), l2e = make_f2(LOG2E, LOG2E);
    if (!map_row<T>(r, out, a.wide, again || a.rows == ROWS_AGAIN, [&](const uint4& q, int) {
            f2 d[E / 2];
#pragma unroll
            for (int i = 0; i < E / 2; ++i) d[i] = mul2(fma2(Vec<T>::pair(q, i), scale, minus), l2e);
            return slope_vec<T>(d, f);
        })) {
        if (again && a.rows != ROWS_SAVED) distill_grad_again<T, TAIL>(a, t, sh);
        return;
    }
    __syncthreads();
    for (int k = threadIdx.x; k < a.K; k += nt)
        if (t.id[k] != NO_ID && r.holds((int)t.id[k])) out[t.id[k]] = from_float<T>(at_id(t, a.K, k, s, ex2(fmaf(t.z[k], a.scale, -lse) * LOG2E)));
}

// ------------------------------------------------------------------ launches
// most vectors of a row of V, whatever its alignment
long long most_vectors(int64_t V, int size) { return (V + 2 * (16 / size - 1)) / (16 / size); }

constexpr int SMS = 148;

struct Shape { int nt, blocks; size_t smem; bool keep; };

// Threads of a row's block: few enough that a thread has some eight vectors at least (its share of the row's last steps is
// dear: 65536 rows of 1000 take 102 us with 128 threads, 55 with 32), and a quarter more than alternatives, whose K-th the
// K-th largest of the threads' maxima bounds: with as many threads as alternatives it is the smallest of the maxima, and
// far too many elements reach it.  16384 rows of 4000 bf16, us with 64, 128 and 256 threads: K = 20 84, 105, 191; 48
// 140, 141, 211; 64 272, 181, 244; 100 -, 232, 316; 128 -, 447, 396
int threads_for(long long vectors, int K) {
    int least = K == 0 ? 32 : 64, nt = MAX_THREADS;
    while (least < K + K / 4) least *= 2;
    while (nt > least && vectors <= nt * 8) nt /= 2;
    return nt;
}

// Statistics and alternatives: a block per row; few rows are split over a cluster until the blocks fill the SMs six
// times over, each with a batch at least
Shape stream_shape(int64_t N, long long vectors, int K) {
    Shape s{threads_for(vectors, K), 1, 0, false};
    while (s.blocks < MAX_BLOCKS && N * s.blocks < 6 * SMS && (long long)s.blocks * s.nt * VPT < vectors) s.blocks *= 2;
    return s;
}
// The loss with its gradient: the row is cut into as many shares as keep the most of an SM's shared memory in use, the
// smaller shares where two counts do as well (2 shares of 50 KB for a row of 100 KB, four blocks to an SM: 184 us where
// 4 shares take 199; 8 of 32 KB for one of 256 KB: 227 us, with 4 shares 244; 3, 5 or 7 blocks fit the chip's groups of SMs
// worse, 239 to 249).  Few rows are split further, down to half a batch per thread
constexpr int SHARE_MOST = 200 * 1024 / 16;
int keep_threads(long long share) { return share <= 256 ? 32 : share <= 512 ? 64 : share <= 2048 ? 128 : MAX_THREADS; }
Shape keep_shape(int64_t N, long long vectors) {
    constexpr long long SM_BYTES = 227 * 1024, OWN = 5 * 1024;   // of an SM; what a block takes beside its share
    Shape s{128, MAX_BLOCKS, 0, true};
    long long best = 0;
    for (int b = MAX_BLOCKS; b >= 1; b /= 2) {
        const long long share = (vectors + b - 1) / b, fit = SM_BYTES / (16 * share + OWN), threads = 1024 / keep_threads(share);
        const long long used = (fit < threads ? fit : threads) * share;
        if (fit < 3 || used <= best || (b > 1 && share < 1024)) continue;
        best = used;
        s.blocks = b;
    }
    while (s.blocks < MAX_BLOCKS && N * s.blocks < 6 * SMS && (long long)s.blocks * 512 < vectors) s.blocks *= 2;
    const long long share = (vectors + s.blocks - 1) / s.blocks;
    s.nt = keep_threads(share);
    s.keep = share <= SHARE_MOST;
    s.smem = s.keep ? 16 * (size_t)share : 0;
    return s;
}

template <class K>
cudaError_t launch_rows(K kernel, const Shape& s, RowArgs a, bool cluster, cudaStream_t st) {
    a.parts = 0;
    while ((1 << a.parts) < s.blocks) ++a.parts;
    if (cluster && s.blocks > 8) {                 // (more than every GPU has to offer: this one does)
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return e;
    }
    if (s.smem > 32 * 1024) {                      // (the limit is the function's, for all threads: every call sets the same one)
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 16 * SHARE_MOST);
        if (e != cudaSuccess) return e;
    }
    const long long most = 0x7fffffffll / s.blocks;              // rows per launch
    for (a.row0 = 0; a.row0 < a.N; a.row0 += most) {
        const long long rows = a.N - a.row0 < most ? a.N - a.row0 : most;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)(rows * s.blocks));
        cfg.blockDim = dim3((unsigned)s.nt);
        cfg.dynamicSmemBytes = s.smem;
        cfg.stream = st;
        cudaLaunchAttribute attr;
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = (unsigned)s.blocks;
        attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
        cfg.attrs = &attr;
        cfg.numAttrs = cluster && s.blocks > 1 ? 1 : 0;
        const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, a);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

// The backward calls: blocks with some sixteen vectors per thread of their row, or four where there are few rows
Shape grad_shape(int64_t N, long long vectors) {
    Shape s{vectors <= 2048 ? 64 : MAX_THREADS, 1, 0, false};
    while ((long long)s.blocks * s.nt * 16 < vectors ||
           (s.blocks < AGAIN_BLOCKS && N * s.blocks < 8 * SMS && (long long)s.blocks * s.nt * 4 < vectors)) s.blocks *= 2;
    return s;
}
// a row in a cluster, or in more blocks than one holds: then the rows whose statistics are taken again follow (see LSE_RANGE)
template <class K>
cudaError_t launch_grad(K kernel, RowArgs a, long long vectors, cudaStream_t st) {
    Shape s = grad_shape(a.N, vectors);
    a.rows = s.blocks <= AGAIN_BLOCKS ? ROWS_ALL : ROWS_SAVED;
    const cudaError_t e = launch_rows(kernel, s, a, a.rows == ROWS_ALL, st);
    if (e != cudaSuccess || a.rows == ROWS_ALL) return e;
    s.blocks = AGAIN_BLOCKS;
    a.rows = ROWS_AGAIN;
    return launch_rows(kernel, s, a, true, st);
}

template <class T>
cudaError_t launch_token_logp(RowArgs a, cudaStream_t st) {
    Shape s = stream_shape(a.N, most_vectors(a.V, sizeof(T)), a.K);
    if (a.K > 0) {
        const long long share = (most_vectors(a.V, sizeof(T)) + s.blocks - 1) / s.blocks, batches = (share + s.nt * VPT - 1) / (s.nt * VPT);
        a.per = (int)((batches + SLOTS - 1) / SLOTS);
        // (a slot more: the loop may close the last one)
        s.smem = (s.blocks > 1 ? sizeof(unsigned long long) * CANDS : 0) + sizeof(float) * s.nt * ((batches + a.per - 1) / a.per + 1);
    }
    return launch_rows(a.K > 0 ? token_logp_kernel<T, true> : token_logp_kernel<T, false>, s, a, true, st);
}
template <class T>
cudaError_t launch_token_logp_grad(const RowArgs& a, cudaStream_t st) {
    return launch_grad(a.g2 ? token_logp_grad_kernel<T, true> : token_logp_grad_kernel<T, false>, a, most_vectors(a.V, sizeof(T)), st);
}
template <class T>
cudaError_t launch_distill(const RowArgs& a, bool tail, cudaStream_t st) {
    const long long vectors = most_vectors(a.V, sizeof(T));
    const Shape s = keep_shape(a.N, vectors);
    if (s.keep) return launch_rows(tail ? distill_kernel<T, true, true> : distill_kernel<T, true, false>, s, a, true, st);
    return launch_rows(tail ? distill_kernel<T, false, true> : distill_kernel<T, false, false>, s, a, true, st);
}
template <class T>
cudaError_t launch_distill_grad(const RowArgs& a, bool tail, cudaStream_t st) {
    return launch_grad(tail ? distill_grad_kernel<T, true> : distill_grad_kernel<T, false>, a, most_vectors(a.V, sizeof(T)), st);
}

// Two seconds, or less: QSPARSE_WAIT_LIMIT_NS, read once; 0 gives up at once (a test of what follows)
unsigned long long wait_limit() {
    static const unsigned long long ns = [] {
        const char* e = std::getenv("QSPARSE_WAIT_LIMIT_NS");
        return e ? std::min(std::strtoull(e, nullptr, 10), WAIT_LIMIT_NS) : WAIT_LIMIT_NS;
    }();
    return ns;
}

#define QS_BY_TYPE(launch, type, ...) \
    status_of((type) == QS_F32 ? launch<float>(__VA_ARGS__) : (type) == QS_BF16 ? launch<__nv_bfloat16>(__VA_ARGS__) : launch<__half>(__VA_ARGS__))

// whether gradient rows lie like logits rows within 16 bytes
int lie_alike(const void* z, int64_t stride, const void* g, int64_t g_stride, int size) {
    return ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(g)) & 15u) == 0 && (stride - g_stride) * size % 16 == 0;
}

bool bad_rows(int64_t N, int64_t V, int type, int64_t stride, float scale) {
    return N < 0 || V < 1 || !size_of_type(type) || stride < V || !(scale > 0.0f) || !std::isfinite(scale);
}
bool rows_too_large(int64_t N, int64_t V) { return N > (1ll << 30) || V > (1ll << 30); }
bool ok_floats(const void* p) { return aligned_to(p, 4); }

// the gradient may take the logits' own place, row for row, or other columns of the same rows; any other overlap is refused
bool overlap(const void* z, int64_t stride, const void* g, int64_t g_stride, int64_t N, int64_t V, int size) {
    typedef __int128 wide;
    const wide z0 = reinterpret_cast<uintptr_t>(z), g0 = reinterpret_cast<uintptr_t>(g), row = (wide)stride * size, len = (wide)V * size;
    if (z0 == g0 && stride == g_stride) return false;
    const wide z1 = z0 + (N - 1) * row + len, g1 = g0 + (N - 1) * (wide)g_stride * size + len;
    if (z1 <= g0 || g1 <= z0) return false;
    if (stride != g_stride) return true;
    const wide apart = ((g0 - z0) % row + row) % row;            // from a row of logits to the next row of results
    return apart < len || apart + len > row;
}

}  // namespace

extern "C" {

int qs_token_logp(int64_t N, int64_t V, const void* logits, int type, int64_t row_stride, const void* tokens, int token_type,
                  float scale, int top, float* logp, float* lse, float* entropy, void* top_ids, float* top_logp, int* status,
                  void* cuda_stream) {
    if (bad_rows(N, V, type, row_stride, scale) || !is_id_type(token_type) || top < 0 || top > QS_MAX_TOP || top > V) return QS_INVALID_ARG;
    if (rows_too_large(N, V)) return QS_TOO_LARGE;
    if (N == 0) return QS_OK;
    const int id_bytes = token_type == QS_I64 ? 8 : 4;
    if (!logits || !aligned_to(logits, size_of_type(type)) || (logp && !tokens) || !aligned_to(tokens, id_bytes) || !ok_floats(logp) ||
        !ok_floats(lse) || !ok_floats(entropy) || !ok_floats(status) ||
        (top && (!top_ids || !top_logp || !aligned_to(top_ids, id_bytes) || !ok_floats(top_logp)))) return QS_INVALID_ARG;
    RowArgs a{};
    a.N = N; a.V = V; a.logits = logits; a.stride = row_stride; a.scale = scale;
    a.tok = Ids{tokens, token_type == QS_I64}; a.K = top;
    a.logp = logp; a.lse = lse; a.entropy = entropy; a.top_ids = top_ids; a.top_logp = top_logp; a.status = status;
    return QS_BY_TYPE(launch_token_logp, type, a, static_cast<cudaStream_t>(cuda_stream));
}

int qs_token_logp_grad(int64_t N, int64_t V, const void* logits, int type, int64_t row_stride, const void* tokens, int token_type,
                       float scale, const float* lse, const float* entropy, const float* grad_logp, float grad_logp_all,
                       const float* grad_entropy, void* grad, int64_t grad_stride, int* status, void* cuda_stream) {
    if (bad_rows(N, V, type, row_stride, scale) || !is_id_type(token_type) || grad_stride < V) return QS_INVALID_ARG;
    if (rows_too_large(N, V)) return QS_TOO_LARGE;
    if (N == 0) return QS_OK;
    const int size = size_of_type(type);
    if (!logits || !grad || !lse || (grad_entropy && !entropy) || !aligned_to(logits, size) || !aligned_to(grad, size) ||
        !aligned_to(tokens, token_type == QS_I64 ? 8 : 4) || !ok_floats(lse) || !ok_floats(entropy) || !ok_floats(grad_logp) ||
        !ok_floats(grad_entropy) || !ok_floats(status) || overlap(logits, row_stride, grad, grad_stride, N, V, size)) return QS_INVALID_ARG;
    RowArgs a{};
    a.N = N; a.V = V; a.logits = logits; a.stride = row_stride; a.scale = scale;
    a.tok = Ids{tokens, token_type == QS_I64};
    a.in_lse = lse; a.in_entropy = entropy; a.g1 = grad_logp; a.g_all = grad_logp_all; a.g2 = grad_entropy;
    a.grad = grad; a.grad_stride = grad_stride; a.status = status;
    a.wide = lie_alike(logits, row_stride, grad, grad_stride, size);
    return QS_BY_TYPE(launch_token_logp_grad, type, a, static_cast<cudaStream_t>(cuda_stream));
}

int qs_distill(int64_t N, int64_t V, int K, const void* logits, int type, int64_t row_stride, const void* ids, int id_type,
               const void* teacher, int teacher_type, float scale, float teacher_scale, int tail, float* loss, float* lse,
               float* log_tail, const float* weight, float weight_all, void* grad, int64_t grad_stride, int* status, void* cuda_stream) {
    if (bad_rows(N, V, type, row_stride, scale) || !is_id_type(id_type) || !size_of_type(teacher_type) || K < 1 || K > QS_MAX_TOP ||
        !std::isfinite(teacher_scale) || (grad && grad_stride < V)) return QS_INVALID_ARG;
    if (rows_too_large(N, V)) return QS_TOO_LARGE;
    if (N == 0) return QS_OK;
    const int size = size_of_type(type);
    if (!logits || !ids || !teacher || !aligned_to(logits, size) || !aligned_to(ids, id_type == QS_I64 ? 8 : 4) ||
        !aligned_to(teacher, size_of_type(teacher_type)) || !ok_floats(loss) || !ok_floats(lse) || !ok_floats(log_tail) || !ok_floats(weight) ||
        !ok_floats(status) || (grad && (!aligned_to(grad, size) || overlap(logits, row_stride, grad, grad_stride, N, V, size)))) return QS_INVALID_ARG;
    RowArgs a{};
    a.N = N; a.V = V; a.logits = logits; a.stride = row_stride; a.scale = scale;
    a.tok = Ids{ids, id_type == QS_I64}; a.K = K; a.teacher = teacher; a.teacher_type = teacher_type; a.teacher_scale = teacher_scale;
    a.loss = loss; a.lse = lse; a.log_tail = log_tail; a.g1 = weight; a.g_all = weight_all; a.wait_ns = wait_limit();
    a.grad = grad; a.grad_stride = grad_stride; a.status = status;
    a.wide = grad && lie_alike(logits, row_stride, grad, grad_stride, size);
    return QS_BY_TYPE(launch_distill, type, a, tail != 0, static_cast<cudaStream_t>(cuda_stream));
}

int qs_distill_grad(int64_t N, int64_t V, int K, const void* logits, int type, int64_t row_stride, const void* ids, int id_type,
                    const void* teacher, int teacher_type, float scale, float teacher_scale, int tail, const float* lse,
                    const float* log_tail, const float* weight, float weight_all, void* grad, int64_t grad_stride, int* status,
                    void* cuda_stream) {
    if (bad_rows(N, V, type, row_stride, scale) || !is_id_type(id_type) || !size_of_type(teacher_type) || K < 1 || K > QS_MAX_TOP ||
        !std::isfinite(teacher_scale) || grad_stride < V) return QS_INVALID_ARG;
    if (rows_too_large(N, V)) return QS_TOO_LARGE;
    if (N == 0) return QS_OK;
    const int size = size_of_type(type);
    if (!logits || !ids || !teacher || !lse || (tail && !log_tail) || !grad || !aligned_to(logits, size) ||
        !aligned_to(ids, id_type == QS_I64 ? 8 : 4) || !aligned_to(teacher, size_of_type(teacher_type)) || !ok_floats(lse) ||
        !ok_floats(log_tail) || !ok_floats(weight) || !ok_floats(status) || !aligned_to(grad, size) ||
        overlap(logits, row_stride, grad, grad_stride, N, V, size)) return QS_INVALID_ARG;
    RowArgs a{};
    a.N = N; a.V = V; a.logits = logits; a.stride = row_stride; a.scale = scale;
    a.tok = Ids{ids, id_type == QS_I64}; a.K = K; a.teacher = teacher; a.teacher_type = teacher_type; a.teacher_scale = teacher_scale;
    a.in_lse = lse; a.in_log_tail = log_tail; a.g1 = weight; a.g_all = weight_all;
    a.grad = grad; a.grad_stride = grad_stride; a.status = status;
    a.wide = lie_alike(logits, row_stride, grad, grad_stride, size);
    return QS_BY_TYPE(launch_distill_grad, type, a, tail != 0, static_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"
