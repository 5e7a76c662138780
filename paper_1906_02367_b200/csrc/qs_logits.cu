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
// one.  So a row is read once.  A cluster of up to 8 blocks holds it in registers (qs_rows.cuh); the blocks put
// their statistics into one another's shared memory, and the same registers then give the gradient or the
// alternatives.  The backward calls, which start from a saved lse, need no cluster.
#include "qs_rows.cuh"

namespace {

using namespace qs;

constexpr int MAX_BLOCKS = 8;              // blocks of a row's cluster
constexpr int MAX_WARPS = 16;              // warps of a block
constexpr int MAX_THREADS = 32 * MAX_WARPS;
constexpr int PARTS = MAX_BLOCKS * MAX_WARPS;
constexpr int MAX_GROUPS = 1024;           // maxima that bound the K-th alternative
constexpr int CANDS = 1024;                // candidates a row's blocks may send, CANDS / blocks each (>= QS_MAX_TOP)
constexpr int RANK_MOST = 256;             // candidates ranked against one another without a further cut (>= QS_MAX_TOP)

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
    int blocks;                            // blocks per row
    int groups;                            // maxima per warp that bound the K-th alternative
    int* status;
};

// ------------------------------------------------------------------ log probabilities
// Places that a cut takes: key above the cut's, or equal to it with a column at or below the cut's
struct Cut { uint32_t key, idx; };
__device__ __forceinline__ bool takes(Cut c, uint32_t key, uint32_t idx) { return key > c.key || (key == c.key && idx <= c.idx); }

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

// A cut that takes between K and `most` places, by bisection over the keys and then, where equal keys alone are more
// than that, over the columns.  `count(cut)` is the number of places a cut takes; Cut{lo, ~0} takes more than `most`
template <class Count>
__device__ Cut find_cut(int K, int most, uint32_t lo, uint32_t columns, Count count) {
    uint32_t hi = 0xffffffffu;
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

// calls f(key, column) for the elements of the share
template <class T, int VPT, bool ONE, class F>
__device__ __forceinline__ void each_element(const Share<T>& r, uint4 (&q)[VPT], F f) {
    const int nt = blockDim.x;
    for (int base = r.v0; base < r.v1; base += nt * VPT) {
        if (!ONE) load_share<T, VPT>(r, base, nt, q);
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int e0 = r.first(base + j * nt + (int)threadIdx.x);
#pragma unroll
            for (int i = 0; i < Vec<T>::E / 2; ++i) {
                const float2 p = parts(Vec<T>::pair(q[j], i));
                f(p.x, (uint32_t)(e0 + 2 * i));
                f(p.y, (uint32_t)(e0 + 2 * i + 1));
            }
        }
    }
}

struct TopShared {
    uint32_t group[MAX_GROUPS];            // keys of the group maxima of the whole row
    unsigned long long cand[CANDS];        // (key, ~column); block b's at b * CANDS / blocks
    int count[MAX_BLOCKS];                 // of which there are
    int mine, sums[MAX_WARPS];
    uint32_t bound;
};

// The largest key found that at least K of the row's group maxima reach: no alternative lies below it.  One warp
__device__ __forceinline__ uint32_t group_bound(const uint32_t* group, int n, int K) {
    const int lane = threadIdx.x & 31;
    uint32_t top = 0;
    int live = 0;
    for (int i = lane; i < n; i += 32) {
        top = max(top, group[i]);
        live += group[i] >= KEY_LOWEST;
    }
    top = __reduce_max_sync(~0u, top);
    if (__reduce_add_sync(~0u, live) < K) return KEY_LOWEST;
    uint32_t lo = KEY_LOWEST, hi = top + 1;
    while (hi - lo > 1) {
        const uint32_t mid = lo + (hi - lo) / 2;
        int c = 0;
        for (int i = lane; i < n; i += 32) c += group[i] >= mid;
        c = __reduce_add_sync(~0u, c);
        if (c >= K) {
            lo = mid;
            if (c <= K + K / 4 + 1) break;
        } else {
            hi = mid;
        }
    }
    return lo;
}

template <class T, int VPT, bool ONE, bool TOP>
__global__ void __launch_bounds__(MAX_THREADS) token_logp_kernel(const RowArgs a) {
    __shared__ float4 part[PARTS];
    __shared__ float row_m, row_ls, row_lse;
    __shared__ TopShared top[1];                   // (no room where it is not used)
    const int nt = blockDim.x, warps = nt >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, blocks = a.blocks;
    const int rank = blocks == 1 ? 0 : (int)cluster_rank();
    const long long n = a.row0 + blockIdx.x / blocks;
    const float c2 = a.scale * LOG2E;
    if (blocks > 1) cluster_arrive();              // the blocks have started: their shared memory may be written
    const Share<T> r(a.logits, a.stride, n, a.V, rank, blocks);
    uint4 q[VPT];
    Stat st{neg_inf(), 0.0f, 0.0f};
    float mine = neg_inf();
    if (ONE) {
        load_share<T, VPT>(r, r.v0, nt, q);
        mine = thread_max_of<T, VPT>(q);
        st = warp_stat<T, VPT, true>(q, mine, c2);
    } else {
        for (int base = r.v0; base < r.v1; base += nt * VPT) {
            load_share<T, VPT>(r, base, nt, q);
            const float tm = thread_max_of<T, VPT>(q);
            const Stat now = warp_stat<T, VPT, true>(q, tm, c2);
            const float m = fmaxf(st.m, now.m);
            const Stat x = rescale(st, m, c2), y = rescale(now, m, c2);
            st = Stat{m, x.s + y.s, x.u + y.u};
            mine = fmaxf(mine, tm);
        }
    }
    long long t = -1;
    float zt = 0.0f;
    if (rank == 0 && threadIdx.x == 32 && a.logp) {
        t = a.tok.at(n);
        if (t >= a.V) flag_status(a.status, QS_INVALID_ARG);
        else if (t >= 0) zt = to_float(r.z[t]);
    }
    if (blocks > 1) cluster_wait();
    const float4 sent = make_float4(st.m, st.s, st.u, 0.0f);
    if (blocks == 1) {
        if (lane == 0) part[warp] = sent;
    } else if (lane < (TOP ? blocks : 1)) {
        remote_store(remote_addr(&part[rank * warps + warp], lane), sent);
    }
    if (TOP) {
        const int width = 32 / a.groups;
        float g = mine;
        for (int o = 1; o < width; o <<= 1) g = fmaxf(g, __shfl_xor_sync(~0u, g, o));
        const int at = (rank * warps + warp) * a.groups + lane / width;
        if (lane % width == 0) {
            if (blocks == 1) top->group[at] = key_of(g);
            else
                for (int b = 0; b < blocks; ++b) remote_store(remote_addr(&top->group[at], b), key_of(g));
        }
    }
    if (blocks == 1) {
        __syncthreads();
    } else {
        cluster_arrive();
        if (!TOP && rank != 0) return;             // nothing is written into this block's memory
        cluster_wait();
    }
    if (rank == 0 && warp == 1) {
        const Stat v = join_parts(part, warps * blocks, c2);
        const bool empty = v.m == neg_inf() && v.s == 0.0f;
        const float ls = logf(v.s), lse = empty ? neg_inf() : fmaf(v.m, a.scale, ls);
        if (lane == 0) {
            if (a.lse) a.lse[n] = lse;
            if (a.entropy) a.entropy[n] = empty ? 0.0f : ls - LN2 * (v.u / v.s);
            if (a.logp) a.logp[n] = t >= a.V ? quiet_nan() : t < 0 ? 0.0f : empty ? neg_inf() : fmaf(zt - v.m, a.scale, -ls);
            row_m = v.m; row_ls = ls; row_lse = lse;
        }
    }
    if (!TOP) return;

    if (warp == 0) {
        const uint32_t b = group_bound(top->group, warps * blocks * a.groups, a.K);
        if (lane == 0) { top->bound = b; top->mine = 0; }
    }
    __syncthreads();
    const int room = CANDS / blocks;
    const float bound = value_of(top->bound);
    auto send = [&](float z, uint32_t col) {
        const int slot = atomicAdd(&top->mine, 1);
        if (slot >= room) return;
        const unsigned long long v = ((unsigned long long)key_of(z) << 32) | (uint32_t)~col;
        if (blocks == 1) top->cand[slot] = v;
        else remote_store(remote_addr(&top->cand[rank * room + slot], 0), v);
    };
    if (mine >= bound) {
        for (int base = r.v0; base < r.v1; base += nt * VPT) {
            if (!ONE) load_share<T, VPT>(r, base, nt, q);
#pragma unroll
            for (int j = 0; j < VPT; ++j) {
                if (!(Vec<T>::top(max_of_words<T>(q[j])) >= bound)) continue;
                const int e0 = r.first(base + j * nt + (int)threadIdx.x);
#pragma unroll
                for (int i = 0; i < Vec<T>::E / 2; ++i) {
                    const float2 p = parts(Vec<T>::pair(q[j], i));
                    if (p.x >= bound) send(p.x, (uint32_t)(e0 + 2 * i));
                    if (p.y >= bound) send(p.y, (uint32_t)(e0 + 2 * i + 1));
                }
            }
        }
    }
    __syncthreads();
    if (top->mine > room) {                        // a mask, ties or an order that defeats the bound: cut exactly
        const Cut cut = find_cut(a.K, room, top->bound, (uint32_t)a.V, [&](Cut c) {
            int k = 0;
            each_element<T, VPT, ONE>(r, q, [&](float z, uint32_t col) { k += z > neg_inf() && takes(c, key_of(z), col); });
            return block_count(k, top->sums);
        });
        __syncthreads();
        if (threadIdx.x == 0) top->mine = 0;
        __syncthreads();
        each_element<T, VPT, ONE>(r, q, [&](float z, uint32_t col) {
            if (z > neg_inf() && takes(cut, key_of(z), col)) send(z, col);
        });
        __syncthreads();
    }
    if (blocks == 1) {
        if (threadIdx.x == 0) top->count[0] = top->mine;
        __syncthreads();
    } else {
        if (threadIdx.x == 0) remote_store(remote_addr(&top->count[rank], 0), (uint32_t)top->mine);
        cluster_arrive();
        if (rank != 0) return;
        cluster_wait();
    }

    // the row's first block ranks the candidates
    int total = 0;
    for (int b = 0; b < blocks; ++b) total += top->count[b];
    const float lse = row_lse, ls = row_ls, m = row_m;
    const bool broken = !(lse == lse);
    Cut cut{0, 0xffffffffu};
    if (total > RANK_MOST)
        cut = find_cut(a.K, RANK_MOST, KEY_LOWEST - 1, (uint32_t)a.V, [&](Cut c) {
            int k = 0;
            for (int b = 0; b < blocks; ++b)
                for (int i = threadIdx.x; i < top->count[b]; i += nt) {
                    const unsigned long long v = top->cand[b * room + i];
                    k += takes(c, (uint32_t)(v >> 32), ~(uint32_t)v);
                }
            return block_count(k, top->sums);
        });
    auto put = [&](int at, long long id, float lp) {
        if (a.tok.wide) static_cast<long long*>(a.top_ids)[n * a.K + at] = id;
        else static_cast<int*>(a.top_ids)[n * a.K + at] = (int)id;
        a.top_logp[n * a.K + at] = lp;
    };
    for (int b = 0; b < blocks && !broken; ++b)
        for (int i = threadIdx.x; i < top->count[b]; i += nt) {
            const unsigned long long v = top->cand[b * room + i];
            const uint32_t key = (uint32_t)(v >> 32), col = ~(uint32_t)v;
            if (!takes(cut, key, col)) continue;
            int place = 0;
            for (int d = 0; d < blocks; ++d)
                for (int x = 0; x < top->count[d]; ++x) place += top->cand[d * room + x] > v;
            if (place < a.K) put(place, col, fmaf(value_of(key) - m, a.scale, -ls));
        }
    for (int k = (broken ? 0 : total) + (int)threadIdx.x; k < a.K; k += nt) put(k, -1, broken ? lse : neg_inf());
}

template <class T, int VPT, bool ENT>
__global__ void __launch_bounds__(256) token_logp_grad_kernel(const RowArgs a) {
    const int nt = blockDim.x;
    const long long n = a.row0 + blockIdx.x / a.blocks;
    const Share<T> r(a.logits, a.stride, n, a.V, (int)(blockIdx.x % a.blocks), a.blocks);
    uint4 q[VPT];
    load_share<T, VPT>(r, r.v0, nt, q);
    T* out = static_cast<T*>(a.grad) + n * a.grad_stride;
    const long long t = a.tok.p ? a.tok.at(n) : -1;
    const float lse = a.in_lse[n];
    const bool empty = lse == neg_inf();
    float g = t < 0 ? 0.0f : t >= a.V ? quiet_nan() : a.g1 ? a.g1[n] : a.g_all;
    float h = ENT ? a.g2[n] : 0.0f, shift = -lse;
    if (t >= a.V && threadIdx.x == 0) flag_status(a.status, QS_INVALID_ARG);
    if (empty) {                                   // zeros, unless the token makes the row NaN
        h = 0.0f;
        if (t < a.V) g = 0.0f;
        shift = LOW_EXP;
    }
    const float at_one = (g + h * (ENT ? a.in_entropy[n] : 0.0f)) * a.scale;
    const f2 scale = make_f2(a.scale, a.scale), minus = make_f2(shift, shift), l2e = make_f2(LOG2E, LOG2E);
    const f2 slope = make_f2(-h * a.scale, -h * a.scale), offset = make_f2(-at_one, -at_one);
    const int hot = t >= 0 && t < a.V ? (int)((t + r.head) / Vec<T>::E) : -1;
    const float hot_g = g * a.scale;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int vec = r.v0 + j * nt + (int)threadIdx.x;
        if (vec >= r.v1) continue;
        f2 d[Vec<T>::E / 2];
#pragma unroll
        for (int i = 0; i < Vec<T>::E / 2; ++i) {
            // log p; p times minus (g + h (log p + entropy))
            f2 lp = fma2(Vec<T>::pair(q[j], i), scale, minus);
            if (ENT) lp = floor2(lp);
            d[i] = mul2(ex2_2(mul2(lp, l2e)), ENT ? fma2(lp, slope, offset) : offset);
        }
        if (vec == hot) {
            const int e = (int)t + r.head - vec * Vec<T>::E;
#pragma unroll
            for (int i = 0; i < Vec<T>::E / 2; ++i) {
                const float2 p = parts(d[i]);
                d[i] = make_f2(2 * i == e ? p.x + hot_g : p.x, 2 * i + 1 == e ? p.y + hot_g : p.y);
            }
        }
        store_vec(r, out, vec, Vec<T>::pack(d), a.wide);
    }
}

// ------------------------------------------------------------------ distillation
constexpr uint32_t NO_ID = 0xffffffffu;

struct TeacherShared {
    float q[QS_MAX_TOP], logq[QS_MAX_TOP], z[QS_MAX_TOP];
    uint32_t id[QS_MAX_TOP];
    float Q, rest;                         // sum of q, mass left to the other columns (tail)
    int bad;                               // an id past the last column
};

__device__ __forceinline__ float teacher_at(const RowArgs& a, long long i) {
    return a.teacher_type == QS_F32 ? static_cast<const float*>(a.teacher)[i]
         : a.teacher_type == QS_BF16 ? to_float(static_cast<const __nv_bfloat16*>(a.teacher)[i])
                                     : to_float(static_cast<const __half*>(a.teacher)[i]);
}

// One warp: the row's entries, their probabilities, and the logits at those ids that are in the share (`all`: at all)
template <class T, bool TAIL>
__device__ void load_teacher(const RowArgs& a, long long n, const Share<T>& r, bool all, TeacherShared& s) {
    constexpr int PER = QS_MAX_TOP / 32;
    const int lane = threadIdx.x & 31;
    float u[PER];
    bool bad = false;
    float m = neg_inf();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int k = lane + 32 * i;
        u[i] = neg_inf();
        if (k >= a.K) continue;
        const long long id = a.tok.at(n * a.K + k);
        const bool named = id >= 0 && id < a.V;
        bad |= id >= a.V;
        s.id[k] = named ? (uint32_t)id : NO_ID;
        if (!named) continue;
        u[i] = teacher_at(a, n * a.K + k) * a.teacher_scale;
        if (all || r.holds((int)id)) s.z[k] = to_float(r.z[id]);
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
        s.Q = sum;
        s.rest = !TAIL ? 0.0f : sum == sum ? fmaxf(0.0f, 1.0f - sum) : sum;
        s.bad = bad;
        if (bad && r.v0 == 0) flag_status(a.status, QS_INVALID_ARG);
    }
    __syncwarp();
}

// What turns a row's probabilities into its gradient: outside the ids f p with f = w (Q + q_T - q_T / p_T), or, where
// p_T is too small for the quotient, w p (Q + q_T) - w q_T exp(log p - log p_T)
struct Slope {
    float w, in, out;                      // weight * scale, Q + q_T, and out = f / w
    float rest, log_tail;
    int thin, empty;
};
template <bool TAIL>
__device__ __forceinline__ Slope slope_of(const RowArgs& a, long long n, const TeacherShared& t, float lse, float log_tail) {
    Slope s;
    s.w = (a.g1 ? a.g1[n] : a.g_all) * a.scale;
    s.in = t.bad ? quiet_nan() : t.Q + t.rest;
    s.rest = t.rest;
    s.log_tail = log_tail;
    s.thin = TAIL && t.rest > 0.0f && log_tail < -60.0f;
    s.out = !TAIL ? s.in : s.thin ? s.in : s.in - (t.rest > 0.0f ? t.rest * ex2(-log_tail * LOG2E) : t.rest);
    s.empty = lse == neg_inf();
    return s;
}

// the gradient at an id of the row: all entries that name it count
__device__ __forceinline__ float at_id(const TeacherShared& t, int K, int k, const Slope& s, float p) {
    float q = 0.0f;
    for (int j = 0; j < K; ++j) q += t.id[j] == t.id[k] ? t.q[j] : 0.0f;
    return s.empty ? (t.bad ? s.in : 0.0f) : s.w * fmaf(p, s.in, -q);
}

// the gradient of one vector outside the ids, from d = log2 of p up to the factor 1 / norm
template <class T, bool TAIL>
__device__ __forceinline__ uint4 slope_vec(const f2* d, const Slope& s, float norm) {
    constexpr int P = Vec<T>::E / 2;
    f2 g[P];
    const float f = s.empty ? (s.in == s.in ? 0.0f : s.in) : s.w * s.out * norm;
    const f2 ff = make_f2(f, f);
#pragma unroll
    for (int i = 0; i < P; ++i) g[i] = mul2(ex2_2(d[i]), ff);
    if (TAIL && s.thin && !s.empty && s.log_tail > neg_inf()) {
        // 2^d norm / p_T, exponents first: norm is 1 / sum of the row's exponentials, or 1
        const float sub = s.log_tail * LOG2E - log2f(norm), c = -s.w * s.rest;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const float2 x = parts(d[i]), y = parts(g[i]);
            g[i] = make_f2(fmaf(c, ex2(x.x - sub), y.x), fmaf(c, ex2(x.y - sub), y.y));
        }
    }
    return Vec<T>::pack(g);
}

template <class T, int VPT, bool ONE, bool TAIL>
__global__ void __launch_bounds__(MAX_THREADS) distill_kernel(const RowArgs a) {
    constexpr int E = Vec<T>::E;
    __shared__ float4 part[PARTS];
    __shared__ float4 in_part[MAX_BLOCKS];         // tail: the statistics of the ids' own columns, block by block
    __shared__ TeacherShared t;
    __shared__ float row_m, row_by;                // maximum, one over the sum
    __shared__ Slope row;
    __shared__ __align__(16) uint8_t named[TAIL ? MAX_THREADS * VPT : 1];      // per vector of the round: places that an id names
    const int nt = blockDim.x, warps = nt >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, blocks = a.blocks;
    const int rank = blocks == 1 ? 0 : (int)cluster_rank();
    const long long n = a.row0 + blockIdx.x / blocks;
    const float c2 = a.scale * LOG2E;
    if (blocks > 1) cluster_arrive();              // the blocks have started: their shared memory may be written
    const Share<T> r(a.logits, a.stride, n, a.V, rank, blocks);
    uint4 q[VPT];
    if (ONE) load_share<T, VPT>(r, r.v0, nt, q);
    if (warp == 0) load_teacher<T, TAIL>(a, n, r, rank == 0, t);
    Stat st{neg_inf(), 0.0f, 0.0f};
    if (TAIL) __syncthreads();
    for (int base = r.v0; base < r.v1; base += nt * VPT) {
        if (!ONE) load_share<T, VPT>(r, base, nt, q);
        if (TAIL) {                                // the ids' columns leave the sum: their own statistics join later
            uint32_t* words = reinterpret_cast<uint32_t*>(named);
            for (int i = threadIdx.x; i < nt * VPT / 4; i += nt) words[i] = 0;
            __syncthreads();
            for (int k = threadIdx.x; k < a.K; k += nt) {
                if (t.id[k] == NO_ID) continue;
                const int place = (int)t.id[k] + r.head, at = place / E - base;
                if (at >= 0 && at < nt * VPT && place / E < r.v1) atomicOr(&words[at >> 2], 1u << ((at & 3) * 8 + place % E));
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < VPT; ++j) {
                const uint32_t bits = named[j * nt + threadIdx.x];
                if (bits)
                    for (int i = 0; i < E; ++i)
                        if (bits >> i & 1) drop<T>(q[j], i);
            }
        }
        const Stat now = warp_stat<T, VPT, false>(q, thread_max_of<T, VPT>(q), c2);
        if (ONE) {
            st = now;
        } else {
            const float m = fmaxf(st.m, now.m);
            st = Stat{m, rescale(st, m, c2).s + rescale(now, m, c2).s, 0.0f};
            if (TAIL) __syncthreads();
        }
    }
    const int readers = a.grad ? blocks : 1;       // blocks that need the row's statistics
    if (blocks > 1) cluster_wait();
    const float4 sent = make_float4(st.m, st.s, 0.0f, 0.0f);
    if (blocks == 1) {
        if (lane == 0) part[warp] = sent;
    } else if (lane < readers) {
        remote_store(remote_addr(&part[rank * warps + warp], lane), sent);
    }
    if (TAIL && warp == 0) {
        float z[QS_MAX_TOP / 32], m = neg_inf(), s = 0.0f;
#pragma unroll
        for (int i = 0; i < QS_MAX_TOP / 32; ++i) {
            const int k = lane + 32 * i;
            z[i] = neg_inf();
            if (k >= a.K || t.id[k] == NO_ID || !r.holds((int)t.id[k])) continue;
            bool first = true;                     // an id given twice is one column
            for (int j = 0; j < k; ++j) first &= t.id[j] != t.id[k];
            if (first) z[i] = t.z[k];
            m = fmaxf(m, z[i]);
        }
        m = warp_max(m);
#pragma unroll
        for (int i = 0; i < QS_MAX_TOP / 32; ++i) s += ex2((z[i] - shift_of(m)) * c2);
        s = warp_sum(s);
        const float4 v = make_float4(m, s, 0.0f, 0.0f);
        if (blocks == 1) {
            if (lane == 0) in_part[0] = v;
        } else if (lane < readers) {
            remote_store(remote_addr(&in_part[rank], lane), v);
        }
    }
    if (blocks == 1) {
        __syncthreads();
    } else {
        cluster_arrive();
        if (!a.grad && rank != 0) return;          // nothing is written into this block's memory
        cluster_wait();
    }
    if (warp == 0) {
        Stat v = join_parts(part, warps * blocks, c2);
        float log_tail = 0.0f;
        if (TAIL) {
            const Stat in = join_parts(in_part, blocks, c2);
            const float m = fmaxf(v.m, in.m);
            const Stat x = rescale(v, m, c2), y = rescale(in, m, c2);
            const float s = x.s + y.s;
            // log of the share outside: near 1 the difference of two logs would cancel
            log_tail = v.m == neg_inf() && v.s == 0.0f ? neg_inf() : fmaf(v.m - m, a.scale, logf(v.s) - logf(s));
            if (log_tail > -0.5f) log_tail = -log1pf(y.s / x.s);
            v = Stat{m, s, 0.0f};
        }
        const bool empty = v.m == neg_inf() && v.s == 0.0f;
        const float ls = logf(v.s), lse = empty ? neg_inf() : fmaf(v.m, a.scale, ls);
        const Slope s = slope_of<TAIL>(a, n, t, lse, log_tail);
        if (lane == 0) {
            row_m = shift_of(v.m);
            row_by = empty ? 0.0f : 1.0f / v.s;
            row = s;
        }
        if (rank == 0) {
            float loss = 0.0f;
            bool beyond = false;                   // an entry where the student has no mass at all
            for (int k = lane; k < a.K; k += 32) {
                if (t.id[k] == NO_ID || t.q[k] == 0.0f) continue;
                const float lp = empty ? neg_inf() : fmaf(t.z[k] - v.m, a.scale, -ls);
                beyond |= lp == neg_inf();
                loss = fmaf(t.q[k], t.logq[k] - lp, loss);
            }
            loss = warp_sum(loss);
            // a mean of log p at a mask of the lowest value: only its rounding passes the largest number
            if (!__any_sync(~0u, beyond) && loss == -neg_inf()) loss = FLT_MAX;
            if (TAIL && t.rest != 0.0f) loss = fmaf(t.rest, logf(t.rest) - log_tail, loss);
            if (lane == 0) {
                if (a.loss) a.loss[n] = t.bad ? quiet_nan() : loss;
                if (a.lse) a.lse[n] = lse;
                if (TAIL && a.log_tail) a.log_tail[n] = log_tail;
            }
        }
    }
    if (!a.grad) return;
    __syncthreads();
    const Slope s = row;
    const float m = row_m, by = row_by;
    T* out = static_cast<T*>(a.grad) + n * a.grad_stride;
    const f2 minus = make_f2(-m, -m), c = make_f2(c2, c2);
    for (int base = r.v0; base < r.v1; base += nt * VPT) {
        if (!ONE) load_share<T, VPT>(r, base, nt, q);
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int vec = base + j * nt + (int)threadIdx.x;
            if (vec >= r.v1) continue;
            f2 d[E / 2];
#pragma unroll
            for (int i = 0; i < E / 2; ++i) d[i] = mul2(add2(Vec<T>::pair(q[j], i), minus), c);
            store_vec(r, out, vec, slope_vec<T, TAIL>(d, s, by), a.wide);
        }
    }
    __syncthreads();                               // the ids' places are written last
    for (int k = threadIdx.x; k < a.K; k += nt)
        if (t.id[k] != NO_ID && r.holds((int)t.id[k]))
            out[t.id[k]] = from_float<T>(at_id(t, a.K, k, s, ex2((t.z[k] - m) * c2) * by));
}

template <class T, int VPT, bool TAIL>
__global__ void __launch_bounds__(256) distill_grad_kernel(const RowArgs a) {
    constexpr int E = Vec<T>::E;
    __shared__ TeacherShared t;
    const int nt = blockDim.x;
    const long long n = a.row0 + blockIdx.x / a.blocks;
    const Share<T> r(a.logits, a.stride, n, a.V, (int)(blockIdx.x % a.blocks), a.blocks);
    uint4 q[VPT];
    load_share<T, VPT>(r, r.v0, nt, q);
    if (threadIdx.x < 32) load_teacher<T, TAIL>(a, n, r, false, t);
    const float lse = a.in_lse[n], log_tail = TAIL ? a.in_log_tail[n] : 0.0f;
    __syncthreads();
    const Slope s = slope_of<TAIL>(a, n, t, lse, log_tail);
    T* out = static_cast<T*>(a.grad) + n * a.grad_stride;
    const float shift = s.empty ? LOW_EXP : -lse;
    const f2 scale = make_f2(a.scale, a.scale), minus = make_f2(shift, shift), l2e = make_f2(LOG2E, LOG2E);
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int vec = r.v0 + j * nt + (int)threadIdx.x;
        if (vec >= r.v1) continue;
        f2 d[E / 2];
#pragma unroll
        for (int i = 0; i < E / 2; ++i) d[i] = mul2(fma2(Vec<T>::pair(q[j], i), scale, minus), l2e);
        store_vec(r, out, vec, slope_vec<T, TAIL>(d, s, 1.0f), a.wide);
    }
    __syncthreads();
    for (int k = threadIdx.x; k < a.K; k += nt)
        if (t.id[k] != NO_ID && r.holds((int)t.id[k]))
            out[t.id[k]] = from_float<T>(at_id(t, a.K, k, s, ex2(fmaf(t.z[k], a.scale, -lse) * LOG2E)));
}

// ------------------------------------------------------------------ launches
// Threads per block, vectors per thread and blocks per row
struct Shape { int nt, vpt, blocks; bool one; };

// most vectors of a row of V, whatever its alignment
long long most_vectors(int64_t V, int size) { return (V + 2 * (16 / size - 1)) / (16 / size); }

// A row in the registers of one cluster if it fits, else in rounds
Shape row_shape(int64_t V, int size) {
    const long long n = most_vectors(V, size);
    if (n <= 128 * 2) return Shape{128, 2, 1, true};
    if (n <= 128 * 8) return Shape{128, 8, 1, true};
    if (n <= 256 * 8 * MAX_BLOCKS) return Shape{256, 8, (int)((n + 256 * 8 - 1) / (256 * 8)), true};
    if (n <= 512 * 8 * MAX_BLOCKS) return Shape{512, 8, (int)((n + 512 * 8 - 1) / (512 * 8)), true};
    return Shape{512, 8, MAX_BLOCKS, false};
}
// independent blocks, each with one round of its row
Shape grad_shape(int64_t V, int size) {
    const long long n = most_vectors(V, size);
    if (n <= 128 * 2) return Shape{128, 2, 1, true};
    if (n <= 128 * 4) return Shape{128, 4, 1, true};
    return Shape{256, 4, (int)((n + 256 * 4 - 1) / (256 * 4)), true};
}

template <class K>
cudaError_t launch_rows(K kernel, const Shape& s, RowArgs a, bool cluster, cudaStream_t st) {
    a.blocks = s.blocks;
    const long long most = 0x7fffffffll / s.blocks;              // rows per launch
    for (a.row0 = 0; a.row0 < a.N; a.row0 += most) {
        const long long rows = a.N - a.row0 < most ? a.N - a.row0 : most;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)(rows * s.blocks));
        cfg.blockDim = dim3((unsigned)s.nt);
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

template <class T>
cudaError_t launch_token_logp(const RowArgs& a, cudaStream_t st) {
    const Shape s = row_shape(a.V, sizeof(T));
    const bool top = a.K > 0;
    if (s.vpt == 2) return launch_rows(top ? token_logp_kernel<T, 2, true, true> : token_logp_kernel<T, 2, true, false>, s, a, true, st);
    if (s.one) return launch_rows(top ? token_logp_kernel<T, 8, true, true> : token_logp_kernel<T, 8, true, false>, s, a, true, st);
    return launch_rows(top ? token_logp_kernel<T, 8, false, true> : token_logp_kernel<T, 8, false, false>, s, a, true, st);
}
template <class T>
cudaError_t launch_token_logp_grad(const RowArgs& a, cudaStream_t st) {
    const Shape s = grad_shape(a.V, sizeof(T));
    const bool ent = a.g2 != nullptr;
    if (s.vpt == 2) return launch_rows(ent ? token_logp_grad_kernel<T, 2, true> : token_logp_grad_kernel<T, 2, false>, s, a, false, st);
    return launch_rows(ent ? token_logp_grad_kernel<T, 4, true> : token_logp_grad_kernel<T, 4, false>, s, a, false, st);
}
template <class T>
cudaError_t launch_distill(const RowArgs& a, bool tail, cudaStream_t st) {
    const Shape s = row_shape(a.V, sizeof(T));
    if (s.vpt == 2) return launch_rows(tail ? distill_kernel<T, 2, true, true> : distill_kernel<T, 2, true, false>, s, a, true, st);
    if (s.one) return launch_rows(tail ? distill_kernel<T, 8, true, true> : distill_kernel<T, 8, true, false>, s, a, true, st);
    return launch_rows(tail ? distill_kernel<T, 8, false, true> : distill_kernel<T, 8, false, false>, s, a, true, st);
}
template <class T>
cudaError_t launch_distill_grad(const RowArgs& a, bool tail, cudaStream_t st) {
    const Shape s = grad_shape(a.V, sizeof(T));
    if (s.vpt == 2) return launch_rows(tail ? distill_grad_kernel<T, 2, true> : distill_grad_kernel<T, 2, false>, s, a, false, st);
    return launch_rows(tail ? distill_grad_kernel<T, 4, true> : distill_grad_kernel<T, 4, false>, s, a, false, st);
}

// how many maxima per warp bound the K-th alternative: about four for each alternative asked for
int groups_for(int K, const Shape& s) {
    const int warps = s.nt / 32 * s.blocks;
    int g = 1;
    while (g < 32 && warps * g < 4 * K && warps * g * 2 <= MAX_GROUPS) g *= 2;
    return g;
}

int status_of(cudaError_t e) {
    if (e == cudaSuccess) return QS_OK;
    cudaGetLastError();
    return QS_CUDA;
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

// the gradient may take the logits' own place, row for row; any other overlap is refused
bool overlap(const void* z, int64_t stride, const void* g, int64_t g_stride, int64_t N, int64_t V, int size) {
    const uintptr_t z0 = reinterpret_cast<uintptr_t>(z), g0 = reinterpret_cast<uintptr_t>(g);
    if (z0 == g0 && stride == g_stride) return false;
    const uintptr_t z1 = z0 + ((N - 1) * stride + V) * size, g1 = g0 + ((N - 1) * g_stride + V) * size;
    return z0 < g1 && g0 < z1;
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
    a.groups = groups_for(top, row_shape(V, size_of_type(type)));
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
    a.loss = loss; a.lse = lse; a.log_tail = log_tail; a.g1 = weight; a.g_all = weight_all;
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
