// Rows of logits as streams of 16-byte vectors.
//
// A row is cut into 16-byte vectors counted from the 16-byte boundary at or before its first element, so that
// rows of any alignment are read with wide accesses; places of the first and the last vector outside the row
// count as -inf.  A row belongs to one block or to a cluster of blocks, each with a contiguous share of the
// vectors; blocks stay and take row after row.  A Feed brings a block's shares through a ring of chunks in
// shared memory with bulk copies, several chunks ahead and across rows, so that the memory never waits
// for a row's last steps.
//
// Statistics: with y = scale * z, a part of a row is held as (m, s, u): m = max z, s = sum e and
// u = sum e * d with d = (z - m) * scale * log2(e) and e = 2^d.  Parts join exactly up to rounding; the
// difference z - m is formed first, so that a row at the type's lowest value loses nothing.
#pragma once
#include "qs_bulk.cuh"
#include "qs_lm.cuh"

namespace qs {

// ------------------------------------------------------------------ two fp32 numbers in one register pair
struct f2 { unsigned long long v; };
__device__ __forceinline__ f2 make_f2(float a, float b) {
    f2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float2 parts(f2 a) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a.v));
    return r;
}
__device__ __forceinline__ f2 add2(f2 a, f2 b) {
    f2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ f2 mul2(f2 a, f2 b) {
    f2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) {
    f2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}
__device__ __forceinline__ f2 ex2_2(f2 a) {
    const float2 p = parts(a);
    return make_f2(ex2(p.x), ex2(p.y));
}
__device__ __forceinline__ float max_nan(float a, float b) {     // NaN if either is
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
constexpr float LOW_EXP = -2000.0f;        // 2^LOW_EXP is 0; a finite stand-in for -inf where a product with 0 follows
__device__ __forceinline__ f2 floor2(f2 a) {
    const float2 p = parts(a);
    return make_f2(max_nan(p.x, LOW_EXP), max_nan(p.y, LOW_EXP));
}

// ------------------------------------------------------------------ vectors of a type
template <class T> struct Vec;
template <> struct Vec<float> {
    static constexpr int E = 4;
    static constexpr uint32_t LOWEST = 0xff800000u;              // -inf in every place of a word
    static __device__ __forceinline__ f2 pair(const uint4& q, int i) {
        return i == 0 ? make_f2(__uint_as_float(q.x), __uint_as_float(q.y)) : make_f2(__uint_as_float(q.z), __uint_as_float(q.w));
    }
    static __device__ __forceinline__ uint32_t max_word(uint32_t a, uint32_t b) {
        return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
    }
    static __device__ __forceinline__ float top(uint32_t w) { return __uint_as_float(w); }
    static __device__ __forceinline__ uint4 pack(const f2* p) {
        const float2 a = parts(p[0]), b = parts(p[1]);
        return make_uint4(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y));
    }
};
template <> struct Vec<__nv_bfloat16> {
    static constexpr int E = 8;
    static constexpr uint32_t LOWEST = 0xff80ff80u;
    static __device__ __forceinline__ f2 pair(const uint4& q, int i) {
        const uint32_t w = i == 0 ? q.x : i == 1 ? q.y : i == 2 ? q.z : q.w;
        return make_f2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    }
    static __device__ __forceinline__ uint32_t max_word(uint32_t a, uint32_t b) {
        const __nv_bfloat162 m = __hmax2(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<__nv_bfloat162*>(&b));
        return *reinterpret_cast<const uint32_t*>(&m);
    }
    static __device__ __forceinline__ float top(uint32_t w) {
        return fmaxf(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    }
    static __device__ __forceinline__ uint32_t word(f2 a) {
        const float2 p = parts(a);
        const __nv_bfloat162 h = __floats2bfloat162_rn(p.x, p.y);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    static __device__ __forceinline__ uint4 pack(const f2* p) { return make_uint4(word(p[0]), word(p[1]), word(p[2]), word(p[3])); }
};
template <> struct Vec<__half> {
    static constexpr int E = 8;
    static constexpr uint32_t LOWEST = 0xfc00fc00u;
    static __device__ __forceinline__ f2 pair(const uint4& q, int i) {
        const uint32_t w = i == 0 ? q.x : i == 1 ? q.y : i == 2 ? q.z : q.w;
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
        return make_f2(f.x, f.y);
    }
    static __device__ __forceinline__ uint32_t max_word(uint32_t a, uint32_t b) {
        const __half2 m = __hmax2(*reinterpret_cast<__half2*>(&a), *reinterpret_cast<__half2*>(&b));
        return *reinterpret_cast<const uint32_t*>(&m);
    }
    static __device__ __forceinline__ float top(uint32_t w) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
        return fmaxf(f.x, f.y);
    }
    static __device__ __forceinline__ uint32_t word(f2 a) {
        const float2 p = parts(a);
        const __half2 h = __floats2half2_rn(p.x, p.y);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    static __device__ __forceinline__ uint4 pack(const f2* p) { return make_uint4(word(p[0]), word(p[1]), word(p[2]), word(p[3])); }
};
template <class T> __device__ __forceinline__ uint4 all_lowest() {
    constexpr uint32_t w = Vec<T>::LOWEST;
    return make_uint4(w, w, w, w);
}
template <class T> __device__ __forceinline__ uint32_t max_of_words(const uint4& q) {
    return Vec<T>::max_word(Vec<T>::max_word(q.x, q.y), Vec<T>::max_word(q.z, q.w));
}
// element i of a vector replaced by -inf
template <class T> __device__ __forceinline__ void drop(uint4& q, int i) {
    uint32_t* w = &q.x;
    if (sizeof(T) == 4) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j == i) w[j] = Vec<T>::LOWEST;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j == i >> 1) w[j] = i & 1 ? (w[j] & 0xffffu) | (Vec<T>::LOWEST & 0xffff0000u) : (w[j] & 0xffff0000u) | (Vec<T>::LOWEST & 0xffffu);
    }
}

// ------------------------------------------------------------------ a row and a block's share of it
template <class T>
struct Share {
    const T* z;                // the row's first element
    int V, head;               // elements; places between the 16-byte boundary and the first
    int v0, v1;                // the block's vectors

    __device__ __forceinline__ Share(const void* logits, long long stride, long long n, long long len, int part, int nparts) {
        z = static_cast<const T*>(logits) + n * stride;
        V = (int)len;
        head = (int)((reinterpret_cast<uintptr_t>(z) & 15u) / sizeof(T));
        const int nvec = (V + head + Vec<T>::E - 1) / Vec<T>::E, per = (nvec + nparts - 1) / nparts;
        v0 = min(part * per, nvec);
        v1 = min(v0 + per, nvec);
    }
    __device__ __forceinline__ int first(int vec) const { return vec * Vec<T>::E - head; }      // element of place 0, may be < 0
    __device__ __forceinline__ bool whole(int vec) const { return first(vec) >= 0 && first(vec) <= V - Vec<T>::E; }
    __device__ __forceinline__ bool holds(int id) const {
        const int vec = (id + head) / Vec<T>::E;
        return vec >= v0 && vec < v1;
    }
};

// vectors base + j NT + t of the share, j < VPT; what is not there is -inf.  Read past the L1, evicted first:
// nothing reads them again through the caches unless the share takes more than one round
template <class T, int VPT>
__device__ __forceinline__ void load_share(const Share<T>& r, int base, int nt, uint4 (&q)[VPT]) {
    const uint4* p = reinterpret_cast<const uint4*>(r.z - r.head);
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int vec = base + j * nt + (int)threadIdx.x;
        q[j] = all_lowest<T>();
        if (vec < r.v1 && r.whole(vec)) q[j] = __ldcs(p + vec);
    }
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int vec = base + j * nt + (int)threadIdx.x;
        if (vec < r.v1 && !r.whole(vec)) {
            const int e0 = r.first(vec);
            uint32_t* w = &q[j].x;
#pragma unroll
            for (int i = 0; i < Vec<T>::E; ++i) {
                if (e0 + i < 0 || e0 + i >= r.V) continue;
                if (sizeof(T) == 4) w[i] = reinterpret_cast<const uint32_t*>(r.z)[e0 + i];
                else {
                    const uint32_t h = reinterpret_cast<const uint16_t*>(r.z)[e0 + i];
                    w[i / 2] = i & 1 ? (w[i / 2] & 0xffffu) | (h << 16) : (w[i / 2] & 0xffff0000u) | h;
                }
            }
        }
    }
}

// one vector of results; `wide`: the row's vectors have the same places in memory as the logits'
template <class T>
__device__ __forceinline__ void store_vec(const Share<T>& r, T* out, int vec, const uint4& q, bool wide) {
    if (wide && r.whole(vec)) {
        __stcs(reinterpret_cast<uint4*>(out - r.head) + vec, q);
        return;
    }
    const int e0 = r.first(vec);
    const uint32_t* w = &q.x;
#pragma unroll
    for (int i = 0; i < Vec<T>::E; ++i) {
        if (e0 + i < 0 || e0 + i >= r.V) continue;
        if (sizeof(T) == 4) reinterpret_cast<uint32_t*>(out)[e0 + i] = w[i];
        else reinterpret_cast<uint16_t*>(out)[e0 + i] = (uint16_t)(i & 1 ? w[i / 2] >> 16 : w[i / 2]);
    }
}

// ------------------------------------------------------------------ chunks of rows through shared memory
struct FeedArgs {
    int blocks;                // of a row's cluster
    int chunks;                // per share
    int chunk;                 // vectors per chunk
    int slots;                 // chunks the ring holds
    int passes;                // times a share is read
    long long clusters;        // rows row, row + clusters, .. are one cluster's
};
constexpr int MAX_SLOTS = 8;

template <class T>
struct Feed {
    const void* logits;
    long long stride, N, V;
    FeedArgs f;
    uint4* ring;
    uint64_t* full;
    int rank;
    // what is issued next (one thread), and the slot that is read next
    long long row;
    int pass, chunk, slot;
    long long issued, taken;
    int at;
    uint32_t parity;

    __device__ __forceinline__ Feed(const void* z, long long st, long long n, long long v, const FeedArgs& fa, uint4* r, uint64_t* bars, int rk,
                                    long long first)
        : logits(z), stride(st), N(n), V(v), f(fa), ring(r), full(bars), rank(rk), row(first), pass(0), chunk(0), slot(0), issued(0), taken(0), at(0), parity(0) {}

    // whether a vector's 16 bytes all belong to the tensor (its first and last vector may not)
    __device__ __forceinline__ bool inside(const Share<T>& r, int vec) const {
        const T* p = r.z + r.first(vec);
        return p >= static_cast<const T*>(logits) && p + Vec<T>::E <= static_cast<const T*>(logits) + (N - 1) * stride + V;
    }
    // the next chunk of the sequence into the next slot
    __device__ void issue() {
        if (row >= N) return;
        const Share<T> r(logits, stride, row, V, rank, f.blocks);
        const int first = r.v0 + chunk * f.chunk;
        int lo = first, hi = min(first + f.chunk, r.v1);
        if (lo < hi && !inside(r, lo)) ++lo;
        if (lo < hi && !inside(r, hi - 1)) --hi;
        const uint32_t bytes = hi > lo ? (uint32_t)(hi - lo) * 16u : 0u;
        ++issued;
        mbar_expect(&full[slot], bytes);
        if (bytes) bulk_load(ring + slot * f.chunk + (lo - first), reinterpret_cast<const uint4*>(r.z - r.head) + lo, bytes, &full[slot]);
        if (++slot == f.slots) slot = 0;
        if (++chunk < f.chunks) return;
        chunk = 0;
        if (++pass < f.passes) return;
        pass = 0;
        row += f.clusters;
    }
    __device__ __forceinline__ bool wait() const { return mbar_wait(&full[at], parity); }
    // the thread that issues, after a wait that ran out: says so, and lets the copies under way arrive (each wait is
    // bounded) before the block's memory goes to another
    __device__ void give_up(int* status) {
        flag_status(status, QS_TIMEOUT);
        for (; taken < issued; next()) wait();
    }
    __device__ __forceinline__ void next() {
        ++taken;
        if (++at == f.slots) {
            at = 0;
            parity ^= 1u;
        }
    }
    // this thread's vectors of a landed chunk; places outside the row are -inf
    template <int VPT>
    __device__ __forceinline__ void read(const Share<T>& r, int c, int slot_at, uint4 (&q)[VPT]) const {
        const int first = r.v0 + c * f.chunk, end = min(first + f.chunk, r.v1), nt = blockDim.x;
        const uint4* p = ring + slot_at * f.chunk;
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int i = j * nt + (int)threadIdx.x;
            q[j] = all_lowest<T>();
            if (i < f.chunk && first + i < end) q[j] = p[i];
        }
        // only a row's first and last vector: a look at the share's ends tells whether the chunk can hold them
        if (first != 0 && end * Vec<T>::E - r.head <= r.V) return;
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int i = j * nt + (int)threadIdx.x, vec = first + i, e0 = r.first(vec);
            if (i >= f.chunk || vec >= end || r.whole(vec)) continue;
            if (!inside(r, vec)) q[j] = edge_vec(r, vec);
            else
                for (int e = 0; e < Vec<T>::E; ++e)
                    if (e0 + e < 0 || e0 + e >= r.V) drop<T>(q[j], e);
        }
    }
    // a vector that is not whole, element by element
    static __device__ uint4 edge_vec(const Share<T>& r, int vec) {
        uint4 q = all_lowest<T>();
        uint32_t* w = &q.x;
        const int e0 = r.first(vec);
#pragma unroll
        for (int i = 0; i < Vec<T>::E; ++i) {
            if (e0 + i < 0 || e0 + i >= r.V) continue;
            if (sizeof(T) == 4) w[i] = reinterpret_cast<const uint32_t*>(r.z)[e0 + i];
            else {
                const uint32_t h = reinterpret_cast<const uint16_t*>(r.z)[e0 + i];
                w[i / 2] = i & 1 ? (w[i / 2] & 0xffffu) | (h << 16) : (w[i / 2] & 0xffff0000u) | h;
            }
        }
        return q;
    }
};

// ------------------------------------------------------------------ statistics
struct Stat { float m, s, u; };

__device__ __forceinline__ float warp_max(float v) {             // NaN is passed over
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
}
// the shift that a part's exponents take: its maximum, or 0 where everything is masked
__device__ __forceinline__ float shift_of(float m) { return m == neg_inf() ? 0.0f : m; }

template <class T, int VPT, bool ENT>
__device__ __forceinline__ void add_exps(const uint4 (&q)[VPT], float m, float c2, f2& s, f2& u) {
    const float sh = shift_of(m);
    const f2 minus = make_f2(-sh, -sh), c = make_f2(c2, c2);
#pragma unroll
    for (int j = 0; j < VPT; ++j)
#pragma unroll
        for (int i = 0; i < Vec<T>::E / 2; ++i) {
            f2 d = mul2(add2(Vec<T>::pair(q[j], i), minus), c);
            if (ENT) d = floor2(d);
            const f2 e = ex2_2(d);
            s = add2(s, e);
            if (ENT) u = fma2(e, d, u);
        }
}

// the larger maximum takes over
__device__ __forceinline__ Stat rescale(Stat a, float m, float c2) {
    if (a.m == neg_inf()) return Stat{m, a.s, a.u};              // a masked part: s = u = 0 (or NaN)
    const float d = fmaxf((a.m - m) * c2, LOW_EXP), w = ex2(d);
    return Stat{m, a.s * w, w * fmaf(a.s, d, a.u)};
}

template <class T, int VPT>
__device__ __forceinline__ float thread_max_of(const uint4 (&q)[VPT]) {
    uint32_t m = max_of_words<T>(q[0]);
#pragma unroll
    for (int j = 1; j < VPT; ++j) m = Vec<T>::max_word(m, max_of_words<T>(q[j]));
    return Vec<T>::top(m);
}

// a thread's running statistics take in the vectors of a chunk
template <class T, int VPT, bool ENT>
__device__ __forceinline__ void take_chunk(Stat& st, const uint4 (&q)[VPT], float c2) {
    const float m = fmaxf(st.m, thread_max_of<T, VPT>(q));
    if (m > st.m) st = rescale(st, m, c2);
    f2 s = make_f2(st.s, 0.0f), u = make_f2(st.u, 0.0f);
    add_exps<T, VPT, ENT>(q, m, c2, s, u);
    const float2 ps = parts(s), pu = parts(u);
    st.s = ps.x + ps.y;
    if (ENT) st.u = pu.x + pu.y;
}

// the warp's statistics from its threads'
template <bool ENT>
__device__ __forceinline__ Stat join_warp(Stat st, float c2) {
    const float m = warp_max(st.m);
    const Stat r = rescale(st, m, c2);
    return Stat{m, warp_sum(r.s), ENT ? warp_sum(r.u) : 0.0f};
}

// one warp joins n parts
__device__ __forceinline__ Stat join_parts(const float4* part, int n, float c2) {
    const int lane = threadIdx.x & 31;
    float m = neg_inf();
    for (int i = lane; i < n; i += 32) m = fmaxf(m, part[i].x);
    m = warp_max(m);
    float s = 0.0f, u = 0.0f;
    for (int i = lane; i < n; i += 32) {
        const Stat a = rescale(Stat{part[i].x, part[i].y, part[i].z}, m, c2);
        s += a.s;
        u += a.u;
    }
    return Stat{m, warp_sum(s), warp_sum(u)};
}

// ------------------------------------------------------------------ clusters
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t remote_addr(const void* p, uint32_t rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ void remote_store(uint32_t addr, float4 v) {
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
__device__ __forceinline__ void remote_store(uint32_t addr, uint32_t v) {
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
__device__ __forceinline__ void remote_store(uint32_t addr, unsigned long long v) {
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(addr), "l"(v) : "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
// ------------------------------------------------------------------ order of alternatives
// whole numbers in the order of the floats (-0 equals +0, no NaN), and with the column behind them: larger logit
// first, then lower index
__device__ __forceinline__ uint32_t key_of(float z) {
    const uint32_t b = __float_as_uint(z + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }
constexpr uint32_t KEY_LOWEST = 0x00800000u;                     // key of the lowest finite number

}  // namespace qs
