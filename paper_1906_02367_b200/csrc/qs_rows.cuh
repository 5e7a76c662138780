// Rows of logits as 16-byte vectors.
//
// A row is cut into 16-byte vectors counted from the 16-byte boundary at or before its first element, so that
// rows of any alignment are read with wide accesses; the first and the last vector may hold only some elements of
// the row and are read one by one, their other places counting as -inf.  A row belongs to one block or to a cluster
// of blocks, each with a contiguous share of the vectors.
//
// Statistics: with y = scale * z, a part of a row is held as (m, s, u): m = max z, s = sum e and u = sum e * d with
// e = 2^d and d = z c2 - fl(m c2), c2 = scale * log2(e): one multiply-add.  Where m c2 is too large for that, as in a row
// at the type's lowest value, d = (z - m) c2, so that nothing is lost.  Parts join exactly up to rounding.
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
    int w0, w1;                // those of them that are whole

    __device__ __forceinline__ Share(const void* logits, long long stride, long long n, long long len, int part, int log_parts) {
        z = static_cast<const T*>(logits) + n * stride;
        V = (int)len;
        head = (int)((reinterpret_cast<uintptr_t>(z) & 15u) / sizeof(T));
        const int nvec = (V + head + Vec<T>::E - 1) / Vec<T>::E, per = (nvec + (1 << log_parts) - 1) >> log_parts;
        v0 = min(part * per, nvec);
        v1 = min(v0 + per, nvec);
        w0 = v0 < v1 && !whole(v0) ? v0 + 1 : v0;
        w1 = w0 < v1 && !whole(v1 - 1) ? v1 - 1 : v1;
    }
    __device__ __forceinline__ const uint4* vectors() const { return reinterpret_cast<const uint4*>(z - head); }
    // a vector that is not whole, element by element
    __device__ __noinline__ uint4 edge(int vec) const {
        uint32_t w[4];
        constexpr uint32_t low = Vec<T>::LOWEST;
        const int e0 = first(vec);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = low;
#pragma unroll
        for (int i = 0; i < Vec<T>::E; ++i) {
            if (e0 + i < 0 || e0 + i >= V) continue;
            if (sizeof(T) == 4) w[i] = reinterpret_cast<const uint32_t*>(z)[e0 + i];
            else {
                const uint32_t h = reinterpret_cast<const uint16_t*>(z)[e0 + i];
                w[i / 2] = i & 1 ? (w[i / 2] & 0xffffu) | (h << 16) : (w[i / 2] & 0xffff0000u) | h;
            }
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ __forceinline__ int first(int vec) const { return vec * Vec<T>::E - head; }      // element of place 0, may be < 0
    __device__ __forceinline__ bool whole(int vec) const { return first(vec) >= 0 && first(vec) <= V - Vec<T>::E; }
    __device__ __forceinline__ bool holds(int id) const {
        const int vec = (id + head) / Vec<T>::E;
        return vec >= v0 && vec < v1;
    }
};

// vectors base + j NT + t of the share, j < VPT; what is not there is -inf.  Read past the L1, evicted first
template <class T, int VPT>
__device__ __forceinline__ void load_share(const Share<T>& r, int base, int nt, uint4 (&q)[VPT]) {
    const uint4* p = r.vectors();
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int vec = base + j * nt + (int)threadIdx.x;
        q[j] = all_lowest<T>();
        if (vec >= r.w0 && vec < r.w1) q[j] = __ldcs(p + vec);
    }
    if (r.w0 == r.v0 && r.w1 == r.v1) return;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int vec = base + j * nt + (int)threadIdx.x;
        if (vec < r.v1 && (vec < r.w0 || vec >= r.w1)) q[j] = r.edge(vec);
    }
}

// calls f(q, vec, more) for the share's vectors, nt apart from vec on: batches of VPT per thread, then the rest in one
// batch (`more`: vectors at or past w1 are no vectors, -inf), then those that are not whole.  AGAIN: some will be read again soon
struct Full { static constexpr bool value = false; };
struct Rest { static constexpr bool value = true; };
template <bool AGAIN> __device__ __forceinline__ uint4 read_vec(const uint4* p) { return AGAIN ? __ldcg(p) : __ldcs(p); }
template <class T, int VPT, bool AGAIN, class F>
__device__ __forceinline__ void each_batch(const Share<T>& r, F f) {
    const int nt = blockDim.x;
    const uint4* p = r.vectors();
    int base = r.w0;
    for (; base + nt * VPT <= r.w1; base += nt * VPT) {
        const int vec = base + (int)threadIdx.x;
        uint4 q[VPT];
#pragma unroll
        for (int j = 0; j < VPT; ++j) q[j] = read_vec<AGAIN>(p + vec + j * nt);
        f(q, vec, Full());
    }
    if (base + nt < r.w1) {
        const int vec = base + (int)threadIdx.x;
        uint4 q[VPT];
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            q[j] = all_lowest<T>();
            if (vec + j * nt < r.w1) q[j] = read_vec<AGAIN>(p + vec + j * nt);
        }
        f(q, vec, Rest());
    } else if (base + (int)threadIdx.x < r.w1) {
        const int vec = base + (int)threadIdx.x;
        uint4 q[1] = {read_vec<AGAIN>(p + vec)};
        f(q, vec, Full());
    }
    if (threadIdx.x == 0 && r.w0 > r.v0) {
        uint4 q[1] = {r.edge(r.v0)};
        f(q, r.v0, Full());
    }
    if ((int)threadIdx.x == nt - 1 && r.w1 < r.v1) {
        uint4 q[1] = {r.edge(r.w1)};
        f(q, r.w1, Full());
    }
}

// one vector of results, element by element: one that is not whole, or rows that do not lie like the logits' rows
template <class T>
__device__ __noinline__ void store_edge(const Share<T>& r, T* out, int vec, uint4 q) {
    const int e0 = r.first(vec);
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < Vec<T>::E; ++i) {
        if (e0 + i < 0 || e0 + i >= r.V) continue;
        if (sizeof(T) == 4) reinterpret_cast<uint32_t*>(out)[e0 + i] = w[i];
        else reinterpret_cast<uint16_t*>(out)[e0 + i] = (uint16_t)(i & 1 ? w[i / 2] >> 16 : w[i / 2]);
    }
}

// a whole vector of results where rows do not lie like the logits' rows
template <class T>
__device__ __forceinline__ void store_whole(T* out, const uint4& q) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 16 / (int)sizeof(T); ++i) {
        if (sizeof(T) == 4) reinterpret_cast<uint32_t*>(out)[i] = w[i];
        else reinterpret_cast<uint16_t*>(out)[i] = (uint16_t)(i & 1 ? w[i / 2] >> 16 : w[i / 2]);
    }
}

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

// A part's sums are held relative to 2^ref with ref = fl(m c2), so that an exponent is one multiply-add, d = z c2 - ref;
// that rounding of m c2 is the same in every term, and final_stat takes it out at the end.  Beyond the range in which
// ref has fractions enough (a row at a mask of the lowest value), exponents are (z - m) c2 instead.
constexpr float REF_RANGE = 65536.0f;
__device__ __forceinline__ bool in_range(float m, float c2) { return fabsf(m * c2) < REF_RANGE; }
// distance of two references: where only one of them is a rounded product, with what its rounding left out (up to 2^-9 at
// the end of the range)
__device__ __forceinline__ float left_out(float m, float c2) { return in_range(m, c2) ? fmaf(m, c2, -(m * c2)) : 0.0f; }
__device__ __forceinline__ float ref_diff(float a, float b, float c2) {
    if (in_range(a, c2) && in_range(b, c2)) return a * c2 - b * c2;
    return (a - b) * c2 - left_out(a, c2) + left_out(b, c2);
}

// The exponentials of a batch: s += sum e, u += sum e d.  FLOOR: exponents are kept finite, for a batch with places that
// hold nothing.  False where this form does not serve: u turns to NaN where a
// place is masked (0 times -inf), and m c2 may be out of range
template <class T, int VPT, bool ENT, bool FLOOR>
__device__ __forceinline__ bool add_exps(const uint4 (&q)[VPT], float ref, float c2, float& s_all, float& u_all) {
    const f2 minus = make_f2(-ref, -ref), c = make_f2(c2, c2);
    f2 s = make_f2(0.0f, 0.0f), u = s;
#pragma unroll
    for (int j = 0; j < VPT; ++j)
#pragma unroll
        for (int i = 0; i < Vec<T>::E / 2; ++i) {
            f2 d = fma2(Vec<T>::pair(q[j], i), c, minus);
            if (FLOOR) d = floor2(d);
            const f2 e = ex2_2(d);
            s = add2(s, e);
            if (ENT) u = fma2(e, d, u);
        }
    const float2 ps = parts(s), pu = parts(u);
    const float sum_d = pu.x + pu.y;
    if (!(fabsf(ref) < REF_RANGE) || (ENT && !(sum_d == sum_d))) return false;
    s_all += ps.x + ps.y;
    if (ENT) u_all += sum_d;
    return true;
}
// the same for one vector in a form that serves always: masked places and overflow made finite
template <class T>
__device__ __noinline__ float2 add_exps_exact(uint4 q, float m, float c2) {
    const bool far = !in_range(m, c2);
    const float ref = m * c2;
    const f2 minus = far ? make_f2(-m, -m) : make_f2(-ref, -ref), c = make_f2(c2, c2);
    f2 s = make_f2(0.0f, 0.0f), u = s;
#pragma unroll
    for (int i = 0; i < Vec<T>::E / 2; ++i) {
        const f2 z = Vec<T>::pair(q, i), d = floor2(far ? mul2(add2(z, minus), c) : fma2(z, c, minus)), e = ex2_2(d);
        s = add2(s, e);
        u = fma2(e, d, u);
    }
    const float2 ps = parts(s), pu = parts(u);
    return make_float2(ps.x + ps.y, pu.x + pu.y);
}

// the larger maximum takes over
__device__ __forceinline__ Stat rescale(Stat a, float m, float c2) {
    if (a.m == neg_inf()) return Stat{m, a.s, a.u};              // a masked part: s = u = 0 (or NaN)
    const float d = fmaxf(ref_diff(a.m, m, c2), LOW_EXP), w = ex2(d);
    return Stat{m, a.s * w, w * fmaf(a.s, d, a.u)};
}
// sums relative to the maximum itself
__device__ __forceinline__ Stat final_stat(Stat a, float c2) {
    if (a.m == neg_inf() || !in_range(a.m, c2)) return a;
    const float delta = fmaf(a.m, c2, -(a.m * c2)), w = ex2(-delta), s = a.s * w;
    return Stat{a.m, s, fmaf(-delta, s, a.u * w)};
}

// whether a row has no live column at all (a NaN is one)
__device__ __forceinline__ bool is_empty(Stat a) { return a.m == neg_inf() && a.s == 0.0f; }
// lse = m scale + ls of final statistics.  -inf says that the row is empty: one that merely passes the largest number (a
// row at the type's lowest value, a scale above 1) is that number
__device__ __forceinline__ float lse_of(Stat a, float scale, float ls) {
    const float lse = fmaf(a.m, scale, ls);
    return is_empty(a) ? neg_inf() : isinf(lse) ? copysignf(FLT_MAX, lse) : lse;
}

template <class T, int VPT>
__device__ __forceinline__ float thread_max_of(const uint4 (&q)[VPT]) {
    uint32_t m = max_of_words<T>(q[0]);
#pragma unroll
    for (int j = 1; j < VPT; ++j) m = Vec<T>::max_word(m, max_of_words<T>(q[j]));
    return Vec<T>::top(m);
}

// A thread's running statistics take in a batch of vectors, of which m is the largest value.  Their reference st.m
// moves when the exponents would pass 2^REACH, so that most batches need no new scale; the reach is small because the
// entropy's u loses REACH units in the last place when it moves on to the row's maximum at the end
constexpr float REACH = 3.0f;
template <class T, int VPT, bool ENT, bool FLOOR>
__device__ __forceinline__ void take(Stat& st, const uint4 (&q)[VPT], float m, float c2) {
    if (!((m - st.m) * c2 <= REACH) && m > st.m) st = rescale(st, m, c2);
    const float at = shift_of(st.m);
    if (add_exps<T, VPT, ENT, FLOOR && ENT>(q, at * c2, c2, st.s, st.u)) return;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const float2 x = add_exps_exact<T>(q[j], at, c2);
        st.s += x.x;
        if (ENT) st.u += x.y;
    }
}

// the warp's statistics from its threads'; `largest` is the thread's largest value
template <bool ENT>
__device__ __forceinline__ Stat join_warp(Stat st, float largest, float c2) {
    const float m = warp_max(largest);
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
// stores that count at the receiving block's barrier: its phase ends when all the bytes it expects are there
__device__ __forceinline__ void send(uint32_t addr, float4 v, uint32_t bar) {
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(addr), "f"(v.x), "f"(v.y),
                 "f"(v.z), "f"(v.w), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void send(uint32_t addr, float v, uint32_t bar) {
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.f32 [%0], %1, [%2];" ::"r"(addr), "f"(v), "r"(bar) : "memory");
}
__device__ __forceinline__ void fence_barrier_init() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
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
