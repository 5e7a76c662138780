// Matrix products of a network's layers, with bias, activation and residual in the same kernel, and their gradients:
//
//   z = x w^T (+ bias);  out = act(z) (+ residual);  dx = dz w;  dw = dz^T x;  dz = g act'(z)
//
// All three products are one kernel's: D[m, n] = sum over k of A[m, k] B[n, k], per worker, where an operand lies along k
// or across it (w in dx, both in dw): the tensor maps and the matrix unit's descriptors take either.
#include <algorithm>
#include <cstdlib>

#include "qs_parts.cuh"

namespace qs {
namespace {

typedef __nv_bfloat16 bf16;

// ------------------------------------------------------------------ what follows the sums
struct Finish {
    long long M, N;                                  // of one worker
    const void* bias; int bias_type; long long bias_worker;
    int act;
    const void* res; long long res_stride;           // rows of all workers, one after the other
    void* pre; long long pre_stride;
    void* out; int type; long long out_stride, out_worker;
    const float* a_scale; const float* b_scale;      // per row and per column, of 8-bit operands
    long long b_scale_worker;
    int accumulate;                                  // added to what `out` holds
    int vec;                                         // rows of 16-byte vectors all around
};

__device__ __forceinline__ float rcp(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float logistic(float z) { return rcp(1.0f + ex2(-LOG2E * z)); }
template <int N>
__device__ __forceinline__ float polynomial(const float (&c)[N], float x) {
    float p = c[N - 1];
#pragma unroll
    for (int i = N - 2; i >= 0; --i) p = __fmaf_rn(p, x, c[i]);
    return p;
}
// Phi(z) and e^(-z^2 / 2), for a = |z|: Phi(-a) = t P(t) e^(-a^2 / 2) with t = 1 / (1 + c a), relative to the value however small it is; the coefficients
// are least-maximum fits made for this.  For results in 16 bits nine for all a >= 0, within 1.3e-7.  FP32, for results in fp32: nine for a >= 1,
// within 2.1e-8, and 1/2 + z Q(z^2) below, within 1e-9 of it.  The exponent's rounding is 0.6 a^2 2^-23 of the value.  (us in 16 bits, fp32, and
// with CUDA's normcdff: 8 x 4096 x 4096 x 1024 in bf16 258, into fp32 396, 750; gradient of 16384 x 4096 in fp32 136, 217)
struct Normal { float phi, density; };
template <bool FP32>
__device__ __forceinline__ Normal normal(float z) {
    const float a = fabsf(z), s = a * a, e = ex2(-0.72134752f * s);                  // -log2(e) / 2
    if (FP32) {
        constexpr float P[9] = {0.119682692f,    0.119682021f, 0.108939894f,  0.0868976414f, 0.0618129857f,
                                0.00897625927f, 0.0464471877f, -0.080664888f, 0.0282582119f};
        constexpr float Q[6] = {0.398942292f, -0.0664903522f, 0.00997328479f, -0.00118621089f, 0.000113337694f, -7.58989427e-06f};
        const float t = rcp(__fmaf_rn(0.3f, a, 1.0f)), tail = polynomial(P, t) * t * e, middle = __fmaf_rn(z, polynomial(Q, s), 0.5f);
        return {a < 1.0f ? middle : z < 0.0f ? tail : 1.0f - tail, e};
    }
    constexpr float P[9] = {0.112837933f,    0.112834752f, 0.103922084f,  0.0842660293f, 0.0707334131f,
                            -0.0028393846f, 0.0845832974f, -0.0914751291f, 0.0251370706f};
    const float t = rcp(__fmaf_rn(0.28284273f, a, 1.0f)), tail = polynomial(P, t) * t * e;
    return {z < 0.0f ? tail : 1.0f - tail, e};
}
template <int ACT, bool FP32>
__device__ __forceinline__ float activate(float z) {
    if (ACT == QS_ACT_RELU) return z < 0.0f ? 0.0f : z;
    if (ACT == QS_ACT_SILU) return z * logistic(z);
    if (ACT == QS_ACT_GELU) return z * normal<FP32>(z).phi;
    return z;
}
template <int ACT, bool FP32>
__device__ __forceinline__ float slope(float z) {
    if (ACT == QS_ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
    if (ACT == QS_ACT_SILU) {
        const float p = logistic(z);
        return p * __fmaf_rn(z, 1.0f - p, 1.0f);
    }
    if (ACT == QS_ACT_GELU) {
        const Normal n = normal<FP32>(z);
        return __fmaf_rn(z * 0.39894228f, n.density, n.phi);
    }
    return 1.0f;
}

__device__ __forceinline__ float element(const void* p, int type, long long i) {
    return type == QS_F32 ? static_cast<const float*>(p)[i] : type == QS_BF16 ? to_float(static_cast<const bf16*>(p)[i]) : to_float(static_cast<const __half*>(p)[i]);
}

// V columns from n on of a row: what belongs to the columns
template <int V> struct Columns { float bias[V], scale[V]; };
template <int V>
__device__ __forceinline__ void load_columns(const Finish& f, int r, long long n, Columns<V>& c) {
#pragma unroll
    for (int i = 0; i < V; ++i) c.bias[i] = 0.0f, c.scale[i] = 1.0f;
    if (f.bias) {
        const long long at = r * f.bias_worker + n;
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (n + i < f.N) c.bias[i] = element(f.bias, f.bias_type, at + i);
    }
    if (f.b_scale)
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (n + i < f.N) c.scale[i] = f.b_scale[r * f.b_scale_worker + n + i];
}
// Sums of row m (of worker r), columns n on, on their way to the result.  ADD: to what the result holds; RAW: nothing but that
enum { ADD = 1, RAW = 2 };
template <int ACT, int V, class T>
__device__ __forceinline__ void finish(const Finish& f, int r, long long m, long long n, float (&v)[V], const Columns<V>& c, int how) {
    const long long row = r * f.M + m;
    T* out = static_cast<T*>(f.out) + r * f.out_worker + m * f.out_stride + n;
    float t[V];
    if (how & ADD) {
        load_vec<V>(t, out);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] += t[i];
    }
    if (!(how & RAW)) {
        if (f.a_scale) {
            const float s = f.a_scale[row];
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = v[i] * s * c.scale[i];
        }
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] += c.bias[i];
        if (f.pre) store_vec<V>(static_cast<T*>(f.pre) + row * f.pre_stride + n, v);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = activate<ACT, sizeof(T) == 4>(v[i]);
        if (f.res) {
            load_vec<V>(t, static_cast<const T*>(f.res) + row * f.res_stride + n);
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] += t[i];
        }
    }
    store_vec<V>(out, v);
}
template <int V, class T>
__device__ __forceinline__ void finish_as(const Finish& f, int r, long long m, long long n, float (&v)[V], const Columns<V>& c, int how) {
    switch (f.act) {
    case QS_ACT_RELU: return finish<QS_ACT_RELU, V, T>(f, r, m, n, v, c, how);
    case QS_ACT_SILU: return finish<QS_ACT_SILU, V, T>(f, r, m, n, v, c, how);
    case QS_ACT_GELU: return finish<QS_ACT_GELU, V, T>(f, r, m, n, v, c, how);
    default: return finish<QS_ACT_NONE, V, T>(f, r, m, n, v, c, how);
    }
}
template <int V>
__device__ __forceinline__ void finish_any(const Finish& f, int r, long long m, long long n, float (&v)[V], const Columns<V>& c, int how) {
    if (f.type == QS_F32) finish_as<V, float>(f, r, m, n, v, c, how);
    else if (f.type == QS_BF16) finish_as<V, bf16>(f, r, m, n, v, c, how);
    else finish_as<V, __half>(f, r, m, n, v, c, how);
}

// The same for 32 x 32 sums, one row per lane, on their way to a tile of shared memory that a copy takes to the result (and
// another to `pre`): rows of 128 bytes, pieces of 16 bytes at place piece ^ (row & 7).
template <class T> struct Raw32 { uint4 a[2 * sizeof(T)]; };                 // 32 elements
// (whole pieces alone: where there is anything to read, rows end with one.  FRESH: what this kernel's copies wrote is not
// looked for in the L1)
template <class T, bool FRESH>
__device__ __forceinline__ void load_raw(Raw32<T>& q, const T* p, int left) {
    constexpr int W = 16 / sizeof(T);
#pragma unroll
    for (int k = 0; k < 2 * (int)sizeof(T); ++k) {
        q.a[k] = make_uint4(0, 0, 0, 0);
        const uint4* at = reinterpret_cast<const uint4*>(p) + k;
        if (k * W < left) q.a[k] = FRESH ? __ldcg(at) : *at;
    }
}
template <class T>
__device__ __forceinline__ void add_raw(float (&v)[32], const Raw32<T>& q) {
    constexpr int W = 16 / sizeof(T);
#pragma unroll
    for (int k = 0; k < 2 * (int)sizeof(T); ++k) {
        float t[W];
        unpack<T, W>(t, *reinterpret_cast<const Pack<T, W>*>(&q.a[k]));
#pragma unroll
        for (int i = 0; i < W; ++i) v[k * W + i] += t[i];
    }
}
__device__ __forceinline__ void store_shared(uint32_t at, uint4 v) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ float4 load_shared(uint32_t at) {
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
    return v;
}
template <class T>
__device__ __forceinline__ void put_row(uint32_t row, int lane, int first, const float (&v)[32]) {
    constexpr int W = 16 / sizeof(T);
#pragma unroll
    for (int k = 0; k < 2 * (int)sizeof(T); ++k) {
        const Pack<T, W> q = pack_of<T, W>(v + k * W);
        store_shared(row + (((first + k) ^ (lane & 7)) << 4), *reinterpret_cast<const uint4*>(&q));
    }
}
// What there is to do, in one register: looking at the arguments for each of 32 columns cost more than the arithmetic
enum { SCALED = 4, BIASED = 8, KEPT = 16, ADDED_RES = 32 };
__device__ __forceinline__ int todo_of(const Finish& f) {
    return (f.a_scale ? SCALED : 0) | (f.bias ? BIASED : 0) | (f.pre ? KEPT : 0) | (f.res ? ADDED_RES : 0);
}
// `first`: the row's pieces in front of these; bias, scale: of the 32 columns; left: columns that there are
template <int ACT, class T>
__device__ __forceinline__ void finish_row(int todo, float (&v)[32], const T* out, const T* res, int left, float a_scale, uint32_t bias, uint32_t scale,
                                           uint32_t out_tile, uint32_t pre_tile, int first, int lane) {
    Raw32<T> q;
    if (todo & ADD) {
        load_raw<T, true>(q, out, left);
        add_raw<T>(v, q);
    }
    if (!(todo & RAW)) {
        if (todo & ADDED_RES) load_raw<T, false>(q, res, left);
        if (todo & SCALED) {
#pragma unroll
            for (int i = 0; i < 32; i += 4) {
                const float4 s = load_shared(scale + 4 * i);
                v[i] = v[i] * a_scale * s.x, v[i + 1] = v[i + 1] * a_scale * s.y, v[i + 2] = v[i + 2] * a_scale * s.z, v[i + 3] = v[i + 3] * a_scale * s.w;
            }
        }
        if (todo & BIASED) {
#pragma unroll
            for (int i = 0; i < 32; i += 4) {
                const float4 b = load_shared(bias + 4 * i);
                v[i] += b.x, v[i + 1] += b.y, v[i + 2] += b.z, v[i + 3] += b.w;
            }
        }
        if (todo & KEPT) put_row<T>(pre_tile, lane, first, v);
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = activate<ACT, sizeof(T) == 4>(v[i]);
        if (todo & ADDED_RES) add_raw<T>(v, q);
    }
    put_row<T>(out_tile, lane, first, v);
}
// Where rows are not on 16-byte boundaries: the sums in shared memory (row i's group j of four columns at place j ^ (i & 7)), a
// column per lane
template <int ACT, class T>
__device__ __forceinline__ void finish_columns(const Finish& f, int r, long long m0, long long n, int rows, const float* pass, int lane, int how) {
    const long long row = r * f.M + m0;
    T* out = static_cast<T*>(f.out) + r * f.out_worker + m0 * f.out_stride + n;
    const T* res = static_cast<const T*>(f.res) + row * f.res_stride + n;
    T* pre = static_cast<T*>(f.pre) + row * f.pre_stride + n;
    Columns<1> c;
    load_columns(f, r, n, c);
#pragma unroll 1
    for (int i = 0; i < rows; i += 8) {              // (eight rows under way together)
        float v[8];
#pragma unroll
        for (int p = 0; p < 8; ++p) v[p] = pass[(i + p) * 32 + ((lane >> 2) ^ p) * 4 + (lane & 3)];
        if (how & ADD) {
#pragma unroll
            for (int p = 0; p < 8; ++p)
                if (i + p < rows) v[p] += to_float(out[p * f.out_stride]);
        }
        if (!(how & RAW)) {
            if (f.a_scale) {
#pragma unroll
                for (int p = 0; p < 8; ++p)
                    if (i + p < rows) v[p] = v[p] * f.a_scale[row + i + p] * c.scale[0];
            }
#pragma unroll
            for (int p = 0; p < 8; ++p) v[p] += c.bias[0];
            if (f.pre) {
#pragma unroll
                for (int p = 0; p < 8; ++p)
                    if (i + p < rows) pre[p * f.pre_stride] = from_float<T>(v[p]);
                pre += 8 * f.pre_stride;
            }
#pragma unroll
            for (int p = 0; p < 8; ++p) v[p] = activate<ACT, sizeof(T) == 4>(v[p]);
            if (f.res) {
#pragma unroll
                for (int p = 0; p < 8; ++p)
                    if (i + p < rows) v[p] += to_float(res[p * f.res_stride]);
                res += 8 * f.res_stride;
            }
        }
#pragma unroll
        for (int p = 0; p < 8; ++p)
            if (i + p < rows) out[p * f.out_stride] = from_float<T>(v[p]);
        out += 8 * f.out_stride;
    }
}

// ------------------------------------------------------------------ operands for the matrix unit
// Operands that the tensor maps cannot take as they lie (another type, rows off the 16-byte boundary) are laid out in the
// workspace: fp32 rounded to the other operand's 16 bits, or taken apart into three bf16 parts x = x0 + x1 + x2, each what
// the ones before left, rounded: 24 bits in all, exactly.
// 16 bytes from any address, of which the first and the last are there: by the aligned pieces that hold them
__device__ __forceinline__ uint4 bytes_at(uintptr_t at) {
    const uint4* q = reinterpret_cast<const uint4*>(at & ~(uintptr_t)15);
    const uint4 a = q[0];
    if ((at & 15) == 0) return a;
    const uint4 b = q[1];
    uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    if (at & 8)
#pragma unroll
        for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
    if (at & 4)
#pragma unroll
        for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
    const uint32_t s = (uint32_t)(at & 3) * 8;
    return make_uint4(__funnelshift_r(w[0], w[1], s), __funnelshift_r(w[1], w[2], s), __funnelshift_r(w[2], w[3], s), __funnelshift_r(w[3], w[4], s));
}
struct LayArgs {
    const void* src; int src_type; long long src_stride, src_worker;
    void* dst; int dst_type, planes; long long ld;   // (workers, planes, rows, ld)
    long long rows, cols; int workers;
};
// Eight numbers rounded to bf16 (middles away from zero), as pairs; v keeps the rest (exactly).  In the first part, where one of them would be
// past the largest number, they are cut off instead, and infinities are NaN, as what they enter is: their rest has no value.  (By the
// conversion's own rounding 16 x 8192 x 8192 takes 240 us, 210 so; 189 with all cut off)
template <bool FIRST>
__device__ __forceinline__ uint4 parts_of(float (&v)[8]) {
    uint32_t u[8], most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        u[i] = __float_as_uint(v[i]);
        if (FIRST) most = max(most, u[i] & 0x7fffffffu);
    }
    if (FIRST && most >= 0x7f7f8000u) {
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = (u[i] & 0x7fffffffu) < 0x7f800000u ? u[i] & 0xffff0000u : 0x7fff0000u;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = (u[i] + 0x8000u) & 0xffff0000u;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] -= __uint_as_float(u[i]);
    return make_uint4(__byte_perm(u[0], u[1], 0x7632), __byte_perm(u[2], u[3], 0x7632), __byte_perm(u[4], u[5], 0x7632), __byte_perm(u[6], u[7], 0x7632));
}

// parts of the operands whose products are added, the small ones first: x1 y2, x2 y1 and x2 y2 are left out, 2^-26 of a product: a rest is
// 2^-9 of what it is left from at most, and of either sign.  (Cut off instead of rounded, 2^-8 and of one sign: sums of the worst numbers were
// 5e-7 off)
__device__ __forceinline__ int part_a(int pairs, int p) { return pairs == 1 ? 0 : (0x010120 >> (4 * p)) & 15; }
__device__ __forceinline__ int part_b(int pairs, int p) { return pairs == 1 ? 0 : (0x001102 >> (4 * p)) & 15; }

struct LayBoth { LayArgs side[2]; };
__global__ void __launch_bounds__(256) lay_kernel(const LayBoth both) {
    const LayArgs& a = both.side[blockIdx.z];
    if (blockIdx.y >= a.workers) return;
    const int size = a.dst_type == QS_E4M3 ? 1 : 2, n = 16 / size, from_size = a.src_type == QS_F32 ? 4 : size;      // n elements a unit
    const long long units = a.ld / n, r = blockIdx.y, items = a.rows * units;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < items; i += (long long)gridDim.x * 256) {
        const long long row = i / units, c = (i - row * units) * n, from = r * a.src_worker + row * a.src_stride + c;
        const uintptr_t at = reinterpret_cast<uintptr_t>(a.src) + (uintptr_t)from * from_size;
        const bool whole = c + n <= a.cols;
        if (from_size != 4) {                        // as they are
            uint4 q = make_uint4(0, 0, 0, 0);
            if (whole) {
                q = bytes_at(at);
            } else {
                uint32_t w[4] = {};
                const int left = (int)max(0ll, a.cols - c) * size;
#pragma unroll
                for (int b = 0; b < 16; ++b)
                    if (b < left) w[b / 4] |= (uint32_t)reinterpret_cast<const uint8_t*>(at)[b] << (b % 4 * 8);
                q = make_uint4(w[0], w[1], w[2], w[3]);
            }
            *reinterpret_cast<uint4*>(static_cast<uint8_t*>(a.dst) + ((r * a.rows + row) * a.ld + c) * size) = q;
            continue;
        }
        float v[8];
        if (whole) {
            const uint4 q0 = bytes_at(at), q1 = bytes_at(at + 16);
            const uint32_t w[8] = {q0.x, q0.y, q0.z, q0.w, q1.x, q1.y, q1.z, q1.w};
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(w[j]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = c + j < a.cols ? static_cast<const float*>(a.src)[from + j] : 0.0f;
        }
        if (a.dst_type == QS_F16) {
            store_vec<8>(static_cast<__half*>(a.dst) + (r * a.rows + row) * a.ld + c, v);
        } else {
            if (a.planes == 1) store_vec<8>(static_cast<bf16*>(a.dst) + (r * a.rows + row) * a.ld + c, v);
            else
#pragma unroll
                for (int p = 0; p < 3; ++p)
                    *reinterpret_cast<uint4*>(static_cast<bf16*>(a.dst) + ((r * 3 + p) * a.rows + row) * a.ld + c) = p ? parts_of<false>(v) : parts_of<true>(v);
        }
    }
}

// ------------------------------------------------------------------ the product
constexpr int TILE_M = 128;                          // rows of a block's part of a tile: the lanes of tensor memory
constexpr int STAGES = 5;
constexpr int GEMM_THREADS = 384;                    // warps: copies, products, tensor memory, (none), eight that finish
// The matrix unit cuts what lies below the last bits of a sum at every addition, always towards zero: less than 2^-23 of the sum so
// far for every 8 elements of 16 bits or 16 of 8.  Of the result that is, in the mean, for sums of mixed signs 8.6e-7 after 1024
// elements of 16 bits, 7.9e-6 after 8192, 6.6e-5 after 65536; of one sign in bf16 2.2e-6, 3.5e-5, 3.9e-4, in fp16 6.1e-6, 5.3e-5, 4.3e-4, in
// e4m3 1.7e-7, 3.5e-6, 5.7e-5.  Sums are therefore added up, rounded to nearest, from those over this many blocks of 128 bytes:
// results in fp32 from 1024 elements of 16 bits (weights' gradient of 8 x 4096 rows, 4096 x 1024: 205 us with 64 blocks, 218 with
// 32; 240 with 16); those in 16 bits, which are rounded by 2^-9 (bf16) or 2^-12 (fp16) of their size at most, from 16384 and 8192: the cut is a
// quarter of that at most.  (4096 x 4096 x 32768 in bf16 5 to 15 % longer than in one sum, 4096 x 4096 x 16384 in fp16 10 to 20 %)
constexpr int CHUNK_BLOCKS = 16, CHUNK_BF16 = 256, CHUNK_F16 = 128;
constexpr int PASS_BYTES = 8 * 2 * 4096;             // two tiles of 32 rows of 128 bytes on their way out, per finishing warp

struct GemmArgs {
    int R;
    long long M, N;
    int tiles_m, tiles_n, splits, units;             // units of work: workers x splits x tiles
    int k_blocks, k_step, pairs;                     // blocks of 128 bytes along k; pairs of parts
    int per_split, more;                             // blocks along k of a split; the first `more` take one more
    int chunk;                                       // blocks along k that are summed by the matrix unit before they are added up
    int a_across, b_across;                          // operand lies across k
    int a_worker, b_worker;                          // 0: one operand for all workers
    int eight;                                       // 8-bit operands
    uint32_t idesc;
    int columns;                                     // there is a bias or a scale of the columns
    int l2_adds;                                     // nothing but sums, in fp32: the copies out add what is to be added
    unsigned long long limit;
    int* status;
    Finish f;
};

struct Unit { int r, split, tm, tn, kb0, kb1; };      // blocks [kb0, kb1) along k of one tile
__device__ __forceinline__ Unit unit_of(const GemmArgs& g, int u) {
    Unit t;
    const unsigned tiles = g.tiles_m * g.tiles_n, n = g.tiles_n;
    const unsigned rs = (unsigned)u / tiles;
    unsigned i = (unsigned)u - rs * tiles;
    t.r = rs, t.split = 0;
    if (g.splits > 1) t.r = rs / (unsigned)g.splits, t.split = rs - t.r * g.splits;
    // bands of eight tile rows, so that the blocks at work share operands in the L2
    const unsigned band = i / (8 * n), rows = min(8u, g.tiles_m - band * 8);
    i -= band * 8 * n;
    t.tn = rows == 8 ? i >> 3 : i / rows;
    t.tm = band * 8 + (i - t.tn * rows);
    // the first `more` splits take one block along k more than the others
    t.kb0 = t.split * g.per_split + min(t.split, g.more);
    t.kb1 = t.kb0 + g.per_split + (t.split < g.more);
    return t;
}

template <int CG, int BN> __host__ __device__ constexpr int stage_bytes() { return TILE_M * 128 + BN / CG * 128; }
struct Small {                                       // beside the ring and the tiles on their way out
    float bias[256], scale[256];                     // of the columns at hand, per half of the finishing warps
    uint64_t full[STAGES], empty[STAGES], acc_full[2], acc_empty[2], drained;
    uint32_t tmem_at;
};
template <int CG, int BN> __host__ __device__ constexpr int gemm_smem() { return STAGES * stage_bytes<CG, BN>() + PASS_BYTES + (int)sizeof(Small); }

// A tile of TILE_M CG x BN per cluster of CG blocks.  One warp per block keeps a ring of STAGES tiles of both operands filling; one
// of the leading block issues the products into one of two accumulators; eight warps per block take the other one out, a row
// per lane, finish it and leave it in tiles of shared memory that bulk copies take to the result (rows off the 16-byte boundary
// are turned there and stored a column per lane).  Bound by the products for long sums: 516 of 512 cycles per slot in bf16 and in
// e4m3 (8192 x 8192 x 8192 in short loops: 725 us, 1516 TFLOP/s under the power limit; e4m3 365 us, 3014.  8192 x 16384 x 4096 in e4m3 takes 400
// us so, 473 to 496 in a loop of seconds); for short ones by the finishing warps' instructions (8 x 4096 x 4096 x 1024: 203 us, 222 with silu, 248 with the saved values too).
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, unsigned long long limit) {
    return __all_sync(~0u, mbar_wait_asleep(bar, parity, limit));                // (the lanes give up together)
}
template <int CG, int BN, class T>
__global__ void __launch_bounds__(GEMM_THREADS, 1)
gemm_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_out,
            const __grid_constant__ CUtensorMap map_pre, const __grid_constant__ GemmArgs g) {
    extern __shared__ __align__(1024) uint8_t ring[];
    constexpr int A_BYTES = TILE_M * 128, B_ROWS = BN / CG, STAGE = stage_bytes<CG, BN>();
    // Tiles of 64 columns: the two halves of the finishing warps take units in turn, else half of the columns of each
    constexpr bool TURNS = BN == 64;
    Small& small = *reinterpret_cast<Small*>(ring + STAGES * STAGE + PASS_BYTES);
    uint64_t *full = small.full, *empty = small.empty, *acc_full = small.acc_full, *acc_empty = small.acc_empty;
    // (tiles are swizzled by their addresses: off the 1024-byte boundary nothing is begun, as with a wait that runs out at once)
    const unsigned long long limit = smem_addr(ring) & 1023 ? 0 : g.limit;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = CG == 2 ? cluster_rank() : 0;
    const int cluster = blockIdx.x / CG, clusters = gridDim.x / CG;

    if (threadIdx.x == 0) {
        for (int i = 0; i < STAGES; ++i) mbar_init(&full[i], 1), mbar_init(&empty[i], 1);
        for (int i = 0; i < 2; ++i) mbar_init(&acc_full[i], 1), mbar_init(&acc_empty[i], (TURNS ? 4 : 8) * CG);
        mbar_init(&small.drained, 1);
        fence_barrier_init();
    }
    if (warp == 2) tmem_alloc<CG>(&small.tmem_at, 2 * BN);
    tc_fence_before();
    if (CG == 2) cluster_sync();
    else __syncthreads();
    tc_fence_after();
    const uint32_t tmem = small.tmem_at;
    after_launch();

    // (Both of these warps run as one: a single lane's loop around the products left the matrix unit idle for 300 of 810 cycles
    // per slot, 8192 x 8192 x 8192 in bf16 took 870 us)
    if (warp == 0) {
        const bool me = elected();
        int slot = 0, count = 0;
        uint32_t phase = 1;                          // (of a new barrier: the phase before counts as over)
        bool fine = limit != 0;
        for (int u = cluster; u < g.units && fine; u += clusters) {
            const Unit t = unit_of(g, u);
            const int m0 = (t.tm * CG + (int)rank) * TILE_M, n0 = t.tn * BN + (int)rank * B_ROWS, ra = t.r * g.a_worker, rb = t.r * g.b_worker;
            for (int kb0 = t.kb0; kb0 < t.kb1 && fine; kb0 += g.chunk) {
                const int kb1 = min(t.kb1, kb0 + g.chunk);
                for (int p = 0; p < g.pairs && fine; ++p) {
                    const int pa = part_a(g.pairs, p), pb = part_b(g.pairs, p);
                    for (int kb = kb0; kb < kb1; ++kb) {
                        if (!(fine = warp_wait(&empty[slot], phase, limit))) break;
                        if (me) {
                            const int k0 = kb * g.k_step;
                            if (rank == 0) mbar_expect(&full[slot], STAGE * CG);
                            const uint32_t bar = CG == 2 ? in_block(smem_addr(&full[slot]), 0) : smem_addr(&full[slot]);
                            const uint32_t a = smem_addr(ring + slot * STAGE), b = a + A_BYTES;
                            if (g.a_across) {
                                for (int j = 0; j < TILE_M / 64; ++j) tile_load<CG>(a + j * 8192, &map_a, bar, m0 + j * 64, k0, pa, ra);
                            } else {
                                tile_load<CG>(a, &map_a, bar, k0, m0, pa, ra);
                            }
                            if (g.b_across) {
                                for (int j = 0; j < B_ROWS / 64; ++j) tile_load<CG>(b + j * 8192, &map_b, bar, n0 + j * 64, k0, pb, rb);
                            } else {
                                tile_load<CG>(b, &map_b, bar, k0, n0, pb, rb);
                            }
                        }
                        __syncwarp();
                        ++count;
                        if (++slot == STAGES) slot = 0, phase ^= 1;
                    }
                }
            }
        }
        if (limit == 0) count = 0;
        if (fine) {
            // the last products' arrivals, which may come from the other block, are in before this one ends
            for (int i = 0; i < STAGES; ++i) {
                if (count >= STAGES || slot < count) warp_wait(&empty[slot], phase, limit);
                if (++slot == STAGES) slot = 0, phase ^= 1;
            }
        } else if (count > 0 && rank == 0) {
            // after a wait that ran out: the copies under way (of both blocks: they count here) land before the memory is given up
            for (int i = max(0, count - STAGES); i < count; ++i) warp_wait(&full[i % STAGES], (i / STAGES) & 1, WAIT_LIMIT_NS);
        } else if (count > 0) {
            // (the second block's count at the first: it cannot look, and gives them far more time than a copy takes)
            const unsigned long long t0 = global_ns();
            while (global_ns() - t0 < 10000000ull) {}
        }
    } else if (warp == 1) {
        if (rank == 0 && limit != 0) {
            const bool me = elected();
            int n = 0, slot = 0;
            uint32_t phase = 0;
            bool fine = true;
            const uint64_t step_a = (g.a_across ? 2048 : 32) >> 4, step_b = (g.b_across ? 2048 : 32) >> 4;   // 16 (8 bits: 32) along k
            const uint64_t first = tile_descriptor(smem_addr(ring), 8192);
            for (int u = cluster; u < g.units && fine; u += clusters) {
                const Unit t = unit_of(g, u);
                for (int kb0 = t.kb0; kb0 < t.kb1 && fine; kb0 += g.chunk, ++n) {
                    const uint32_t d = tmem + (n & 1) * BN;
                    if (!(fine = warp_wait(&acc_empty[n & 1], ((n >> 1) & 1) ^ 1, limit))) break;
                    tc_fence_after();
                    const int todo = (min(t.kb1, kb0 + g.chunk) - kb0) * g.pairs;
                    for (int it = 0; it < todo; ++it) {
                        if (!(fine = warp_wait(&full[slot], phase, limit))) break;
                        tc_fence_after();
                        if (me) {
                            const uint64_t da = first + slot * (STAGE >> 4), db = da + (A_BYTES >> 4);
                            // (four in a row behind one branch: with a branch at each, 649 cycles per slot in 16 bits, not 516)
                            if (g.eight) {
#pragma unroll
                                for (int k = 0; k < 4; ++k) mma<CG, true>(d, da + k * step_a, db + k * step_b, g.idesc, it | k);
                            } else {
#pragma unroll
                                for (int k = 0; k < 4; ++k) mma<CG, false>(d, da + k * step_a, db + k * step_b, g.idesc, it | k);
                            }
                            mma_commit<CG>(&empty[slot]);
                        }
                        __syncwarp();
                        if (++slot == STAGES) slot = 0, phase ^= 1;
                    }
                    if (fine && me) mma_commit<CG>(&acc_full[n & 1]);
                    __syncwarp();
                }
            }
            // the products under way are done before their tensor memory is given up
            if (me) mma_commit_here<CG>(&small.drained);
            __syncwarp();
            warp_wait(&small.drained, 0, WAIT_LIMIT_NS);
        }
    } else if (warp >= 4) {
        constexpr int HALF = TURNS ? BN : BN / 2, WIDE = 128 / sizeof(T);    // columns of a warp; of a tile on its way out
        const int q = warp & 3, half = (warp - 4) >> 2;
        uint8_t* pass = ring + STAGES * STAGE + (warp - 4) * 8192;
        float *bias = small.bias + half * HALF, *scale = small.scale + half * HALF;
        const uint32_t leader[2] = {CG == 2 ? in_block(smem_addr(&acc_empty[0]), 0) : smem_addr(&acc_empty[0]),
                                    CG == 2 ? in_block(smem_addr(&acc_empty[1]), 0) : smem_addr(&acc_empty[1])};
        const uint32_t bias_at = smem_addr(bias), scale_at = smem_addr(scale), row_at = smem_addr(pass) + lane * 128;
        const uint32_t from = tmem + ((uint32_t)(q * 32) << 16) + (TURNS ? 0 : half * HALF);
        const int has = todo_of(g.f), act = g.f.act, vec = g.f.vec, splits = g.splits, chunk = g.chunk;
        int n = 0, out_buf = 0, turn = 0;
        bool fine = limit != 0;
        for (int u = cluster; u < g.units; u += clusters) {
            const Unit t = unit_of(g, u);
            const long long m0 = (long long)(t.tm * CG + (int)rank) * TILE_M + q * 32, n0 = (long long)t.tn * BN + (TURNS ? 0 : half * HALF);
            if (TURNS && (turn++ & 1) != half) {
                n += (t.kb1 - t.kb0 + g.chunk - 1) / g.chunk;
                continue;
            }
            const long long m = m0 + lane, row = t.r * g.M + m;
            const bool in = m < g.M;
            if (g.columns) {                         // (uniform) what belongs to the columns, for the four warps of this half
                asm volatile("bar.sync %0, 128;" ::"r"(1 + half) : "memory");
                const int i = q * 32 + lane;
                if (i < HALF) {
                    const bool there = n0 + i < g.N;
                    bias[i] = g.f.bias && there ? element(g.f.bias, g.f.bias_type, t.r * g.f.bias_worker + n0 + i) : 0.0f;
                    scale[i] = g.f.b_scale && there ? g.f.b_scale[t.r * g.f.b_scale_worker + n0 + i] : 1.0f;
                }
                asm volatile("bar.sync %0, 128;" ::"r"(1 + half) : "memory");
            }
            const float a_scale = has & SCALED && in ? g.f.a_scale[row] : 1.0f;
            const T* out_row = static_cast<const T*>(g.f.out) + t.r * g.f.out_worker + m * g.f.out_stride + n0;
            const T* res_row = static_cast<const T*>(g.f.res) + row * g.f.res_stride + n0;
            const int cols = (int)max(0ll, min((long long)HALF, g.N - n0)), rows = (int)max(0ll, min(32ll, g.M - m0));
            for (int kb0 = t.kb0; kb0 < t.kb1; kb0 += chunk, ++n) {
                const bool more = g.f.accumulate || kb0 > t.kb0, added = more && g.l2_adds;
                const int buf = n & 1, how = (more && !added ? ADD : 0) | (kb0 + chunk < t.kb1 || splits > 1 ? RAW : 0), todo = has | how;
                if (fine) fine = warp_wait(&acc_full[buf], (n >> 1) & 1, limit);
                if (!fine && lane == 0) flag_status(g.status, QS_TIMEOUT);
                tc_fence_after();
                // sums of the chunks before have arrived where they are read again or added to, in this order
                if (more) {
                    bulk_wait_all();
                    __syncwarp();
                }
#pragma unroll 1
                for (int c0 = 0; c0 < HALF; c0 += WIDE) {
                    const bool some = rows > 0 && c0 < cols;
                    uint8_t* tile = pass + (has & KEPT ? 0 : out_buf * 4096);
                    if (some && vec) {               // the tile's last copy has been read
                        if (has & KEPT) bulk_wait_read<0>();
                        else bulk_wait_read<1>();
                        __syncwarp();
                    }
#pragma unroll 1
                    for (int c = 0; c < WIDE; c += 32) {
                        uint32_t raw[32];
                        float v[32];
                        if (fine) {
                            tmem_load32(raw, from + buf * BN + c0 + c);
                            tmem_wait_load();
                        } else {
#pragma unroll
                            for (int i = 0; i < 32; ++i) raw[i] = 0x7fffffff;
                        }
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(raw[i]);
                        if (c0 + c + 32 == HALF && fine) {           // the accumulator is free once its last columns are in registers
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) mbar_arrive_at(leader[buf]);
                        }
                        if (!some) continue;
                        const int at = c0 + c;
                        if (vec) {
                            const int left = in ? max(0, min(32, cols - at)) : 0, first = c * (int)sizeof(T) / 16;
                            const uint32_t to = row_at + (has & KEPT ? 0 : out_buf * 4096);
#define QS_FINISH(ACT) finish_row<ACT, T>(todo, v, out_row + at, res_row + at, left, a_scale, bias_at + 4 * at, scale_at + 4 * at, to, row_at + 4096, first, lane)
                            switch (act) {
                            case QS_ACT_RELU: QS_FINISH(QS_ACT_RELU); break;
                            case QS_ACT_SILU: QS_FINISH(QS_ACT_SILU); break;
                            case QS_ACT_GELU: QS_FINISH(QS_ACT_GELU); break;
                            default: QS_FINISH(QS_ACT_NONE);
                            }
#undef QS_FINISH
                        } else {
                            float* turned = reinterpret_cast<float*>(pass);
#pragma unroll
                            for (int j = 0; j < 8; ++j) *reinterpret_cast<float4*>(turned + lane * 32 + (j ^ (lane & 7)) * 4) = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
                            __syncwarp();
                            if (at + lane < cols) {
                                const long long col = n0 + at + lane;
                                switch (act) {
                                case QS_ACT_RELU: finish_columns<QS_ACT_RELU, T>(g.f, t.r, m0, col, rows, turned, lane, how); break;
                                case QS_ACT_SILU: finish_columns<QS_ACT_SILU, T>(g.f, t.r, m0, col, rows, turned, lane, how); break;
                                case QS_ACT_GELU: finish_columns<QS_ACT_GELU, T>(g.f, t.r, m0, col, rows, turned, lane, how); break;
                                default: finish_columns<QS_ACT_NONE, T>(g.f, t.r, m0, col, rows, turned, lane, how);
                                }
                            }
                            __syncwarp();
                        }
                    }
                    if (some && vec) {
                        fence_async_smem();
                        __syncwarp();
                        if (lane == 0) {
                            const int n1 = (int)n0 + c0;
                            if (added) tile_add(&map_out, smem_addr(tile), n1, (int)m0, t.split, t.r);
                            else tile_store(&map_out, smem_addr(tile), n1, (int)m0, t.split, t.r);
                            if (has & KEPT && !(how & RAW)) tile_store(&map_pre, smem_addr(pass + 4096), n1, (int)m0, 0, t.r);
                            bulk_commit();
                        }
                        out_buf ^= 1;
                    }
                }
            }
        }
        bulk_wait_all();
    }
    tc_fence_before();
    __syncthreads();
    if (CG == 2) cluster_sync();
    tc_fence_after();
    if (warp == 2) tmem_free<CG>(tmem, 2 * BN);
}

// Sums out of the workspace, those of splits joined in order, and what follows
template <int V>
__global__ void __launch_bounds__(256) join_splits_kernel(const float* part, long long ld, int splits, int R, const Finish f) {
    after_launch();
    const long long units = (f.N + V - 1) / V, items = R * f.M * units, plane = f.M * ld;      // part: (R, splits, M, ld)
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < items; i += (long long)gridDim.x * 256) {
        const long long row = i / units, n = (i - row * units) * V;
        const int r = (int)(row / f.M);
        const float* p = part + (row + r * (splits - 1) * f.M) * ld + n;
        float v[V];
        load_floats<V>(v, p);
        for (int s = 1; s < splits; ++s) {
            float t[V];
            load_floats<V>(t, p + s * plane);
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] += t[j];
        }
        Columns<V> c;
        load_columns(f, r, n, c);
        finish_any(f, r, row - r * f.M, n, v, c, f.accumulate ? ADD : 0);
    }
}

// ------------------------------------------------------------------ small products, in fp32 on the ordinary units
struct Side { const void* p; long long row, k, worker; };                // element (row, k) of a worker
__device__ __forceinline__ float e4m3_at(const void* p, long long i) {
    const __half_raw h = __nv_cvt_fp8_to_halfraw(static_cast<const uint8_t*>(p)[i], __NV_E4M3);
    return __half2float(__half(h));
}
// TYPE: as stored; AS: what it is multiplied as (fp32 weights of 16-bit rows are rounded)
template <int TYPE, int AS>
__device__ __forceinline__ float side_at(const Side& s, long long i) {
    if (TYPE == QS_E4M3) return e4m3_at(s.p, i);
    const float v = element(s.p, TYPE, i);
    return TYPE == QS_F32 && AS == QS_BF16 ? to_float(__float2bfloat16_rn(v)) : TYPE == QS_F32 && AS == QS_F16 ? to_float(__float2half_rn(v)) : v;
}
// 32 x 32 results per block.  Four groups of 64 threads each take a quarter of the contraction, 16 at a time, the next 16 on
// their way to registers while these are multiplied; their sums are joined in order.
template <int TA, int TB>
__global__ void __launch_bounds__(256, 3) small_kernel(const Side a, const Side b, int K, const Finish f) {
    __shared__ float4 tiles[4][2][16][9];            // (group, operand, k, rows by four; one place of padding)
    const int r = blockIdx.z, group = threadIdx.x >> 6, t = threadIdx.x & 63, tx = t & 7, ty = t >> 3;
    const int per = ((K + 3) / 4 + 15) / 16 * 16, k0 = min(K, group * per), k1 = min(K, k0 + per);
    const long long n0 = (long long)blockIdx.x * 32;
    for (long long m0 = (long long)blockIdx.y * 32; m0 < f.M; m0 += (long long)gridDim.y * 32) {
        float acc[4][4] = {}, next[2][8];
        const auto fetch = [&](int k) {
#pragma unroll
            for (int o = 0; o < 2; ++o) {
                const Side& s = o ? b : a;
                const long long first = o ? n0 : m0, most = o ? f.N : f.M;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int e = t + 64 * i, row = s.k == 1 ? e >> 4 : e & 31, kk = s.k == 1 ? e & 15 : e >> 5;
                    next[o][i] = first + row < most && k + kk < k1 ? (o ? side_at<TB, TA>(s, r * s.worker + (first + row) * s.row + (k + kk) * s.k) : side_at<TA, TA>(s, r * s.worker + (first + row) * s.row + (k + kk) * s.k)) : 0.0f;
                }
            }
        };
        if (k0 < k1) fetch(k0);
        for (int k = k0; k < k0 + per; k += 16) {    // (all groups take as many steps: the barriers are the block's)
            __syncthreads();
#pragma unroll
            for (int o = 0; o < 2; ++o) {
                const Side& s = o ? b : a;
                float* to = reinterpret_cast<float*>(tiles[group][o]);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int e = t + 64 * i, row = s.k == 1 ? e >> 4 : e & 31, kk = s.k == 1 ? e & 15 : e >> 5;
                    to[kk * 36 + row] = k < k1 ? next[o][i] : 0.0f;
                }
            }
            __syncthreads();
            if (k + 16 < k1) fetch(k + 16);
#pragma unroll
            for (int kk = 0; kk < 16; ++kk) {
                const float4 x = tiles[group][0][kk][ty], y = tiles[group][1][kk][tx];
                const float xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[i][j] = __fmaf_rn(xs[i], ys[j], acc[i][j]);
            }
        }
        __syncthreads();
        float* sums = reinterpret_cast<float*>(tiles);                       // (group, m, n) of 32 x 33
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) sums[(group * 32 + ty * 4 + i) * 33 + tx * 4 + j] = acc[i][j];
        __syncthreads();
        const int col = threadIdx.x & 31;
        if (n0 + col < f.N) {
            Columns<1> c;
            load_columns(f, r, n0 + col, c);
            for (int i = threadIdx.x >> 5; i < 32 && m0 + i < f.M; i += 8) {
                const float* q = sums + i * 33 + col;
                float v[1] = {(q[0] + q[32 * 33]) + (q[2 * 32 * 33] + q[3 * 32 * 33])};
                finish_any(f, r, m0 + i, n0 + col, v, c, f.accumulate ? ADD : 0);
            }
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------ few rows: the weights go by once
// Decoding: up to 32 rows of x, so the weights' bytes are all there is.  A block takes 16 or 32 rows of the weights (the matrix
// instruction's 16 rows), its eight warps stretches of 64 along k in turn; their sums are joined in order.  The order along k
// within a stretch is free, so a lane's four places in two products are eight neighbours in memory: one load of 16 bytes per row
// and two products.  fp32 weights are rounded, or cut in three, on the way: nothing is laid out first.  (us, one row of x, 8192 x 8192
// weights: bf16 28, 4.8 TB/s; e4m3 12.4.  Streaming hints on the loads: 31 to 35, and 18: the halves of a line are read by two
// loads.  8 x 2048 x 8192, weights in the L2: 6.3; 16 rows 8.5; the same from fp32 weights 9.1)
constexpr int FEW = 32;                              // rows of x
struct FewArgs {
    const void* x; long long x_stride, x_worker;
    const void* w; long long w_stride, w_worker;
    int K;
    Finish f;
};
struct Eight { uint32_t v[4]; };                     // eight elements of 16 bits
template <bool HALF>
__device__ __forceinline__ uint32_t pair_of(float lo, float hi) {
    return HALF ? pack_two<__half>(lo, hi) : pack_two<bf16>(lo, hi);
}
// Elements [k, k + 8) of a row (BITS 8: sixteen, [2 k, 2 k + 16)); those at K and beyond are zero.  BITS: of an element; VEC: rows on 16-byte
// boundaries
template <bool VEC>
__device__ __forceinline__ void floats_at(float (&v)[8], const float* p, int k, int K) {
    if (VEC && k + 8 <= K) return load_floats<8>(v, p + k);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = k + i < K ? p[k + i] : 0.0f;
}
template <int BITS, bool HALF, bool VEC>
__device__ __forceinline__ Eight eight_at(const void* p, long long row, int k, int K) {
    Eight e = {};
    if (BITS == 8) k *= 2;
    if (k >= K) return e;
    if (VEC && k + (BITS == 8 ? 16 : 8) <= K) {
        const uint4* q = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(p) + (row + k) * (BITS / 8));
        const uint4 a = *q;
        if (BITS == 32) {
            const uint4 b = q[1];
            e.v[0] = pair_of<HALF>(__uint_as_float(a.x), __uint_as_float(a.y)), e.v[1] = pair_of<HALF>(__uint_as_float(a.z), __uint_as_float(a.w));
            e.v[2] = pair_of<HALF>(__uint_as_float(b.x), __uint_as_float(b.y)), e.v[3] = pair_of<HALF>(__uint_as_float(b.z), __uint_as_float(b.w));
        } else {
            e.v[0] = a.x, e.v[1] = a.y, e.v[2] = a.z, e.v[3] = a.w;
        }
        return e;
    }
    if (BITS != 32 && k + (BITS == 8 ? 16 : 8) <= K) {
        const uint4 a = bytes_at(reinterpret_cast<uintptr_t>(p) + (uintptr_t)(row + k) * (BITS / 8));
        e.v[0] = a.x, e.v[1] = a.y, e.v[2] = a.z, e.v[3] = a.w;
        return e;
    }
    if (BITS == 32) {
        float v[8];
        floats_at<false>(v, static_cast<const float*>(p) + row, k, K);
#pragma unroll
        for (int i = 0; i < 4; ++i) e.v[i] = pair_of<HALF>(v[2 * i], v[2 * i + 1]);
    } else if (BITS == 16) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (k + i < K) e.v[i / 2] |= (uint32_t)static_cast<const uint16_t*>(p)[row + k + i] << (i % 2 * 16);
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (k + i < K) e.v[i / 4] |= (uint32_t)static_cast<const uint8_t*>(p)[row + k + i] << (i % 4 * 8);
    }
    return e;
}
template <int BITS, bool HALF>
__device__ __forceinline__ void mma_16x8(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
#define QS_MMA(shape)                                                                                                              \
    asm volatile("mma.sync.aligned." shape " {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"                        \
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1))
    if (BITS == 8) QS_MMA("m16n8k32.row.col.f32.e4m3.e4m3.f32");
    else if (HALF) QS_MMA("m16n8k16.row.col.f32.f16.f16.f32");
    else QS_MMA("m16n8k16.row.col.f32.bf16.bf16.f32");
#undef QS_MMA
}
// fp32 in its three parts
template <bool VEC>
__device__ __forceinline__ void parts_at(Eight (&e)[3], const void* p, long long row, bool ok, int k, int K) {
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.0f;
    if (ok && k < K) floats_at<VEC>(v, static_cast<const float*>(p) + row, k, K);
#pragma unroll
    for (int q = 0; q < 3; ++q) {
        const uint4 u = q ? parts_of<false>(v) : parts_of<true>(v);
        e[q].v[0] = u.x, e[q].v[1] = u.y, e[q].v[2] = u.z, e[q].v[3] = u.w;
    }
}
// MT x 16 rows of the weights per block, NT x 8 rows of x; PARTS 3: both in fp32
template <int MT, int NT, int WBITS, bool HALF, bool VEC, int PARTS>
__global__ void __launch_bounds__(256) few_kernel(const FewArgs a) {
    __shared__ float sums[8][NT * 8][MT * 16 + 1];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, r = blockIdx.y;
    const long long n0 = (long long)blockIdx.x * (MT * 16);
    float acc[MT][NT][4] = {};
    long long wrow[MT][2], xrow[NT];
    bool wok[MT][2], xok[NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const long long n = n0 + i * 16 + h * 8 + g;
            wok[i][h] = n < a.f.N;
            wrow[i][h] = r * a.w_worker + (wok[i][h] ? n : 0) * a.w_stride;
        }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        xok[j] = j * 8 + g < a.f.M;
        xrow[j] = r * a.x_worker + (xok[j] ? j * 8 + g : 0) * a.x_stride;
    }
    const auto product = [&](float (&d)[4], const Eight& w0, const Eight& w1, const Eight& x) {
        mma_16x8<WBITS, HALF>(d, w0.v[0], w1.v[0], w0.v[1], w1.v[1], x.v[0], x.v[1]);
        mma_16x8<WBITS, HALF>(d, w0.v[2], w1.v[2], w0.v[3], w1.v[3], x.v[2], x.v[3]);
    };
    // (the matrix instruction cuts its sums as the large one does: two stretches, then they are added up rounded)
    const auto stretch = [&](float (&acc)[MT][NT][4], int k) {
        if constexpr (PARTS == 3) {
            Eight w[MT][2][3], x[NT][3];
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) parts_at<VEC>(w[i][h], a.w, wrow[i][h], wok[i][h], k, a.K);
#pragma unroll
            for (int j = 0; j < NT; ++j) parts_at<VEC>(x[j], a.x, xrow[j], xok[j], k, a.K);
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int p = 0; p < 6; ++p) product(acc[i][j], w[i][0][part_a(6, p)], w[i][1][part_a(6, p)], x[j][part_b(6, p)]);
        } else {
            Eight w[MT][2], x[NT];
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) w[i][h] = wok[i][h] ? eight_at<WBITS, HALF, VEC>(a.w, wrow[i][h], k, a.K) : Eight{};
#pragma unroll
            for (int j = 0; j < NT; ++j) x[j] = xok[j] ? eight_at<WBITS == 8 ? 8 : 16, HALF, VEC>(a.x, xrow[j], k, a.K) : Eight{};
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) product(acc[i][j], w[i][0], w[i][1], x[j]);
        }
    };
    const int places = WBITS == 8 ? (a.K + 1) / 2 : a.K;     // pairs of 8 bits take the place of 16
#pragma unroll(NT == 1 ? 2 : 1)
    for (int k = warp * 64; k < places; k += 512) {
        float two[MT][NT][4] = {};
        stretch(two, k + t * 8);
        stretch(two, k + 32 + t * 8);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][e] += two[i][j][e];
    }
    // lane (g, t) holds rows g and g + 8 of the weights, rows 2 t and 2 t + 1 of x
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) sums[warp][j * 8 + 2 * t + (e & 1)][i * 16 + g + (e >> 1) * 8] = acc[i][j][e];
    __syncthreads();
    for (int i = threadIdx.x; i < NT * 8 * MT * 16; i += 256) {
        const int m = i / (MT * 16), c = i - m * (MT * 16);
        const long long n = n0 + c;
        if (m >= a.f.M || n >= a.f.N) continue;
        float v[1] = {sums[0][m][c]};
#pragma unroll
        for (int w = 1; w < 8; ++w) v[0] += sums[w][m][c];
        Columns<1> cols;
        load_columns(a.f, r, n, cols);
        finish_any(a.f, r, m, n, v, cols, a.f.accumulate ? ADD : 0);
    }
}

// fp32 by few rows of fp32: ordinary multiply-adds keep up with memory.  Four rows of the weights per block, stretches of 128 along k
// by its eight warps in turn, RM rows of x; their sums are joined in order.  (8 workers, one row, 6912 x 5696: 1.26 GB; by the matrix
// instruction in three parts 367 us)
template <int RM, bool VEC>
__global__ void __launch_bounds__(256, RM <= 4 ? 3 : 2) few_floats_kernel(const FewArgs a) {
    __shared__ float sums[8][4][RM];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r = blockIdx.y;
    const long long n0 = (long long)blockIdx.x * 4;
    const float *w[4], *x[RM];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = static_cast<const float*>(a.w) + r * a.w_worker + min(n0 + i, a.f.N - 1) * a.w_stride;
#pragma unroll
    for (int j = 0; j < RM; ++j) x[j] = static_cast<const float*>(a.x) + r * a.x_worker + min((long long)j, a.f.M - 1) * a.x_stride;
    float acc[4][RM] = {};
#pragma unroll(RM <= 2 ? 2 : 1)
    for (int k = warp * 128; k < a.K; k += 1024) {
        float wv[4][4], xv[RM][4];
        const auto four = [&](float (&v)[4], const float* p) {
            const int at = k + lane * 4;
            if (VEC && at + 4 <= a.K) return load_floats<4>(v, p + at);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = VEC ? at + e : k + 32 * e + lane;
                v[e] = i < a.K ? p[i] : 0.0f;
            }
        };
#pragma unroll
        for (int i = 0; i < 4; ++i) four(wv[i], w[i]);
#pragma unroll
        for (int j = 0; j < RM; ++j) four(xv[j], x[j]);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < RM; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j] = __fmaf_rn(wv[i][e], xv[j][e], acc[i][j]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < RM; ++j) {
            const float s = warp_sum_f(acc[i][j]);
            if (lane == 0) sums[warp][i][j] = s;
        }
    __syncthreads();
    const int i = threadIdx.x & 3, j = threadIdx.x >> 2;
    if (j >= RM || j >= a.f.M || n0 + i >= a.f.N) return;
    float v[1] = {sums[0][i][j]};
#pragma unroll
    for (int q = 1; q < 8; ++q) v[0] += sums[q][i][j];
    Columns<1> c;
    load_columns(a.f, r, n0 + i, c);
    finish_any(a.f, r, j, n0 + i, v, c, a.f.accumulate ? ADD : 0);
}

// ------------------------------------------------------------------ host
struct Operand {
    const void* p; int type;
    long long rows;                                  // of the result's side
    long long ld, worker;                            // between rows in memory, between workers (0: one for all)
    int across;                                      // memory rows run along k
};
struct Product {
    int R; long long M, N, K; int type;              // type: what both operands are multiplied as
    Operand a, b;
};

struct Plan {
    bool small, few, lay_a, lay_b;
    bool kept;                                       // sums in the workspace: of splits, or where the result has no room for them
    int cg, bn, planes, splits;
    long long k_blocks, chunk;                       // blocks along k: in all, and summed by the matrix unit in one go
    long long ld_a, ld_b, part_ld;
    long long off_b, off_part, bytes;
};

long long round_up(long long v, long long to) { return (v + to - 1) / to * to; }
int bytes_of(int type) { return type == QS_E4M3 ? 1 : size_of_type(type); }

long long memory_rows(const Product& p, const Operand& o) { return o.across ? p.K : o.rows; }
long long memory_cols(const Product& p, const Operand& o) { return o.across ? o.rows : p.K; }
bool taken_as_it_lies(const Product& p, const Operand& o) {
    const int size = bytes_of(o.type);
    return o.type == p.type && p.type != QS_F32 && aligned_to(o.p, 16) && (memory_rows(p, o) == 1 || (o.ld * size % 16 == 0 && o.ld < 1ll << 36)) &&
           (p.R == 1 || (o.worker * size % 16 == 0 && o.worker < 1ll << 36));       // (a map's strides end at 2^40 bytes)
}

// Tiles of 256 x 256 by two blocks, of 128 x 128 and 128 x 64 by one.  Measured in bf16, and used for all types (us; each form with the splits that suit it best):
// 512 x 4096 x 4096 24.1, 21.0, 33.7; 2048 x 2048 x 2048 19.5, 21.8, 35.6; 1024 x 1024 x 1024 13.4, 10.2, 9.7; 64 x 4096 x 4096 16.1, 12.2
// (four splits; one 19.7), 14.9
constexpr double FORM_BASE[3] = {8.5, 6.2, 6.2}, FORM_BLOCK[3] = {0.29, 0.22, 0.20};
// in_place: the result lies where something is still to be read.  Sums of several chunks need a place in fp32: the result's, or their own
Plan plan_of(const Product& p, int sms, int out_type, bool in_place) {
    Plan q{};
    q.planes = p.type == QS_F32 ? 3 : 1;
    q.splits = 1;
    const double work = 2.0 * p.R * p.M * p.N * p.K;
    q.few = p.M <= FEW && !p.a.across && !p.b.across;
    // (us, plain and on the matrix unit: fp32, which is laid out first, 64 x 64 x 64 4.7, 10.5; 33 x 200 x 300 12.6, 16.5; 509 x 1000 x 257
    // 34, 20.  bf16 64 x 64 x 64 5.7, 5.5; 33 x 200 x 300 24, 9)
    q.small = !q.few && (p.K == 0 || work < (p.type == QS_F32 ? 5e6 : 5e5));
    if (q.few || q.small) return q;
    const int size = p.type == QS_E4M3 ? 1 : 2;
    q.lay_a = !taken_as_it_lies(p, p.a);
    q.lay_b = !taken_as_it_lies(p, p.b);
    q.ld_a = round_up(memory_cols(p, p.a), 16);
    q.ld_b = round_up(memory_cols(p, p.b), 16);
    // What a tile and a split would take, in us: launch, first loads and last stores; a block along k (latency of the copies, where few
    // blocks are at work, as much as the products); the join of the splits
    const long long k_blocks = (p.K + 128 / size - 1) / (128 / size), pairs = q.planes == 3 ? 6 : 1;
    double best = 0;
    for (int form = 0; form < 3; ++form) {
        const int cg = form == 0 ? 2 : 1, bn = form == 0 ? 256 : form == 1 ? 128 : 64;
        const long long tiles = p.R * ((p.M + cg * TILE_M - 1) / (cg * TILE_M)) * ((p.N + bn - 1) / bn), slots = sms / cg;
        for (long long splits = 1; splits <= 64 && (splits == 1 || k_blocks >= 2 * splits); splits *= 2) {
            if (splits > 1 && tiles >= slots) continue;
            const long long rounds = (tiles * splits + slots - 1) / slots;
            double us = FORM_BASE[form] + rounds * ((double)((k_blocks + splits - 1) / splits) * pairs * FORM_BLOCK[form] + 0.5);
            if (splits > 1) us += 2.0 + 1e-6 * splits * p.R * p.M * p.N;
            if (best == 0 || us < best) best = us, q.cg = cg, q.bn = bn, q.splits = (int)splits;
        }
    }
    long long at = 0;
    const long long wa = p.a.worker || p.R == 1 ? p.R : 1, wb = p.b.worker || p.R == 1 ? p.R : 1;
    if (q.lay_a) at += round_up(wa * q.planes * memory_rows(p, p.a) * q.ld_a * size, 256);
    q.off_b = at;
    if (q.lay_b) at += round_up(wb * q.planes * memory_rows(p, p.b) * q.ld_b * size, 256);
    q.off_part = at;
    q.part_ld = round_up(p.N, 8);
    q.k_blocks = k_blocks;
    q.chunk = out_type == QS_F32 ? CHUNK_BLOCKS : out_type == QS_F16 ? CHUNK_F16 : CHUNK_BF16;
    q.kept = q.splits > 1 || (k_blocks > q.chunk && (in_place || out_type != QS_F32));
    if (q.kept) at += 4ll * q.splits * p.R * p.M * q.part_ld;
    q.bytes = at;
    return q;
}

typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                             CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeFn encoder() {
    static const EncodeFn fn = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            f = nullptr;
        }
        return reinterpret_cast<EncodeFn>(f);
    }();
    return fn;
}
// (inner, outer, plane, worker) in boxes of 128 bytes by `box` rows
bool encode(CUtensorMap* map, const void* p, int type, long long inner, long long outer, int planes, long long workers, long long ld, long long plane,
            long long worker, int box) {
    const int size = bytes_of(type);
    const EncodeFn fn = encoder();
    if (!fn) return false;
    const cuuint64_t dims[4] = {(cuuint64_t)inner, (cuuint64_t)outer, (cuuint64_t)planes, (cuuint64_t)workers};
    // (a dimension of one element has no stride: any that is allowed)
    const long long row = outer > 1 ? ld * size : round_up(inner * size, 16);
    const cuuint64_t strides[3] = {(cuuint64_t)row, (cuuint64_t)(planes > 1 ? plane * size : row), (cuuint64_t)(workers > 1 ? worker * size : row)};
    const cuuint32_t boxes[4] = {(cuuint32_t)(128 / size), (cuuint32_t)box, 1, 1}, ones[4] = {1, 1, 1, 1};
    const CUtensorMapDataType t = type == QS_E4M3  ? CU_TENSOR_MAP_DATA_TYPE_UINT8
                                  : type == QS_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                  : type == QS_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16
                                                   : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    return fn(map, t, 4, const_cast<void*>(p), dims, strides, boxes, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// a result, written in tiles of 32 rows
bool encode_out(CUtensorMap* map, const void* p, int type, long long N, long long M, int planes, long long workers, long long ld, long long plane, long long worker) {
    return encode(map, p, type, N, M, planes, workers, ld, plane, worker, 32);
}

unsigned long long wait_limit() {
    static const unsigned long long ns = [] {
        const char* e = std::getenv("QSPARSE_WAIT_LIMIT_NS");
        return e ? std::min(std::strtoull(e, nullptr, 10), WAIT_LIMIT_NS) : WAIT_LIMIT_NS;
    }();
    return ns;
}

LayArgs lay_args(const Product& p, const Operand& o, void* dst, int dst_type, int planes, long long ld) {
    LayArgs a{};
    a.workers = o.worker || p.R == 1 ? p.R : 1;
    a.src = o.p; a.src_type = o.type; a.src_stride = o.ld; a.src_worker = o.worker;
    a.dst = dst; a.dst_type = dst_type; a.planes = planes; a.ld = ld; a.rows = memory_rows(p, o); a.cols = memory_cols(p, o);
    return a;
}
cudaError_t lay_out(const LayBoth& both, int sides, cudaStream_t st) {
    long long items = 0, workers = 0;
    for (int i = 0; i < sides; ++i) {
        items = std::max(items, both.side[i].rows * (both.side[i].ld / 8));
        workers = std::max<long long>(workers, both.side[i].workers);
    }
    return launch(false, lay_kernel, dim3((unsigned)std::min<long long>((items + 255) / 256, 1 << 16), (unsigned)workers, (unsigned)sides), 256, 0, st, both);
}

template <int CG, int BN, class T>
cudaError_t launch_gemm_as(const CUtensorMap (&map)[4], const GemmArgs& g, bool after, int sms, cudaStream_t st) {
    constexpr int smem = gemm_smem<CG, BN>();
    cudaError_t e = cudaFuncSetAttribute(gemm_kernel<CG, BN, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)std::min(g.units, sms / CG) * CG);
    cfg.blockDim = dim3(GEMM_THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = CG;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = after ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, gemm_kernel<CG, BN, T>, map[0], map[1], map[2], map[3], g);
}
template <int CG, int BN>
cudaError_t launch_gemm(const CUtensorMap (&map)[4], const GemmArgs& g, bool after, int sms, cudaStream_t st) {
    // (sums that are kept are written in fp32 whatever the result's type: one form is enough)
    if (g.f.type == QS_F32) return launch_gemm_as<CG, BN, float>(map, g, after, sms, st);
    return g.f.type == QS_BF16 ? launch_gemm_as<CG, BN, bf16>(map, g, after, sms, st) : launch_gemm_as<CG, BN, __half>(map, g, after, sms, st);
}

template <int WBITS, bool HALF, bool VEC, int PARTS>
cudaError_t launch_few_as(const Product& p, const FewArgs& a, cudaStream_t st) {
    // 32 rows of the weights per block where that still gives every SM one: x is read once per block
    const bool wide = PARTS == 1 && p.M > 8 && p.R * p.N >= 32 * 148;
    const dim3 grid((unsigned)((p.N + (wide ? 31 : 15)) / (wide ? 32 : 16)), (unsigned)p.R);
    if constexpr (PARTS == 1)
        if (wide)
            return p.M <= 16 ? launch(false, few_kernel<2, 2, WBITS, HALF, VEC, 1>, grid, 256, 0, st, a)
                             : launch(false, few_kernel<2, 4, WBITS, HALF, VEC, 1>, grid, 256, 0, st, a);
    return p.M <= 8    ? launch(false, few_kernel<1, 1, WBITS, HALF, VEC, PARTS>, grid, 256, 0, st, a)
           : p.M <= 16 ? launch(false, few_kernel<1, 2, WBITS, HALF, VEC, PARTS>, grid, 256, 0, st, a)
                       : launch(false, few_kernel<1, 4, WBITS, HALF, VEC, PARTS>, grid, 256, 0, st, a);
}
cudaError_t launch_few(const Product& p, const FewArgs& a, bool vec, cudaStream_t st) {
    if (p.type == QS_E4M3) return vec ? launch_few_as<8, true, true, 1>(p, a, st) : launch_few_as<8, true, false, 1>(p, a, st);
    if (p.type == QS_F32 && p.M <= 8) {
        const dim3 grid((unsigned)((p.N + 3) / 4), (unsigned)p.R);
        const auto kernel = p.M == 1   ? (vec ? few_floats_kernel<1, true> : few_floats_kernel<1, false>)
                            : p.M == 2 ? (vec ? few_floats_kernel<2, true> : few_floats_kernel<2, false>)
                            : p.M <= 4 ? (vec ? few_floats_kernel<4, true> : few_floats_kernel<4, false>)
                                       : (vec ? few_floats_kernel<8, true> : few_floats_kernel<8, false>);
        return launch(false, kernel, grid, 256, 0, st, a);
    }
    if (p.type == QS_F32) return vec ? launch_few_as<32, false, true, 3>(p, a, st) : launch_few_as<32, false, false, 3>(p, a, st);
    const bool wide = p.b.type == QS_F32;
    if (p.type == QS_F16)
        return wide ? (vec ? launch_few_as<32, true, true, 1>(p, a, st) : launch_few_as<32, true, false, 1>(p, a, st))
                    : (vec ? launch_few_as<16, true, true, 1>(p, a, st) : launch_few_as<16, true, false, 1>(p, a, st));
    return wide ? (vec ? launch_few_as<32, false, true, 1>(p, a, st) : launch_few_as<32, false, false, 1>(p, a, st))
                : (vec ? launch_few_as<16, false, true, 1>(p, a, st) : launch_few_as<16, false, false, 1>(p, a, st));
}

int run_product(const Product& p, const Finish& f, void* work, int64_t work_bytes, int* status, cudaStream_t st) {
    const int sms = sm_count();
    if (!sms) return QS_CUDA;
    const Plan q = plan_of(p, sms, f.type, f.res && f.res == f.out);
    if (q.small) {
        const auto side = [&](const Operand& o) { return Side{o.p, o.across ? 1 : o.ld, o.across ? o.ld : 1, o.worker}; };
        const bool same = p.b.type == p.type;
        const auto kernel = p.type == QS_E4M3   ? small_kernel<QS_E4M3, QS_E4M3>
                            : p.type == QS_F32  ? small_kernel<QS_F32, QS_F32>
                            : p.type == QS_BF16 ? (same ? small_kernel<QS_BF16, QS_BF16> : small_kernel<QS_BF16, QS_F32>)
                                                : (same ? small_kernel<QS_F16, QS_F16> : small_kernel<QS_F16, QS_F32>);
        return status_of(launch(false, kernel, dim3((unsigned)((p.N + 31) / 32), (unsigned)std::min<long long>((p.M + 31) / 32, 65535), (unsigned)p.R), 256, 0, st,
                                side(p.a), side(p.b), (int)p.K, f));
    }
    if (q.few) {
        FewArgs a{};
        a.x = p.a.p; a.x_stride = p.a.ld; a.x_worker = p.a.worker;
        a.w = p.b.p; a.w_stride = p.b.ld; a.w_worker = p.b.worker;
        a.K = (int)p.K; a.f = f;
        const auto vec = [&](const Operand& o) {
            const int size = bytes_of(o.type);
            return aligned_to(o.p, 16) && (o.rows == 1 || o.ld * size % 16 == 0) && (p.R == 1 || o.worker * size % 16 == 0);
        };
        return status_of(launch_few(p, a, vec(p.a) && vec(p.b), st));
    }
    if (q.bytes > 0 && work && !aligned_to(work, 256)) return QS_INVALID_ARG;
    if ((work ? work_bytes : 0) < q.bytes) return QS_CAPACITY;
    uint8_t* w = static_cast<uint8_t*>(work);
    const int type = p.type == QS_F32 ? QS_BF16 : p.type, size = type == QS_E4M3 ? 1 : 2;
    GemmArgs g{};
    CUtensorMap map[4] = {};
    LayBoth both{};
    int sides = 0;
    for (int i = 0; i < 2; ++i) {
        const Operand& o = i ? p.b : p.a;
        const bool lay = i ? q.lay_b : q.lay_a;
        const long long rows = memory_rows(p, o), cols = memory_cols(p, o), workers = o.worker || p.R == 1 ? p.R : 1;
        const long long ld = lay ? (i ? q.ld_b : q.ld_a) : o.ld;
        const void* at = lay ? w + (i ? q.off_b : 0) : o.p;
        if (lay) {
            both.side[sides++] = lay_args(p, o, w + (i ? q.off_b : 0), type, q.planes, ld);
        }
        (i ? g.b_worker : g.a_worker) = workers > 1;
        (i ? g.b_across : g.a_across) = o.across;
        const int box = o.across ? 64 : i ? q.bn / q.cg : TILE_M;
        if (!encode(&map[i], at, type, cols, rows, q.planes, workers, ld, rows * ld, lay ? q.planes * rows * ld : o.worker, box)) return QS_CUDA;
    }
    g.R = p.R; g.M = p.M; g.N = p.N;
    g.tiles_m = (int)((p.M + TILE_M * q.cg - 1) / (TILE_M * q.cg));
    g.tiles_n = (int)((p.N + q.bn - 1) / q.bn);
    g.splits = q.splits;
    g.units = p.R * g.tiles_m * g.tiles_n * g.splits;
    g.k_step = 128 / size;
    g.k_blocks = (int)q.k_blocks;
    g.pairs = q.planes == 3 ? 6 : 1;
    g.per_split = g.k_blocks / q.splits;
    g.more = g.k_blocks % q.splits;
    g.chunk = (int)q.chunk;
    g.eight = type == QS_E4M3;
    // sums in fp32; operand types (e4m3 and fp16 are 0, bf16 is 1); which lie across k; the tile
    const uint32_t t = type == QS_BF16 ? 1 : 0;
    g.idesc = 1u << 4 | t << 7 | t << 10 | (uint32_t)g.a_across << 15 | (uint32_t)g.b_across << 16 | (uint32_t)(q.bn / 8) << 17 | (uint32_t)(TILE_M * q.cg / 16) << 24;
    g.limit = wait_limit();
    g.status = status;
    g.f = f;
    g.columns = !q.kept && (f.bias || f.b_scale);
    g.l2_adds = f.vec && f.type == QS_F32 && !q.kept && f.act == QS_ACT_NONE && !f.bias && !f.res && !f.pre && !f.a_scale;
    if ((f.res || ((f.accumulate || g.chunk < g.k_blocks) && !g.l2_adds)) && p.N * size_of_type(f.type) % 16) g.f.vec = 0;
    float* part = reinterpret_cast<float*>(w + q.off_part);
    if (q.kept) {                                    // sums instead of results: (R, splits, M, part_ld)
        g.f = Finish{};
        g.f.M = p.M; g.f.N = p.N; g.f.type = QS_F32; g.f.vec = 1;
        g.l2_adds = 1;
        if (!encode_out(&map[2], part, QS_F32, p.N, p.M, q.splits, p.R, q.part_ld, p.M * q.part_ld, q.splits * p.M * q.part_ld)) return QS_CUDA;
    } else if (g.f.vec) {
        if (!encode_out(&map[2], f.out, f.type, p.N, p.M, 1, p.R, f.out_stride, 0, f.out_worker) ||
            (f.pre && !encode_out(&map[3], f.pre, f.type, p.N, p.M, 1, p.R, f.pre_stride, 0, p.M * f.pre_stride))) return QS_CUDA;
    }
    cudaError_t e = sides ? lay_out(both, sides, st) : cudaSuccess;
    if (e != cudaSuccess) return status_of(e);
    const bool after = sides > 0;
    e = q.cg == 2 ? launch_gemm<2, 256>(map, g, after, sms, st) : q.bn == 128 ? launch_gemm<1, 128>(map, g, after, sms, st) : launch_gemm<1, 64>(map, g, after, sms, st);
    if (e != cudaSuccess || !q.kept) return status_of(e);
    const long long items = p.R * p.M * (f.vec ? (p.N + 7) / 8 : p.N);
    const dim3 grid((unsigned)std::min<long long>((items + 255) / 256, 1 << 20));
    e = f.vec && p.N % 8 == 0 ? launch(true, join_splits_kernel<8>, grid, 256, 0, st, (const float*)part, q.part_ld, q.splits, p.R, f)
                              : launch(true, join_splits_kernel<1>, grid, 256, 0, st, (const float*)part, q.part_ld, q.splits, p.R, f);
    return status_of(e);
}

bool is_act(int act) { return act >= QS_ACT_NONE && act <= QS_ACT_GELU; }
bool bad_sizes(int R, int64_t M, int64_t N, int64_t K) { return R < 1 || R > 32 || M < 0 || N < 1 || K < 1; }
// (tile and block counts fit 31 bits, and so do the tensor maps' coordinates)
bool sizes_too_large(int R, int64_t M, int64_t N, int64_t K) {
    return M > (1ll << 28) || N > (1ll << 24) || K > (1ll << 24) || R * M > (1ll << 28) || R * ((M + 127) / 128) * ((N + 127) / 128) > (1ll << 24);
}
bool bad_matrix(const void* p, int64_t stride, int64_t width, int size) { return !p || stride < width || !aligned_to(p, size); }
bool workers_overlap(int R, int64_t worker, int64_t rows, int64_t stride, int64_t width) {
    return R > 1 && worker < (rows - 1) * stride + width && (worker < width || stride < (R - 1) * worker + width);
}

// ------------------------------------------------------------------ gradient in front of the activation
struct ActGradArgs {
    int R; long long M, N;
    const void* g; long long g_stride;
    const void* z; long long z_stride; int act;
    void* out; long long out_stride;
    float* part; int parts;                          // (R, parts, N): column sums of the rows of a block, or null
};
// 8 warps of rows, 32 V columns per block; block (x, p, r) takes rows p * 8 + warp, + 8 parts, ..
template <class T, int V, int ACT>
__global__ void __launch_bounds__(256) act_grad_kernel(const ActGradArgs a) {
    __shared__ float sh[8][32 * V + 1];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = blockIdx.z;
    const long long n = ((long long)blockIdx.x * 32 + lane) * V;
    float sum[V];
#pragma unroll
    for (int j = 0; j < V; ++j) sum[j] = 0.0f;
    if (n < a.N)
#pragma unroll 2
        for (long long m = blockIdx.y * 8 + warp; m < a.M; m += a.parts * 8) {
            const long long row = r * a.M + m;
            float g[V];
            load_vec<V>(g, static_cast<const T*>(a.g) + row * a.g_stride + n);
            if (ACT != QS_ACT_NONE) {
                float z[V];
                load_vec<V>(z, static_cast<const T*>(a.z) + row * a.z_stride + n);
#pragma unroll
                for (int j = 0; j < V; ++j) g[j] *= slope<ACT, sizeof(T) == 4>(z[j]);
            }
            if (a.out) store_vec<V>(static_cast<T*>(a.out) + row * a.out_stride + n, g);
#pragma unroll
            for (int j = 0; j < V; ++j) sum[j] += g[j];
        }
    if (!a.part) return;
#pragma unroll
    for (int j = 0; j < V; ++j) sh[warp][lane * V + j] = sum[j];
    __syncthreads();
    for (int i = threadIdx.x; i < 32 * V; i += 256) {
        const long long c = (long long)blockIdx.x * 32 * V + i;
        if (c >= a.N) break;
        float s = sh[0][i];
#pragma unroll
        for (int w = 1; w < 8; ++w) s += sh[w][i];
        a.part[((long long)r * a.parts + blockIdx.y) * a.N + c] = s;
    }
}
int act_parts(int R, int64_t M, int64_t N) {
    const long long columns = R * ((N + 255) / 256);
    return (int)std::max<long long>(1, std::min<long long>((M + 31) / 32, (148 * 12 + columns - 1) / columns));
}
template <class T, int V>
cudaError_t launch_act_grad_of(const ActGradArgs& a, cudaStream_t st) {
    const dim3 grid((unsigned)((a.N + 32 * V - 1) / (32 * V)), (unsigned)a.parts, (unsigned)a.R);
    switch (a.act) {
    case QS_ACT_RELU: return launch(false, act_grad_kernel<T, V, QS_ACT_RELU>, grid, 256, 0, st, a);
    case QS_ACT_SILU: return launch(false, act_grad_kernel<T, V, QS_ACT_SILU>, grid, 256, 0, st, a);
    case QS_ACT_GELU: return launch(false, act_grad_kernel<T, V, QS_ACT_GELU>, grid, 256, 0, st, a);
    default: return launch(false, act_grad_kernel<T, V, QS_ACT_NONE>, grid, 256, 0, st, a);
    }
}
template <class T>
cudaError_t launch_act_grad(const ActGradArgs& a, bool vec, cudaStream_t st) {
    return vec ? launch_act_grad_of<T, wide_of<T>()>(a, st) : launch_act_grad_of<T, 1>(a, st);
}

Product forward_of(int R, int64_t M, int64_t N, int64_t K, const void* x, int x_type, int64_t x_stride, const void* w, int w_type, int64_t w_worker, int64_t w_stride) {
    return {R, M, N, K, x_type, {x, x_type, M, x_stride, R > 1 ? M * x_stride : 0, 0}, {w, w_type, N, w_stride, w_worker, 0}};
}
// dx (M x K) = sum over n of dz[m, n] w[n, k]
Product input_of(int R, int64_t M, int64_t N, int64_t K, const void* dz, int type, int64_t dz_stride, const void* w, int w_type, int64_t w_worker, int64_t w_stride) {
    return {R, M, K, N, type, {dz, type, M, dz_stride, R > 1 ? M * dz_stride : 0, 0}, {w, w_type, K, w_stride, w_worker, 1}};
}
// dw (N x K) = sum over m of dz[m, n] x[m, k]
Product weight_of(int R, int64_t M, int64_t N, int64_t K, const void* dz, int type, int64_t dz_stride, const void* x, int64_t x_stride) {
    return {R, N, K, M, type, {dz, type, N, dz_stride, R > 1 ? M * dz_stride : 0, 1}, {x, type, K, x_stride, R > 1 ? M * x_stride : 0, 1}};
}
int64_t bytes_for(const Product& p, int out_type, bool in_place) {
    const int sms = sm_count();
    return sms ? plan_of(p, sms, out_type, in_place).bytes : (int64_t)QS_CUDA;
}
bool weight_type_ok(int type, int w_type) { return type == QS_E4M3 ? w_type == QS_E4M3 : size_of_type(type) && (w_type == type || w_type == QS_F32); }

}  // namespace
}  // namespace qs

using namespace qs;

extern "C" {

int64_t qs_linear_bytes(int R, int64_t M, int64_t N, int64_t K, const void* x, int x_type, int64_t x_stride, const void* w, int w_type,
                        int64_t w_worker_stride, int64_t w_stride) {
    if (bad_sizes(R, M, N, K) || !weight_type_ok(x_type, w_type)) return QS_INVALID_ARG;
    if (sizes_too_large(R, M, N, K)) return QS_TOO_LARGE;
    // (a result in fp32 in its residual's place keeps sums where any other does: enough for all)
    return M ? bytes_for(forward_of(R, M, N, K, x, x_type, x_stride, w, w_type, w_worker_stride, w_stride), QS_F32, true) : 0;
}

int64_t qs_linear_call_bytes(int R, int64_t M, int64_t N, int64_t K, const void* x, int x_type, int64_t x_stride, const void* w, int w_type,
                             int64_t w_worker_stride, int64_t w_stride, int out_type, int in_place) {
    if (bad_sizes(R, M, N, K) || !weight_type_ok(x_type, w_type) || !size_of_type(out_type)) return QS_INVALID_ARG;
    if (sizes_too_large(R, M, N, K)) return QS_TOO_LARGE;
    return M ? bytes_for(forward_of(R, M, N, K, x, x_type, x_stride, w, w_type, w_worker_stride, w_stride), out_type, in_place) : 0;
}

int qs_linear(int R, int64_t M, int64_t N, int64_t K, const void* x, int x_type, int64_t x_stride, const float* x_scale, const void* w, int w_type,
              int64_t w_worker_stride, int64_t w_stride, const float* w_scale, const void* bias, int bias_type, int64_t bias_worker_stride,
              int activation, const void* residual, int64_t residual_stride, void* pre, int64_t pre_stride, void* out, int out_type,
              int64_t out_stride, void* work, int64_t work_bytes, int* status, void* cuda_stream) {
    if (bad_sizes(R, M, N, K) || !weight_type_ok(x_type, w_type) || !is_act(activation)) return QS_INVALID_ARG;
    const bool eight = x_type == QS_E4M3;
    const int size = size_of_type(out_type);
    if (!size || (!eight && out_type != x_type && out_type != QS_F32) || eight != (x_scale != nullptr) || eight != (w_scale != nullptr)) return QS_INVALID_ARG;
    if (sizes_too_large(R, M, N, K)) return QS_TOO_LARGE;
    if (M == 0) return QS_OK;
    if (bad_matrix(x, x_stride, K, bytes_of(x_type)) || bad_matrix(w, w_stride, K, bytes_of(w_type)) || w_worker_stride < 0 ||
        (w_worker_stride && workers_overlap(R, w_worker_stride, N, w_stride, K)) || bad_matrix(out, out_stride, N, size) ||
        (residual && bad_matrix(residual, residual_stride, N, size)) || (pre && bad_matrix(pre, pre_stride, N, size)) || !aligned_to(x_scale, 4) ||
        !aligned_to(w_scale, 4) || !aligned_to(status, 4) ||
        (bias && (!size_of_type(bias_type) || !aligned_to(bias, size_of_type(bias_type)) || bias_worker_stride < 0))) return QS_INVALID_ARG;
    const int64_t rows = R * M, bytes = span(rows, out_stride, N, size), pre_bytes = pre ? span(rows, pre_stride, N, size) : 0;
    const int64_t x_bytes = span(rows, x_stride, K, bytes_of(x_type)), w_bytes = (R - 1) * w_worker_stride * bytes_of(w_type) + span(N, w_stride, K, bytes_of(w_type));
    if (!apart(out, bytes, x, x_bytes) || !apart(out, bytes, w, w_bytes) || !apart(pre, pre_bytes, x, x_bytes) || !apart(pre, pre_bytes, w, w_bytes) ||
        !beside(residual, residual_stride, out, out_stride, rows, N, size) || (pre && (pre == out || pre == residual)) ||
        !beside(residual, residual_stride, pre, pre_stride, rows, N, size) || !beside(pre, pre_stride, out, out_stride, rows, N, size)) return QS_INVALID_ARG;
    Finish f{};
    f.M = M; f.N = N; f.bias = bias; f.bias_type = bias_type; f.bias_worker = bias_worker_stride; f.act = activation;
    f.res = residual; f.res_stride = residual_stride; f.pre = pre; f.pre_stride = pre_stride;
    f.out = out; f.type = out_type; f.out_stride = out_stride; f.out_worker = M * out_stride; f.a_scale = x_scale; f.b_scale = w_scale;
    f.b_scale_worker = w_worker_stride ? N : 0;
    f.vec = rows_aligned(out, out_stride, rows, size, 16) && rows_aligned(residual, residual_stride, rows, size, 16) && rows_aligned(pre, pre_stride, rows, size, 16);
    return run_product(forward_of(R, M, N, K, x, x_type, x_stride, w, w_type, w_worker_stride, w_stride), f, work, work_bytes, status,
                       static_cast<cudaStream_t>(cuda_stream));
}

int64_t qs_linear_grad_input_bytes(int R, int64_t M, int64_t N, int64_t K, const void* dz, int type, int64_t dz_stride, const void* w, int w_type,
                                   int64_t w_worker_stride, int64_t w_stride) {
    if (bad_sizes(R, M, N, K) || !size_of_type(type) || !weight_type_ok(type, w_type)) return QS_INVALID_ARG;
    if (sizes_too_large(R, M, N, K) || sizes_too_large(R, M, K, N)) return QS_TOO_LARGE;
    return M ? bytes_for(input_of(R, M, N, K, dz, type, dz_stride, w, w_type, w_worker_stride, w_stride), type, false) : 0;
}

int qs_linear_grad_input(int R, int64_t M, int64_t N, int64_t K, const void* dz, int type, int64_t dz_stride, const void* w, int w_type,
                         int64_t w_worker_stride, int64_t w_stride, void* out, int64_t out_stride, void* work, int64_t work_bytes, int* status,
                         void* cuda_stream) {
    if (bad_sizes(R, M, N, K) || !size_of_type(type) || !weight_type_ok(type, w_type)) return QS_INVALID_ARG;
    if (sizes_too_large(R, M, N, K) || sizes_too_large(R, M, K, N)) return QS_TOO_LARGE;
    if (M == 0) return QS_OK;
    const int size = size_of_type(type);
    if (bad_matrix(dz, dz_stride, N, size) || bad_matrix(w, w_stride, K, size_of_type(w_type)) || bad_matrix(out, out_stride, K, size) || w_worker_stride < 0 ||
        (w_worker_stride && workers_overlap(R, w_worker_stride, N, w_stride, K)) || !aligned_to(status, 4)) return QS_INVALID_ARG;
    const int64_t rows = R * M, bytes = span(rows, out_stride, K, size);
    if (!apart(out, bytes, dz, span(rows, dz_stride, N, size)) ||
        !apart(out, bytes, w, (R - 1) * w_worker_stride * size_of_type(w_type) + span(N, w_stride, K, size_of_type(w_type)))) return QS_INVALID_ARG;
    Finish f{};
    f.M = M; f.N = K; f.out = out; f.type = type; f.out_stride = out_stride; f.out_worker = M * out_stride;
    f.vec = rows_aligned(out, out_stride, rows, size, 16);
    return run_product(input_of(R, M, N, K, dz, type, dz_stride, w, w_type, w_worker_stride, w_stride), f, work, work_bytes, status,
                       static_cast<cudaStream_t>(cuda_stream));
}

int64_t qs_linear_grad_weight_bytes(int R, int64_t M, int64_t N, int64_t K, const void* dz, int type, int64_t dz_stride, const void* x, int64_t x_stride) {
    if (bad_sizes(R, M, N, K) || !size_of_type(type)) return QS_INVALID_ARG;
    if (sizes_too_large(R, M, N, K) || sizes_too_large(R, N, K, 1)) return QS_TOO_LARGE;
    return M ? bytes_for(weight_of(R, M, N, K, dz, type, dz_stride, x, x_stride), type, false) : 0;
}

int64_t qs_linear_grad_weight_call_bytes(int R, int64_t M, int64_t N, int64_t K, const void* dz, int type, int64_t dz_stride, const void* x,
                                         int64_t x_stride, int out_type) {
    if (bad_sizes(R, M, N, K) || !size_of_type(type) || (out_type != type && out_type != QS_F32)) return QS_INVALID_ARG;
    if (sizes_too_large(R, M, N, K) || sizes_too_large(R, N, K, 1)) return QS_TOO_LARGE;
    return M ? bytes_for(weight_of(R, M, N, K, dz, type, dz_stride, x, x_stride), out_type, false) : 0;
}

int qs_linear_grad_weight(int R, int64_t M, int64_t N, int64_t K, const void* dz, int type, int64_t dz_stride, const void* x, int64_t x_stride, void* out,
                          int out_type, int64_t out_worker_stride, int64_t out_stride, int accumulate, void* work, int64_t work_bytes, int* status,
                          void* cuda_stream) {
    const int size = size_of_type(type), out_size = size_of_type(out_type);
    if (bad_sizes(R, M, N, K) || !size || (out_type != type && out_type != QS_F32)) return QS_INVALID_ARG;
    if (sizes_too_large(R, M, N, K) || sizes_too_large(R, N, K, 1)) return QS_TOO_LARGE;
    if (bad_matrix(out, out_stride, K, out_size) || workers_overlap(R, out_worker_stride, N, out_stride, K) || !aligned_to(status, 4)) return QS_INVALID_ARG;
    if (M == 0 && accumulate) return QS_OK;
    if (M && (bad_matrix(dz, dz_stride, N, size) || bad_matrix(x, x_stride, K, size))) return QS_INVALID_ARG;
    const int64_t bytes = ((R - 1) * out_worker_stride + (N - 1) * out_stride + K) * out_size;
    if (M && (!apart(out, bytes, dz, span(R * M, dz_stride, N, size)) || !apart(out, bytes, x, span(R * M, x_stride, K, size)))) return QS_INVALID_ARG;
    Finish f{};
    f.M = N; f.N = K; f.out = out; f.type = out_type; f.out_stride = out_stride; f.out_worker = R > 1 ? out_worker_stride : 0;
    f.accumulate = accumulate;
    f.vec = rows_aligned(out, out_stride, N, out_size, 16) && (R == 1 || out_worker_stride * out_size % 16 == 0);
    return run_product(weight_of(R, M, N, K, dz, type, dz_stride, x, x_stride), f, work, work_bytes, status, static_cast<cudaStream_t>(cuda_stream));
}

int64_t qs_activation_grad_bytes(int R, int64_t M, int64_t N) {
    if (bad_sizes(R, M, N, 1)) return QS_INVALID_ARG;
    if (sizes_too_large(R, M, N, 1)) return QS_TOO_LARGE;
    return 4 * (int64_t)R * act_parts(R, M, N) * N;
}

int qs_activation_grad(int R, int64_t M, int64_t N, const void* grad, int type, int64_t grad_stride, const void* pre, int64_t pre_stride, int activation,
                       void* out, int64_t out_stride, float* grad_bias, int64_t grad_bias_worker_stride, int accumulate, void* work, int64_t work_bytes,
                       void* cuda_stream) {
    const int size = size_of_type(type);
    if (bad_sizes(R, M, N, 1) || !size || !is_act(activation) || (!out && !grad_bias)) return QS_INVALID_ARG;
    if (sizes_too_large(R, M, N, 1)) return QS_TOO_LARGE;
    if (grad_bias && (!aligned_to(grad_bias, 4) || (R > 1 && grad_bias_worker_stride < N))) return QS_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (M == 0) return !grad_bias || accumulate ? QS_OK : status_of(launch_join(false, nullptr, 0, R, N, grad_bias, grad_bias_worker_stride, 0, st));
    const int64_t rows = R * M;
    const bool act = activation != QS_ACT_NONE;
    if (bad_matrix(grad, grad_stride, N, size) || (act && bad_matrix(pre, pre_stride, N, size)) || (out && bad_matrix(out, out_stride, N, size))) return QS_INVALID_ARG;
    if (!beside(grad, grad_stride, out, out_stride, rows, N, size) || (act && !beside(pre, pre_stride, out, out_stride, rows, N, size))) return QS_INVALID_ARG;
    if (grad_bias && (!work || !aligned_to(work, 16))) return QS_INVALID_ARG;
    if (grad_bias && work_bytes < 4 * (int64_t)R * act_parts(R, M, N) * N) return QS_CAPACITY;
    ActGradArgs a{};
    a.R = R; a.M = M; a.N = N; a.g = grad; a.g_stride = grad_stride; a.z = pre; a.z_stride = pre_stride; a.act = activation; a.out = out; a.out_stride = out_stride;
    a.part = grad_bias ? static_cast<float*>(work) : nullptr;
    a.parts = act_parts(R, M, N);
    const int V = 16 / size;
    const bool vec = N % V == 0 && rows_aligned(grad, grad_stride, rows, size, 16) && rows_aligned(act ? pre : nullptr, pre_stride, rows, size, 16) &&
                     rows_aligned(out, out_stride, rows, size, 16);
    const cudaError_t e = type == QS_F32 ? launch_act_grad<float>(a, vec, st) : type == QS_BF16 ? launch_act_grad<bf16>(a, vec, st) : launch_act_grad<__half>(a, vec, st);
    if (e != cudaSuccess || !grad_bias) return status_of(e);
    return status_of(launch_join(true, a.part, a.parts, R, N, grad_bias, grad_bias_worker_stride, accumulate, st));
}

}  // extern "C"
