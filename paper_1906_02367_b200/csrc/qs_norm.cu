// Root-mean-square norm of rows, with the residual's addition in front of it and 8 bits behind it, and its gradient.
//
//   h = x + residual (rounded to the type of x: what the backward pass reads);  rstd = (mean h^2 + eps)^(-1/2)
//   y = h rstd w;  in 8 bits q = e4m3(y / s), s = max(max |y| / 448, 2^-126)
//   dh = grad_hidden + rstd (w g - n mean(w g n)),  n = h rstd;   dw = sum over the rows of g n
//
// Memory-bound: a row is read once, kept in the registers of a warp (short rows) or a block, and written once.  (32768 x 2048 in
// bf16: norm with residual 86 us, 6.3 TB/s; into 8 bits 78, 6.0)
#include <algorithm>

#include "qs_parts.cuh"

namespace qs {
namespace {

constexpr float E4M3_MAX = 448.0f;
constexpr float LEAST_SCALE = 1.17549435e-38f;       // 2^-126: its reciprocal is finite

struct NormArgs {
    int R; long long N, D;                           // R workers, N rows each
    const void* x; long long x_stride;
    const void* res; long long res_stride;
    const void* w; long long w_worker; int w_float;  // weights in fp32, or of the rows' type
    float eps, by_width;
    int norm;                                        // 0: rows are only put into 8 bits
    void* hidden; long long h_stride;
    void* out; long long out_stride;
    float* scale; float* rstd;
};

// Sum (or maximum) over the threads that own a row: a warp, or the block by way of `sh` (two halves used in turn, so that one
// barrier per sum is enough)
template <bool WARP, bool MAX>
__device__ __forceinline__ float over_row(float v, float (*sh)[16], int& turn) {
    v = MAX ? warp_max_f(v) : warp_sum_f(v);
    if (WARP) return v;
    float* s = sh[turn ^= 1];
    const int warps = blockDim.x >> 5;
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
    __syncthreads();
    v = s[0];
    for (int i = 1; i < warps; ++i) v = MAX ? max_nan(v, s[i]) : v + s[i];
    return v;
}

// the weights' type, as a constant for the code behind it (a branch per element, or all three forms and a choice, cost more than
// the norm's own arithmetic)
enum { NO_WEIGHT, FLOATS, LIKE_ROWS };
template <int W, class T, int V>
__device__ __forceinline__ void load_weight(float (&v)[V], const void* w, long long at) {
    if (W == NO_WEIGHT)
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = 1.0f;
    else if (W == FLOATS) load_floats<V>(v, static_cast<const float*>(w) + at);
    else load_vec<V>(v, static_cast<const T*>(w) + at);
}
#define QS_BY_WEIGHT(args, call)                                      \
    do {                                                              \
        if (!(args).w) call(NO_WEIGHT);                               \
        else if ((args).w_float) call(FLOATS);                        \
        else call(LIKE_ROWS);                                         \
    } while (0)
template <class T, int V> __device__ __forceinline__ Pack<T, V> load_streamed(const T* p) {      // read once: not kept in the L1
    Pack<T, V> q;
    if constexpr (sizeof(T) * V == 16) {
        const uint4 u = __ldcs(reinterpret_cast<const uint4*>(p));
        q = *reinterpret_cast<const Pack<T, V>*>(&u);
    } else {
        q.e[0] = __ldcs(p);
    }
    return q;
}

// y / s as fp32 rounds it: elements next to the middle of two 8-bit values are many (16-bit rows and weights give quotients of few bits), and
// a product with 1 / s put some of them on the other side.  By Markstein's step (Computation of elementary functions on the IBM
// RISC System/6000 processor, 1990): the product's rest y - q s is exact, and with it q is the rounded quotient.  Where that rest could leave
// the exponents' range, both are taken 2^64 times as large.  (us, bf16 8192 x 4096 and quantize of 8192 x 8192, and that of fp32: the
// product alone 43, 39, 56; the step 44, 42, 62; a division each 51, 56, 84)
struct Divisor { float s, inv, up; };
__device__ __forceinline__ Divisor divisor(float s) {
    const float up = s < 8.0779357e-28f ? 18446744073709551616.0f : 1.0f;    // 2^-90, 2^64
    return {s * up, 1.0f / (s * up), up};
}
template <int V>
__device__ __forceinline__ void divide(float (&v)[V], const Divisor& d) {
    if (d.up != 1.0f)
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] *= d.up;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const float q = v[j] * d.inv;
        v[j] = __fmaf_rn(__fmaf_rn(-q, d.s, v[j]), d.inv, q);
    }
}

// What follows the row's factor f: y = h f w, stored, or put into 8 bits
template <int W, class T, int V, int U, bool WARP, bool QUANT>
__device__ __forceinline__ void write_row(const NormArgs& a, const Pack<T, V> (&h)[U], float f, long long row, int t, int group, int vecs, float (*sh)[16], int& turn) {
    const long long w0 = blockIdx.y * a.w_worker;
    T* out = static_cast<T*>(a.out) + row * a.out_stride;
    float most = 0.0f, y[QUANT ? U : 1][V];          // (8 bits: y is held until the row's largest is known)
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int i = t + u * group;
        float(&v)[V] = y[QUANT ? u : 0];
        if (i < vecs) {
            float w[V];
            load_weight<W, T, V>(w, a.w, w0 + i * V);
            unpack(v, h[u]);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                v[j] = v[j] * f * w[j];
                if (QUANT) most = max_nan(most, fabsf(v[j]));
            }
            if (!QUANT) store_vec<V>(out + i * V, v);
        }
    }
    if (!QUANT) return;
    most = over_row<WARP, true>(most, sh, turn);
    // a row with a NaN or an infinity stands for NaN throughout
    const float s = most < __int_as_float(0x7f800000) ? fmaxf(most / E4M3_MAX, LEAST_SCALE) : quiet_nan();
    if (t == 0) a.scale[row] = s;
    const Divisor by = divisor(s);
    uint8_t* bytes = static_cast<uint8_t*>(a.out) + row * a.out_stride;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int i = t + u * group;
        float(&v)[V] = y[QUANT ? u : 0];
        if (i < vecs) {
            divide(v, by);
            store_e4m3<V>(bytes + i * V, v);
        }
    }
}

// A row per warp (four in a block) or per block, U vectors of V elements per thread, kept as they are stored until they are used
template <class T, int V, int U, bool WARP, bool QUANT>
__global__ void __launch_bounds__(WARP ? 128 : 512) norm_kernel(const NormArgs a) {
    __shared__ float sh[2][16];
    int turn = 0;
    const int group = WARP ? 32 : blockDim.x, t = WARP ? threadIdx.x & 31 : threadIdx.x;
    const long long n = WARP ? (long long)blockIdx.x * 4 + (threadIdx.x >> 5) : blockIdx.x;
    if (n >= a.N) return;                            // (whole warps, where a row is a warp's)
    const long long row = blockIdx.y * a.N + n;
    const int vecs = (int)(a.D / V);
    Pack<T, V> h[U];
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (t + u * group < vecs) h[u] = load_streamed<T, V>(x + (t + u * group) * V);
    if (a.res) {
        Pack<T, V> q[U];
        const T* res = static_cast<const T*>(a.res) + row * a.res_stride;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (t + u * group < vecs) q[u] = load_streamed<T, V>(res + (t + u * group) * V);
        T* hid = static_cast<T*>(a.hidden) + row * a.h_stride;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (t + u * group < vecs) {
                float v[V], r[V];
                unpack(v, h[u]);
                unpack(r, q[u]);
#pragma unroll
                for (int j = 0; j < V; ++j) v[j] += r[j];
                h[u] = pack_of<T, V>(v);
                *reinterpret_cast<Pack<T, V>*>(hid + (t + u * group) * V) = h[u];
            }
    }
    float f = 1.0f;
    if (a.norm) {
        float ss = 0.0f;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (t + u * group < vecs) {
                float v[V], part = 0.0f;
                unpack(v, h[u]);
#pragma unroll
                for (int j = 0; j < V; ++j) part = __fmaf_rn(v[j], v[j], part);
                ss += part;
            }
        f = rsqrtf(__fmaf_rn(over_row<WARP, false>(ss, sh, turn), a.by_width, a.eps));
        if (a.rstd && t == 0) a.rstd[row] = f;
    }
#define QS_WRITE(W) write_row<W, T, V, U, WARP, QUANT>(a, h, f, row, t, group, vecs, sh, turn)
    QS_BY_WEIGHT(a, QS_WRITE);
#undef QS_WRITE
}

// Rows too long for the registers of a block: read again for each step (from the L2, mostly), every element by one thread
template <int W, class T, int V, bool QUANT>
__device__ __forceinline__ void write_long_row(const NormArgs& a, const T* h_row, float f, long long row, float (*sh)[16], int& turn) {
    const long long vecs = a.D / V, w0 = blockIdx.y * a.w_worker;
    Divisor by = {1.0f, 1.0f, 1.0f};
    for (int pass = QUANT ? 0 : 1; pass < 2; ++pass) {
        float most = 0.0f;
        for (long long i = threadIdx.x; i < vecs; i += blockDim.x) {
            float h[V], w[V];
            load_vec<V>(h, h_row + i * V);
            load_weight<W, T, V>(w, a.w, w0 + i * V);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                h[j] = h[j] * f * w[j];
                if (QUANT && pass == 0) most = max_nan(most, fabsf(h[j]));
            }
            if (pass == 0) continue;
            if (QUANT) divide(h, by);
            if (QUANT) store_e4m3<V>(static_cast<uint8_t*>(a.out) + row * a.out_stride + i * V, h);
            else store_vec<V>(static_cast<T*>(a.out) + row * a.out_stride + i * V, h);
        }
        if (pass == 0) {
            most = over_row<false, true>(most, sh, turn);
            const float s = most < __int_as_float(0x7f800000) ? fmaxf(most / E4M3_MAX, LEAST_SCALE) : quiet_nan();
            if (threadIdx.x == 0) a.scale[row] = s;
            by = divisor(s);
        }
    }
}
template <class T, int V, bool QUANT>
__global__ void __launch_bounds__(512) norm_long_kernel(const NormArgs a) {
    __shared__ float sh[2][16];
    int turn = 0;
    const long long vecs = a.D / V;
    for (long long n = blockIdx.x; n < a.N; n += gridDim.x) {
        const long long row = blockIdx.y * a.N + n;
        const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
        const T* h_row = x;
        float ss = 0.0f;
        if (a.res) {
            const T* res = static_cast<const T*>(a.res) + row * a.res_stride;
            T* hid = static_cast<T*>(a.hidden) + row * a.h_stride;
#pragma unroll 4
            for (long long i = threadIdx.x; i < vecs; i += blockDim.x) {
                float h[V], r[V];
                load_vec<V>(h, x + i * V);
                load_vec<V>(r, res + i * V);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    h[j] = to_float(from_float<T>(h[j] + r[j]));
                    ss = __fmaf_rn(h[j], h[j], ss);
                }
                store_vec<V>(hid + i * V, h);
            }
            h_row = hid;
        } else if (a.norm) {
#pragma unroll 4
            for (long long i = threadIdx.x; i < vecs; i += blockDim.x) {
                float h[V];
                load_vec<V>(h, x + i * V);
#pragma unroll
                for (int j = 0; j < V; ++j) ss = __fmaf_rn(h[j], h[j], ss);
            }
        }
        float f = 1.0f;
        if (a.norm) {
            f = rsqrtf(__fmaf_rn(over_row<false, false>(ss, sh, turn), a.by_width, a.eps));
            if (a.rstd && threadIdx.x == 0) a.rstd[row] = f;
        }
#define QS_WRITE(W) write_long_row<W, T, V, QUANT>(a, h_row, f, row, sh, turn)
        QS_BY_WEIGHT(a, QS_WRITE);
#undef QS_WRITE
    }
}

// ------------------------------------------------------------------ gradient
struct NormGradArgs {
    int R;
    long long N, D;
    const void* g; long long g_stride;
    const void* h; long long h_stride;
    const float* rstd;
    const void* w; long long w_worker; int w_float;
    const void* gh; long long gh_stride;
    void* out; long long out_stride;
    float by_width;
    float* part;                                     // (R, parts, D) sums of g n over some of the rows, or null
    int parts;
    float* dw; long long dw_worker; int accumulate;
};

// Blocks stay: block (b, r) takes rows of worker r in turn (WARP: a row per warp) and keeps its columns' sums of the weights'
// gradient, and their weights, in registers; it leaves one row of partial sums.  (8 x 4096 x 1024 in bf16, fp32 weights: 49 us, 84 with the
// weights read again for every row)
template <int W, class T, int V, int U, bool WARP>
__device__ __forceinline__ void norm_grad_rows_of(const NormGradArgs& a, float (&dw)[U][V], float (*sh)[16], int t, int group, int vecs) {
    int turn = 0;
    float w[U][V];                                   // the block's columns' weights, once
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (t + u * group < vecs) load_weight<W, T, V>(w[u], a.w, blockIdx.y * a.w_worker + (t + u * group) * V);
    const long long first = WARP ? (long long)blockIdx.x * 4 + (threadIdx.x >> 5) : blockIdx.x;
    for (long long n = first; n < a.N; n += WARP ? (long long)gridDim.x * 4 : gridDim.x) {
        const long long row = blockIdx.y * a.N + n;
        Pack<T, V> h[U], g[U], gh[U];
        const float rstd = a.rstd[row];
        const T* hp = static_cast<const T*>(a.h) + row * a.h_stride;
        const T* gp = static_cast<const T*>(a.g) + row * a.g_stride;
        const T* ghp = static_cast<const T*>(a.gh) + row * a.gh_stride;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (t + u * group < vecs) {
                h[u] = load_streamed<T, V>(hp + (t + u * group) * V);
                g[u] = load_streamed<T, V>(gp + (t + u * group) * V);
            }
        if (a.gh)
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (t + u * group < vecs) gh[u] = load_streamed<T, V>(ghp + (t + u * group) * V);
        float dot = 0.0f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = t + u * group;
            if (i < vecs) {
                float hv[V], gv[V];
                unpack(hv, h[u]);
                unpack(gv, g[u]);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float n = hv[j] * rstd;
                    dw[u][j] = __fmaf_rn(gv[j], n, dw[u][j]);
                    dot = __fmaf_rn(gv[j] * w[u][j], n, dot);
                }
            }
        }
        const float along = over_row<WARP, false>(dot, sh, turn) * a.by_width * rstd * rstd;
        T* op = static_cast<T*>(a.out) + row * a.out_stride;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = t + u * group;
            if (i < vecs) {
                float hv[V], gv[V];
                unpack(hv, h[u]);
                unpack(gv, g[u]);
#pragma unroll
                for (int j = 0; j < V; ++j) gv[j] = __fmaf_rn(-along, hv[j], gv[j] * w[u][j] * rstd);
                if (a.gh) {
                    unpack(hv, gh[u]);
#pragma unroll
                    for (int j = 0; j < V; ++j) gv[j] += hv[j];
                }
                store_vec<V>(op + i * V, gv);
            }
        }
    }
}
template <class T, int V, int U, bool WARP>
__global__ void __launch_bounds__(WARP ? 128 : 512) norm_grad_kernel(const NormGradArgs a) {
    __shared__ float sh[2][16];
    extern __shared__ float joined[];                // WARP: (4, D) of the block's warps
    const int group = WARP ? 32 : blockDim.x, t = WARP ? threadIdx.x & 31 : threadIdx.x;
    const int vecs = (int)(a.D / V);
    float dw[U][V];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int j = 0; j < V; ++j) dw[u][j] = 0.0f;
#define QS_ROWS(W) norm_grad_rows_of<W, T, V, U, WARP>(a, dw, sh, t, group, vecs)
    QS_BY_WEIGHT(a, QS_ROWS);
#undef QS_ROWS
    if (!a.part) return;
    float* part = a.part + ((long long)blockIdx.y * a.parts + blockIdx.x) * a.D;
    float* to = WARP ? joined + (threadIdx.x >> 5) * a.D : part;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int i = t + u * group;
        if (i < vecs)
#pragma unroll
            for (int j = 0; j < V; ++j) to[i * V + j] = dw[u][j];
    }
    if (!WARP) return;
    __syncthreads();
    for (int i = threadIdx.x; i < (int)a.D; i += 128) part[i] = (joined[i] + joined[a.D + i]) + (joined[2 * a.D + i] + joined[3 * a.D + i]);
}

// Long rows, read twice
template <int W, class T, int V>
__device__ __forceinline__ void norm_grad_long_rows(const NormGradArgs& a, float (*sh)[16]) {
    int turn = 0;
    const long long vecs = a.D / V, w0 = blockIdx.y * a.w_worker;
    for (long long n = blockIdx.x; n < a.N; n += gridDim.x) {
        const long long row = blockIdx.y * a.N + n;
        const T* hp = static_cast<const T*>(a.h) + row * a.h_stride;
        const T* gp = static_cast<const T*>(a.g) + row * a.g_stride;
        const float rstd = a.rstd[row];
        float dot = 0.0f;
#pragma unroll 4
        for (long long i = threadIdx.x; i < vecs; i += blockDim.x) {
            float h[V], g[V], w[V];
            load_vec<V>(h, hp + i * V);
            load_vec<V>(g, gp + i * V);
            load_weight<W, T, V>(w, a.w, w0 + i * V);
#pragma unroll
            for (int j = 0; j < V; ++j) dot = __fmaf_rn(g[j] * w[j], h[j] * rstd, dot);
        }
        const float along = over_row<false, false>(dot, sh, turn) * a.by_width * rstd * rstd;
        for (long long i = threadIdx.x; i < vecs; i += blockDim.x) {
            float h[V], g[V], w[V];
            load_vec<V>(h, hp + i * V);
            load_vec<V>(g, gp + i * V);
            load_weight<W, T, V>(w, a.w, w0 + i * V);
#pragma unroll
            for (int j = 0; j < V; ++j) g[j] = __fmaf_rn(-along, h[j], g[j] * w[j] * rstd);
            if (a.gh) {
                load_vec<V>(h, static_cast<const T*>(a.gh) + row * a.gh_stride + i * V);
#pragma unroll
                for (int j = 0; j < V; ++j) g[j] += h[j];
            }
            store_vec<V>(static_cast<T*>(a.out) + row * a.out_stride + i * V, g);
        }
    }
}
template <class T, int V>
__global__ void __launch_bounds__(512) norm_grad_long_kernel(const NormGradArgs a) {
    __shared__ float sh[2][16];
#define QS_ROWS(W) norm_grad_long_rows<W, T, V>(a, sh)
    QS_BY_WEIGHT(a, QS_ROWS);
#undef QS_ROWS
}
// and the weights' gradient of such rows: a thread per column, block (x, p, r) the rows p, p + parts, ..
template <class T>
__global__ void __launch_bounds__(256) norm_dw_kernel(const NormGradArgs a) {
    const long long d = (long long)blockIdx.x * 256 + threadIdx.x;
    const int r = blockIdx.z;
    if (d >= a.D) return;
    float s = 0.0f;
    for (long long n = blockIdx.y; n < a.N; n += a.parts) {
        const long long row = r * a.N + n;
        const float v = to_float(static_cast<const T*>(a.h)[row * a.h_stride + d]) * a.rstd[row];
        s = __fmaf_rn(to_float(static_cast<const T*>(a.g)[row * a.g_stride + d]), v, s);
    }
    a.part[((long long)r * a.parts + blockIdx.y) * a.D + d] = s;
}

// ------------------------------------------------------------------ launches
// A row in the registers of `group` threads with up to `per` vectors each; 0: too long.  (32: a warp's, else a block's)
struct RowShape { int group, per; };
RowShape row_shape(long long vecs, int least, int most) {
    if (vecs <= 32 * least) return {32, vecs <= 32 * (least / 2) ? (vecs <= 32 * (least / 4) && least == 4 ? 1 : least / 2) : least};
    int g = 64;
    while (g < 512 && (long long)least * g < vecs) g *= 2;
    int per = least;
    while (per < most && (long long)per * g < vecs) per *= 2;
    return {g, (long long)per * g < vecs ? 0 : per};
}
// Loads in flight against registers: four vectors a thread for the norm, two for its gradient, which keeps sums as well (8192 x
// 4096 in bf16, us with 1, 2, 4 vectors: norm 40, 30, 26; with the residual 57, 49, 47; gradient 69, 66, 86).  Element by element
// what a row costs per thread counts most: eight.
template <int V> RowShape norm_shape(long long vecs) { return V == 1 ? row_shape(vecs, 8, 16) : row_shape(vecs, 4, 4); }
template <int V> RowShape grad_shape(long long vecs) { return V == 1 ? row_shape(vecs, 8, 16) : row_shape(vecs, 2, 4); }

template <class T, int V, bool QUANT, int U>
cudaError_t norm_by(const NormArgs& a, int group, cudaStream_t st) {
    if (group == 32) return launch(false, norm_kernel<T, V, U, true, QUANT>, dim3((unsigned)((a.N + 3) / 4), (unsigned)a.R), 128, 0, st, a);
    return launch(false, norm_kernel<T, V, U, false, QUANT>, dim3((unsigned)a.N, (unsigned)a.R), group, 0, st, a);
}
template <class T, int V, bool QUANT>
cudaError_t norm_of(const NormArgs& a, cudaStream_t st) {
    const RowShape s = norm_shape<V>(a.D / V);
    if constexpr (V == 1) {
        if (s.per == 4) return norm_by<T, V, QUANT, 4>(a, s.group, st);
        if (s.per == 8) return norm_by<T, V, QUANT, 8>(a, s.group, st);
        if (s.per == 16) return norm_by<T, V, QUANT, 16>(a, s.group, st);
    } else {
        if (s.per == 1) return norm_by<T, V, QUANT, 1>(a, s.group, st);
        if (s.per == 2) return norm_by<T, V, QUANT, 2>(a, s.group, st);
        if (s.per == 4) return norm_by<T, V, QUANT, 4>(a, s.group, st);
    }
    return launch(false, norm_long_kernel<T, V, QUANT>, dim3((unsigned)std::min<long long>(a.N, 1 << 20), (unsigned)a.R), 512, 0, st, a);
}
template <class T>
cudaError_t launch_norm(const NormArgs& a, bool vec, bool quant, cudaStream_t st) {
    constexpr int V = wide_of<T>();
    if (quant) return vec ? norm_of<T, V, true>(a, st) : norm_of<T, 1, true>(a, st);
    return vec ? norm_of<T, V, false>(a, st) : norm_of<T, 1, false>(a, st);
}

// Partial sums per worker: no more than there are rows, blocks that fit the GPU together, or 128 MB of them
constexpr int GRAD_BLOCKS = 148 * 16;
int grad_parts(int R, int64_t N, int64_t D) {
    return (int)std::max<long long>(1, std::min<long long>({N, (GRAD_BLOCKS + R - 1) / R, std::max<long long>(1, (32ll << 20) / (R * D))}));
}

template <class T, int V, int U, bool WARP>
cudaError_t norm_grad_by(NormGradArgs& a, int group, int sms, cudaStream_t st) {
    const int threads = WARP ? 128 : group;
    const unsigned smem = WARP ? (unsigned)(16 * a.D) : 0;
    int per_sm = 0;
    cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, norm_grad_kernel<T, V, U, WARP>, threads, smem);
    if (e != cudaSuccess) return e;
    // blocks that are there together, none more (one in a second round would double the time)
    const long long rows = WARP ? (a.N + 3) / 4 : a.N, there = (long long)sms * std::max(1, per_sm) / a.R;
    a.parts = (int)std::max<long long>(1, std::min<long long>({rows, (long long)a.parts, there}));
    return launch(false, norm_grad_kernel<T, V, U, WARP>, dim3((unsigned)a.parts, (unsigned)a.R), threads, smem, st, a);
}
template <class T, int V, int U>
cudaError_t norm_grad_rows(NormGradArgs& a, int group, int sms, cudaStream_t st) {
    return group == 32 ? norm_grad_by<T, V, U, true>(a, group, sms, st) : norm_grad_by<T, V, U, false>(a, group, sms, st);
}

template <class T, int V>
cudaError_t norm_grad_of(NormGradArgs a, int sms, cudaStream_t st) {
    const RowShape s = grad_shape<V>(a.D / V);
    cudaError_t e = cudaSuccess;
    if (s.per) {
        if constexpr (V == 1)
            e = s.per == 4 ? norm_grad_rows<T, V, 4>(a, s.group, sms, st) : s.per == 8 ? norm_grad_rows<T, V, 8>(a, s.group, sms, st) : norm_grad_rows<T, V, 16>(a, s.group, sms, st);
        else
            e = s.per == 1 ? norm_grad_rows<T, V, 1>(a, s.group, sms, st) : s.per == 2 ? norm_grad_rows<T, V, 2>(a, s.group, sms, st) : norm_grad_rows<T, V, 4>(a, s.group, sms, st);
    } else {
        // the weights' sums first: the rows' gradient may take g's place
        if (a.part) e = launch(false, norm_dw_kernel<T>, dim3((unsigned)((a.D + 255) / 256), (unsigned)a.parts, (unsigned)a.R), 256, 0, st, a);
        if (e == cudaSuccess) e = launch(false, norm_grad_long_kernel<T, V>, dim3((unsigned)std::min<long long>(a.N, 1 << 20), (unsigned)a.R), 512, 0, st, a);
    }
    if (e != cudaSuccess || !a.part) return e;
    return launch_join(true, a.part, a.parts, a.R, a.D, a.dw, a.dw_worker, a.accumulate, st);
}
template <class T>
cudaError_t launch_norm_grad(const NormGradArgs& a, bool vec, int sms, cudaStream_t st) {
    return vec ? norm_grad_of<T, wide_of<T>()>(a, sms, st) : norm_grad_of<T, 1>(a, sms, st);
}

bool bad_norm_shape(int R, int64_t N, int64_t D) { return R < 1 || R > 32 || N < 0 || D < 1; }
bool norm_too_large(int R, int64_t N, int64_t D) { return D > (1ll << 24) || N > (1ll << 30) || R * N > (1ll << 30); }
bool bad_rows(const void* p, int64_t stride, int64_t D, int size) { return stride < D || !aligned_to(p, size); }
bool bad_weight(const void* w, int weight_type, int type, int64_t worker_stride) {
    return w && ((weight_type != QS_F32 && weight_type != type) || worker_stride < 0 || !aligned_to(w, size_of_type(weight_type)));
}
bool weight_aligned(const void* w, int weight_type, int64_t worker_stride, int R) {
    return !w || (aligned_to(w, 16) && (R <= 1 || worker_stride * size_of_type(weight_type) % 16 == 0));
}

}  // namespace
}  // namespace qs

using namespace qs;

#define QS_NORM_BY_TYPE(launch, type, ...) \
    status_of((type) == QS_F32 ? launch<float>(__VA_ARGS__) : (type) == QS_BF16 ? launch<__nv_bfloat16>(__VA_ARGS__) : launch<__half>(__VA_ARGS__))

extern "C" {

int qs_rms_norm(int R, int64_t N, int64_t D, const void* x, int type, int64_t x_stride, const void* residual, int64_t residual_stride,
                const void* weight, int weight_type, int64_t weight_worker_stride, float eps, void* hidden, int64_t hidden_stride,
                void* out, int out_type, int64_t out_stride, float* scale, float* rstd, void* cuda_stream) {
    const int size = size_of_type(type);
    const bool quant = out_type == QS_E4M3;
    if (bad_norm_shape(R, N, D) || !size || (!quant && out_type != type) || !(eps > 0.0f) || !(eps < INFINITY)) return QS_INVALID_ARG;
    if (bad_weight(weight, weight_type, type, weight_worker_stride) || (residual != nullptr) != (hidden != nullptr)) return QS_INVALID_ARG;
    if (norm_too_large(R, N, D)) return QS_TOO_LARGE;
    const int64_t rows = R * N;
    if (rows == 0) return QS_OK;
    if (!x || !out || (quant && !scale) || bad_rows(x, x_stride, D, size) || (residual && bad_rows(residual, residual_stride, D, size)) ||
        (hidden && bad_rows(hidden, hidden_stride, D, size)) || bad_rows(out, out_stride, D, quant ? 1 : size) || !aligned_to(scale, 4) ||
        !aligned_to(rstd, 4)) return QS_INVALID_ARG;
    const int64_t out_bytes = span(rows, out_stride, D, quant ? 1 : size);
    if (!beside(x, x_stride, hidden, hidden_stride, rows, D, size) || !beside(residual, residual_stride, hidden, hidden_stride, rows, D, size))
        return QS_INVALID_ARG;
    if (quant) {
        if (!apart(out, out_bytes, x, span(rows, x_stride, D, size)) || !apart(out, out_bytes, residual, span(rows, residual_stride, D, size)) ||
            !apart(out, out_bytes, hidden, span(rows, hidden_stride, D, size))) return QS_INVALID_ARG;
    } else if (!beside(x, x_stride, out, out_stride, rows, D, size) || !beside(residual, residual_stride, out, out_stride, rows, D, size) ||
               (hidden && hidden == out) || !beside(hidden, hidden_stride, out, out_stride, rows, D, size)) {
        return QS_INVALID_ARG;
    }
    NormArgs a{};
    a.R = R; a.N = N; a.D = D; a.by_width = 1.0f / (float)D;
    a.x = x; a.x_stride = x_stride; a.res = residual; a.res_stride = residual_stride;
    a.w = weight; a.w_worker = weight_worker_stride; a.w_float = weight_type == QS_F32;
    a.eps = eps; a.norm = 1; a.hidden = hidden; a.h_stride = hidden_stride; a.out = out; a.out_stride = out_stride; a.scale = scale; a.rstd = rstd;
    const int V = 16 / size;
    const bool vec = D % V == 0 && rows_aligned(x, x_stride, rows, size, 16) && rows_aligned(residual, residual_stride, rows, size, 16) &&
                     rows_aligned(hidden, hidden_stride, rows, size, 16) && rows_aligned(out, out_stride, rows, quant ? 1 : size, quant ? V : 16) &&
                     weight_aligned(weight, weight_type, weight_worker_stride, R);
    return QS_NORM_BY_TYPE(launch_norm, type, a, vec, quant, static_cast<cudaStream_t>(cuda_stream));
}

int qs_quantize_rows(int64_t N, int64_t D, const void* x, int type, int64_t x_stride, void* out, int64_t out_stride, float* scale,
                     void* cuda_stream) {
    const int size = size_of_type(type);
    if (bad_norm_shape(1, N, D) || !size) return QS_INVALID_ARG;
    if (norm_too_large(1, N, D)) return QS_TOO_LARGE;
    if (N == 0) return QS_OK;
    if (!x || !out || !scale || bad_rows(x, x_stride, D, size) || out_stride < D || !aligned_to(scale, 4) ||
        !apart(out, span(N, out_stride, D, 1), x, span(N, x_stride, D, size))) return QS_INVALID_ARG;
    NormArgs a{};
    a.R = 1; a.N = N; a.D = D; a.x = x; a.x_stride = x_stride; a.out = out; a.out_stride = out_stride; a.scale = scale;
    const int V = 16 / size;
    const bool vec = D % V == 0 && rows_aligned(x, x_stride, N, size, 16) && rows_aligned(out, out_stride, N, 1, V);
    return QS_NORM_BY_TYPE(launch_norm, type, a, vec, true, static_cast<cudaStream_t>(cuda_stream));
}

int64_t qs_rms_norm_grad_bytes(int R, int64_t N, int64_t D) {
    if (bad_norm_shape(R, N, D)) return QS_INVALID_ARG;
    if (norm_too_large(R, N, D)) return QS_TOO_LARGE;
    return 4 * (int64_t)R * grad_parts(R, N, D) * D;
}

int qs_rms_norm_grad(int R, int64_t N, int64_t D, const void* grad, int type, int64_t grad_stride, const void* hidden, int64_t hidden_stride,
                     const float* rstd, const void* weight, int weight_type, int64_t weight_worker_stride, const void* grad_hidden,
                     int64_t grad_hidden_stride, void* out, int64_t out_stride, float* grad_weight, int64_t grad_weight_worker_stride,
                     int accumulate, void* work, int64_t work_bytes, void* cuda_stream) {
    const int size = size_of_type(type);
    if (bad_norm_shape(R, N, D) || !size || bad_weight(weight, weight_type, type, weight_worker_stride)) return QS_INVALID_ARG;
    if (norm_too_large(R, N, D)) return QS_TOO_LARGE;
    if (grad_weight && (!aligned_to(grad_weight, 4) || (R > 1 && grad_weight_worker_stride < D))) return QS_INVALID_ARG;
    const int64_t rows = R * N;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (rows == 0) {
        if (!grad_weight || accumulate) return QS_OK;
        return status_of(launch_join(false, nullptr, 0, R, D, grad_weight, grad_weight_worker_stride, 0, st));
    }
    if (!grad || !hidden || !rstd || !out || !aligned_to(rstd, 4) || bad_rows(grad, grad_stride, D, size) || bad_rows(hidden, hidden_stride, D, size) ||
        (grad_hidden && bad_rows(grad_hidden, grad_hidden_stride, D, size)) || bad_rows(out, out_stride, D, size)) return QS_INVALID_ARG;
    if (!beside(grad, grad_stride, out, out_stride, rows, D, size) || !beside(hidden, hidden_stride, out, out_stride, rows, D, size) ||
        !beside(grad_hidden, grad_hidden_stride, out, out_stride, rows, D, size)) return QS_INVALID_ARG;
    if (grad_weight && (!work || !aligned_to(work, 16))) return QS_INVALID_ARG;
    if (grad_weight && work_bytes < 4 * (int64_t)R * grad_parts(R, N, D) * D) return QS_CAPACITY;
    const int sms = sm_count();
    if (!sms) return QS_CUDA;
    NormGradArgs a{};
    a.R = R; a.N = N; a.D = D; a.by_width = 1.0f / (float)D; a.g = grad; a.g_stride = grad_stride; a.h = hidden; a.h_stride = hidden_stride; a.rstd = rstd;
    a.w = weight; a.w_worker = weight_worker_stride; a.w_float = weight_type == QS_F32; a.gh = grad_hidden; a.gh_stride = grad_hidden_stride;
    a.out = out; a.out_stride = out_stride; a.part = grad_weight ? static_cast<float*>(work) : nullptr; a.parts = grad_parts(R, N, D);
    a.dw = grad_weight; a.dw_worker = grad_weight_worker_stride; a.accumulate = accumulate;
    const int V = 16 / size;
    const bool vec = D % V == 0 && rows_aligned(grad, grad_stride, rows, size, 16) && rows_aligned(hidden, hidden_stride, rows, size, 16) &&
                     rows_aligned(grad_hidden, grad_hidden_stride, rows, size, 16) && rows_aligned(out, out_stride, rows, size, 16) &&
                     weight_aligned(weight, weight_type, weight_worker_stride, R);
    return QS_NORM_BY_TYPE(launch_norm_grad, type, a, vec, sms, st);
}

}  // extern "C"
