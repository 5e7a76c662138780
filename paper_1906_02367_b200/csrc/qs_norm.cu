// Root-mean-square norm of rows, with the residual's addition in front of it and 8 bits behind it, and its gradient.
//
//   h = x + residual (rounded to the type of x: what the backward pass reads);  rstd = (mean h^2 + eps)^(-1/2)
//   y = h rstd w;  in 8 bits q = e4m3(y / s), s = max(max |y| / 448, 2^-126)
//   dh = grad_hidden + rstd (w g - n mean(w g n)),  n = h rstd;   dw = sum over the rows of g n
//
// Memory-bound: a row is read once, kept in the registers of a warp (short rows) or a block, and written once.
#include <algorithm>

#include "qs_parts.cuh"

namespace qs {
namespace {

constexpr float E4M3_MAX = 448.0f;
constexpr float LEAST_SCALE = 1.17549435e-38f;       // 2^-126: its reciprocal is finite

struct NormArgs {
    long long rows, N, D;                            // R N rows
    const void* x; long long x_stride;
    const void* res; long long res_stride;
    const void* w; long long w_worker; int w_float;  // weights in fp32, or of the rows' type
    float eps;
    int norm;                                        // 0: rows are only put into 8 bits
    void* hidden; long long h_stride;
    void* out; long long out_stride;
    float* scale; float* rstd;
};

// Sum (or maximum) over the group that owns a row: a warp, or the block by way of `sh` (two halves used in turn, so that
// one barrier per sum is enough)
template <bool WARP, bool MAX>
__device__ __forceinline__ float over_row(float v, float* sh, int& turn) {
    v = MAX ? warp_max_f(v) : warp_sum_f(v);
    if (WARP) return v;
    float* s = sh + (turn ^= 32);
    const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0) s[threadIdx.x >> 5] = v;
    __syncthreads();
    v = lane < warps ? s[lane] : 0.0f;               // (a maximum of magnitudes)
    return MAX ? warp_max_f(v) : warp_sum_f(v);
}

template <class T, int V>
__device__ __forceinline__ void load_weight(float (&v)[V], const void* w, int w_float, long long at) {
    if (!w) {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = 1.0f;
    } else if (w_float) {
        load_floats<V>(v, static_cast<const float*>(w) + at);
    } else {
        load_vec<V>(v, static_cast<const T*>(w) + at);
    }
}

// U vectors of V elements per thread; WARP: a row per warp, else a row per block
template <class T, int V, int U, bool WARP, bool QUANT>
__global__ void __launch_bounds__(WARP ? 128 : 512) norm_kernel(const NormArgs a) {
    __shared__ float sh[64];
    int turn = 0;
    const int group = WARP ? 32 : blockDim.x, t = WARP ? threadIdx.x & 31 : threadIdx.x;
    const long long row = WARP ? (long long)blockIdx.x * 4 + (threadIdx.x >> 5) : blockIdx.x;
    if (row >= a.rows) return;                       // (whole warps, where a row is a warp's)
    const long long vecs = a.D / V;
    float h[U][V], r[U][V];
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const long long i = t + (long long)u * group;
        if (i < vecs) load_vec<V>(h[u], x + i * V);
    }
    if (a.res) {
        const T* res = static_cast<const T*>(a.res) + row * a.res_stride;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long i = t + (long long)u * group;
            if (i < vecs) load_vec<V>(r[u], res + i * V);
        }
        T* hid = static_cast<T*>(a.hidden) + row * a.h_stride;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long i = t + (long long)u * group;
            if (i < vecs) {
#pragma unroll
                for (int j = 0; j < V; ++j) h[u][j] = to_float(from_float<T>(h[u][j] + r[u][j]));
                store_vec<V>(hid + i * V, h[u]);
            }
        }
    }
    float f = 1.0f;
    if (a.norm) {
        float ss = 0.0f;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (t + (long long)u * group < vecs) {
                float part = 0.0f;
#pragma unroll
                for (int j = 0; j < V; ++j) part = __fmaf_rn(h[u][j], h[u][j], part);
                ss += part;
            }
        ss = over_row<WARP, false>(ss, sh, turn);
        f = 1.0f / sqrtf(ss / (float)a.D + a.eps);
        if (a.rstd && t == 0) a.rstd[row] = f;
    }
    const long long w0 = a.w ? row / a.N * a.w_worker : 0;
    float most = 0.0f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const long long i = t + (long long)u * group;
        if (i < vecs) {
            float w[V];
            load_weight<T, V>(w, a.w, a.w_float, w0 + i * V);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                if (a.norm) h[u][j] = h[u][j] * f * w[j];
                if (QUANT) most = max_nan(most, fabsf(h[u][j]));
            }
            if (!QUANT) store_vec<V>(static_cast<T*>(a.out) + row * a.out_stride + i * V, h[u]);
        }
    }
    if (!QUANT) return;
    most = over_row<WARP, true>(most, sh, turn);
    // a row with a NaN or an infinity stands for NaN throughout
    const float s = most < __int_as_float(0x7f800000) ? fmaxf(most / E4M3_MAX, LEAST_SCALE) : quiet_nan();
    if (t == 0) a.scale[row] = s;
    const float inv = 1.0f / s;
    uint8_t* out = static_cast<uint8_t*>(a.out) + row * a.out_stride;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const long long i = t + (long long)u * group;
        if (i < vecs) {
#pragma unroll
            for (int j = 0; j < V; ++j) h[u][j] *= inv;
            store_e4m3<V>(out + i * V, h[u]);
        }
    }
}

// Rows too long for the registers of a block: read again for each step (from the L2, mostly), every element by one thread
template <class T, int V, bool QUANT>
__global__ void __launch_bounds__(1024) norm_long_kernel(const NormArgs a) {
    __shared__ float sh[64];
    int turn = 0;
    const long long vecs = a.D / V, w_step = a.w_worker;
    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
        const T* h_row = x;
        float ss = 0.0f;
        if (a.res) {
            const T* res = static_cast<const T*>(a.res) + row * a.res_stride;
            T* hid = static_cast<T*>(a.hidden) + row * a.h_stride;
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
            for (long long i = threadIdx.x; i < vecs; i += blockDim.x) {
                float h[V];
                load_vec<V>(h, x + i * V);
#pragma unroll
                for (int j = 0; j < V; ++j) ss = __fmaf_rn(h[j], h[j], ss);
            }
        }
        float f = 1.0f;
        if (a.norm) {
            f = 1.0f / sqrtf(over_row<false, false>(ss, sh, turn) / (float)a.D + a.eps);
            if (a.rstd && threadIdx.x == 0) a.rstd[row] = f;
        }
        const long long w0 = a.w ? row / a.N * w_step : 0;
        float s = 1.0f, inv = 1.0f;
        for (int pass = QUANT ? 0 : 1; pass < 2; ++pass) {
            float most = 0.0f;
            for (long long i = threadIdx.x; i < vecs; i += blockDim.x) {
                float h[V], w[V];
                load_vec<V>(h, h_row + i * V);
                load_weight<T, V>(w, a.w, a.w_float, w0 + i * V);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    if (a.norm) h[j] = h[j] * f * w[j];
                    most = max_nan(most, fabsf(h[j]));
                    if (QUANT) h[j] *= inv;
                }
                if (pass == 0) continue;
                if (QUANT) store_e4m3<V>(static_cast<uint8_t*>(a.out) + row * a.out_stride + i * V, h);
                else store_vec<V>(static_cast<T*>(a.out) + row * a.out_stride + i * V, h);
            }
            if (pass == 0) {
                most = over_row<false, true>(most, sh, turn);
                s = most < __int_as_float(0x7f800000) ? fmaxf(most / E4M3_MAX, LEAST_SCALE) : quiet_nan();
                if (threadIdx.x == 0) a.scale[row] = s;
                inv = 1.0f / s;
            }
        }
        __syncthreads();                             // (the sums' halves are used again)
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
    float* part;                                     // (R, parts, D) sums of g n over some of the rows, or null
    int parts;
    float* dw; long long dw_worker; int accumulate;
};

// Blocks stay: block (b, r) takes worker r's rows b, b + gridDim.x, .. (WARP: a warp each four-th of them) and keeps its
// columns' sums of the weights' gradient in registers; one row of partial sums per block.
template <class T, int V, int U, bool WARP>
__global__ void __launch_bounds__(WARP ? 128 : 512) norm_grad_kernel(const NormGradArgs a) {
    __shared__ float sh[64];
    extern __shared__ float warps_dw[];              // WARP: (4, D) of the block's warps
    int turn = 0;
    const int group = WARP ? 32 : blockDim.x, t = WARP ? threadIdx.x & 31 : threadIdx.x, r = blockIdx.y;
    const long long vecs = a.D / V;
    const long long first = WARP ? (long long)blockIdx.x * 4 + (threadIdx.x >> 5) : blockIdx.x, step = WARP ? (long long)gridDim.x * 4 : gridDim.x;
    float dw[U][V];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int j = 0; j < V; ++j) dw[u][j] = 0.0f;
    const float by_width = 1.0f / (float)a.D;
    for (long long n = first; n < a.N; n += step) {
        const long long row = r * a.N + n;
        float h[U][V], g[U][V];
        const float rstd = a.rstd[row];
        const T* hp = static_cast<const T*>(a.h) + row * a.h_stride;
        const T* gp = static_cast<const T*>(a.g) + row * a.g_stride;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long i = t + (long long)u * group;
            if (i < vecs) {
                load_vec<V>(h[u], hp + i * V);
                load_vec<V>(g[u], gp + i * V);
            }
        }
        float dot = 0.0f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long i = t + (long long)u * group;
            if (i < vecs) {
                float w[V];
                load_weight<T, V>(w, a.w, a.w_float, r * a.w_worker + i * V);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    h[u][j] *= rstd;
                    dw[u][j] = __fmaf_rn(g[u][j], h[u][j], dw[u][j]);
                    g[u][j] *= w[j];
                    dot = __fmaf_rn(g[u][j], h[u][j], dot);
                }
            }
        }
        const float mean = over_row<WARP, false>(dot, sh, turn) * by_width;
        T* op = static_cast<T*>(a.out) + row * a.out_stride;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long i = t + (long long)u * group;
            if (i < vecs) {
                float gh[V];
                if (a.gh) load_vec<V>(gh, static_cast<const T*>(a.gh) + row * a.gh_stride + i * V);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float d = rstd * (g[u][j] - h[u][j] * mean);
                    g[u][j] = a.gh ? d + gh[j] : d;
                }
                store_vec<V>(op + i * V, g[u]);
            }
        }
    }
    if (!a.part) return;
    float* part = a.part + ((long long)r * a.parts + blockIdx.x) * a.D;
    if (WARP) {
        float* mine = warps_dw + (threadIdx.x >> 5) * a.D;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long i = t + (long long)u * 32;
            if (i < vecs)
#pragma unroll
                for (int j = 0; j < V; ++j) mine[i * V + j] = dw[u][j];
        }
        __syncthreads();
        for (long long i = threadIdx.x; i < a.D; i += 128)
            part[i] = (warps_dw[i] + warps_dw[a.D + i]) + (warps_dw[2 * a.D + i] + warps_dw[3 * a.D + i]);
    } else {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long i = t + (long long)u * group;
            if (i < vecs)
#pragma unroll
                for (int j = 0; j < V; ++j) part[i * V + j] = dw[u][j];
        }
    }
}

// Long rows, read twice
template <class T, int V>
__global__ void __launch_bounds__(1024) norm_grad_long_kernel(const NormGradArgs a) {
    __shared__ float sh[64];
    int turn = 0;
    const long long vecs = a.D / V;
    const float by_width = 1.0f / (float)a.D;
    for (long long row = blockIdx.x; row < a.R * a.N; row += gridDim.x) {
        const long long w0 = row / a.N * a.w_worker;
        const T* hp = static_cast<const T*>(a.h) + row * a.h_stride;
        const T* gp = static_cast<const T*>(a.g) + row * a.g_stride;
        const float rstd = a.rstd[row];
        float dot = 0.0f;
        for (long long i = threadIdx.x; i < vecs; i += blockDim.x) {
            float h[V], g[V], w[V];
            load_vec<V>(h, hp + i * V);
            load_vec<V>(g, gp + i * V);
            load_weight<T, V>(w, a.w, a.w_float, w0 + i * V);
#pragma unroll
            for (int j = 0; j < V; ++j) dot = __fmaf_rn(g[j] * w[j], h[j] * rstd, dot);
        }
        const float mean = over_row<false, false>(dot, sh, turn) * by_width;
        for (long long i = threadIdx.x; i < vecs; i += blockDim.x) {
            float h[V], g[V], w[V], gh[V];
            load_vec<V>(h, hp + i * V);
            load_vec<V>(g, gp + i * V);
            load_weight<T, V>(w, a.w, a.w_float, w0 + i * V);
            if (a.gh) load_vec<V>(gh, static_cast<const T*>(a.gh) + row * a.gh_stride + i * V);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float d = rstd * (g[j] * w[j] - h[j] * rstd * mean);
                g[j] = a.gh ? d + gh[j] : d;
            }
            store_vec<V>(static_cast<T*>(a.out) + row * a.out_stride + i * V, g);
        }
    }
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
// A row in registers: `group` threads with `per` vectors each; 0 vectors: too long.  Two vectors a thread keep enough loads
// in flight with blocks small enough that several share an SM.
struct RowShape { int group, per; };
RowShape row_shape(long long vecs, int most_per) {
    if (vecs <= 32) return {32, 1};
    if (vecs <= 64) return {32, 2};
    int g = 64;
    while (g < 512 && 2 * g < vecs) g *= 2;
    int per = 1;
    while (per < most_per && (long long)per * g < vecs) per *= 2;
    return {g, (long long)per * g < vecs ? 0 : per};
}

template <class T, int V, bool QUANT>
cudaError_t norm_of(const NormArgs& a, cudaStream_t st) {
    const RowShape s = row_shape(a.D / V, V == 1 ? 8 : 4);
    if (s.per && s.group == 32) {
        const dim3 grid((unsigned)((a.rows + 3) / 4));
        return s.per == 1 ? launch(false, norm_kernel<T, V, 1, true, QUANT>, grid, 128, 0, st, a)
                          : launch(false, norm_kernel<T, V, 2, true, QUANT>, grid, 128, 0, st, a);
    }
    const dim3 grid((unsigned)a.rows);
    switch (s.per) {
    case 1: return launch(false, norm_kernel<T, V, 1, false, QUANT>, grid, s.group, 0, st, a);
    case 2: return launch(false, norm_kernel<T, V, 2, false, QUANT>, grid, s.group, 0, st, a);
    case 4: return launch(false, norm_kernel<T, V, 4, false, QUANT>, grid, s.group, 0, st, a);
    case 8: return launch(false, norm_kernel<T, 1, 8, false, QUANT>, grid, s.group, 0, st, a);
    }
    return launch(false, norm_long_kernel<T, V, QUANT>, dim3((unsigned)std::min<long long>(a.rows, 1 << 20)), 1024, 0, st, a);
}
template <class T>
cudaError_t launch_norm(const NormArgs& a, bool vec, bool quant, cudaStream_t st) {
    constexpr int V = wide_of<T>();
    if (quant) return vec ? norm_of<T, V, true>(a, st) : norm_of<T, 1, true>(a, st);
    return vec ? norm_of<T, V, false>(a, st) : norm_of<T, 1, false>(a, st);
}

// Partial sums per worker: enough blocks to fill the GPU, no more than there are rows (or groups of four)
int grad_parts(int R, int64_t N, int64_t D) {
    const long long want = (148 * 8 + R - 1) / R;
    return (int)std::max<long long>(1, std::min<long long>(N, std::min<long long>(want, std::max<long long>(1, (32ll << 20) / (R * D)))));
}

template <class T, int V>
cudaError_t norm_grad_of(NormGradArgs a, int sms, cudaStream_t st) {
    const RowShape s = row_shape(a.D / V, V == 1 ? 8 : 4);
    const int most = a.parts;
    cudaError_t e;
    if (s.per) {
        // blocks that fit the GPU together: more would only make more partial sums
        const bool warp = s.group == 32;
        const int threads = warp ? 128 : s.group, per_sm = std::max(1, 1024 / threads);
        const long long rows = warp ? (a.N + 3) / 4 : a.N;
        a.parts = (int)std::max<long long>(1, std::min<long long>({rows, (long long)most, (long long)(sms * per_sm + a.R - 1) / a.R}));
        const dim3 grid((unsigned)a.parts, (unsigned)a.R);
        const unsigned smem = warp ? (unsigned)(16 * a.D) : 0;
        if (warp) e = s.per == 1 ? launch(false, norm_grad_kernel<T, V, 1, true>, grid, 128, smem, st, a) : launch(false, norm_grad_kernel<T, V, 2, true>, grid, 128, smem, st, a);
        else if (s.per == 1) e = launch(false, norm_grad_kernel<T, V, 1, false>, grid, s.group, 0, st, a);
        else if (s.per == 2) e = launch(false, norm_grad_kernel<T, V, 2, false>, grid, s.group, 0, st, a);
        else if (s.per == 4) e = launch(false, norm_grad_kernel<T, V, 4, false>, grid, s.group, 0, st, a);
        else e = launch(false, norm_grad_kernel<T, 1, 8, false>, grid, s.group, 0, st, a);
    } else {
        // the weights' sums first: the rows' gradient may take g's place
        e = cudaSuccess;
        if (a.part) e = launch(false, norm_dw_kernel<T>, dim3((unsigned)((a.D + 255) / 256), (unsigned)a.parts, (unsigned)a.R), 256, 0, st, a);
        if (e == cudaSuccess) e = launch(false, norm_grad_long_kernel<T, V>, dim3((unsigned)std::min<long long>(a.R * a.N, 1 << 20)), 1024, 0, st, a);
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
    a.rows = rows; a.N = N; a.D = D;
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
    a.rows = N; a.N = N; a.D = D; a.x = x; a.x_stride = x_stride; a.out = out; a.out_stride = out_stride; a.scale = scale;
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
    a.R = R; a.N = N; a.D = D; a.g = grad; a.g_stride = grad_stride; a.h = hidden; a.h_stride = hidden_stride; a.rstd = rstd;
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
