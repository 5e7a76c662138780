// Dropout from the counter-based generator: no mask is stored, the backward pass draws the same words again.
//
//   out = residual + (word >= T ? c x : 0),   T = floor(p 2^32),  c = 1 / (1 - p)
//
// with one Philox4x32-10 word per element: key = the seed, counter = (element >> 2, worker, round's low half,
// layer << 16 | round's bits 32 to 39 << 8 | 2), word = out[element & 3]; 2 is this operator's stream beside those of
// the sparsifier and the quantizer.  A row is read and written once by vectors of 16 bytes (two or one draws of four words
// each); the generator's ten rounds keep about half of the issue slots busy while memory sets the pace.
#include <algorithm>

#include "qs_common.cuh"
#include "qs_vec.cuh"

namespace qs {
namespace {

struct DropArgs {
    long long rows, per, D;                          // rows in all, rows of one worker, elements of a row
    const void* x; long long x_stride;
    const void* res; long long res_stride;
    void* out; long long out_stride;
    uint32_t seed_lo, seed_hi, round_lo, word3, worker, threshold;
    float c;
    long long vecs;                                  // work items of a row (vectors), or of a worker (groups of four)
};

__device__ __forceinline__ uint4 words_of(const DropArgs& a, uint32_t worker, uint32_t quad) {
    return philox4x32_10(make_uint4(quad, a.worker + worker, a.round_lo, a.word3), make_uint2(a.seed_lo, a.seed_hi));
}
__device__ __forceinline__ float dropped(const DropArgs& a, float x, uint32_t word) { return word >= a.threshold ? x * a.c : 0.0f; }

// Rows whose elements come in vectors of V, the first of each at a multiple of four elements of its worker
template <class T, int V, int U, bool RES>
__global__ void __launch_bounds__(256) dropout_kernel(const DropArgs a) {
    const long long items = a.rows * a.vecs, step = (long long)gridDim.x * 256;
    for (long long i0 = (long long)blockIdx.x * 256 + threadIdx.x; i0 < items; i0 += step * U) {
        float x[U][V], res[U][V];
        long long row[U], at[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long i = i0 + u * step;
            row[u] = a.rows == 1 ? 0 : i / a.vecs;
            at[u] = (i - row[u] * a.vecs) * V;
            if (i >= items || at[u] + V > a.D) continue;
            load_vec<V>(x[u], static_cast<const T*>(a.x) + row[u] * a.x_stride + at[u]);
            if (RES) load_vec<V>(res[u], static_cast<const T*>(a.res) + row[u] * a.res_stride + at[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i0 + u * step >= items) break;
            const long long w = a.per == 1 ? row[u] : row[u] / a.per, e = (row[u] - w * a.per) * a.D + at[u];
            const bool whole = at[u] + V <= a.D;
            if (!whole) {                            // the row's last elements
                const T* p = static_cast<const T*>(a.x) + row[u] * a.x_stride + at[u];
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    x[u][j] = at[u] + j < a.D ? to_float(p[j]) : 0.0f;
                    if (RES) res[u][j] = at[u] + j < a.D ? to_float(static_cast<const T*>(a.res)[row[u] * a.res_stride + at[u] + j]) : 0.0f;
                }
            }
#pragma unroll
            for (int j = 0; j < V; j += 4) {
                const uint4 r = words_of(a, (uint32_t)w, (uint32_t)((e + j) >> 2));
                const uint32_t word[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float v = dropped(a, x[u][j + k], word[k]);
                    x[u][j + k] = RES ? v + res[u][j + k] : v;
                }
            }
            T* o = static_cast<T*>(a.out) + row[u] * a.out_stride + at[u];
            if (whole) {
                store_vec<V>(o, x[u]);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (at[u] + j < a.D) o[j] = from_float<T>(x[u][j]);
            }
        }
    }
}

// Any rows: a thread per draw of four words, whose elements may lie in two rows or more
template <class T, bool RES>
__global__ void __launch_bounds__(256) dropout_loose_kernel(const DropArgs a) {
    const long long workers = a.rows / a.per, items = workers * a.vecs, count = a.per * a.D;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < items; i += (long long)gridDim.x * 256) {
        const long long w = i / a.vecs, e = (i - w * a.vecs) * 4;
        long long row = e / a.D, d = e - row * a.D;
        row += w * a.per;
        const uint4 r = words_of(a, (uint32_t)w, (uint32_t)(e >> 2));
        const uint32_t word[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (e + k >= count) break;
            float v = dropped(a, to_float(static_cast<const T*>(a.x)[row * a.x_stride + d]), word[k]);
            if (RES) v += to_float(static_cast<const T*>(a.res)[row * a.res_stride + d]);
            static_cast<T*>(a.out)[row * a.out_stride + d] = from_float<T>(v);
            if (++d == a.D) d = 0, ++row;
        }
    }
}

template <class T>
cudaError_t launch_dropout(DropArgs a, cudaStream_t st) {
    constexpr int V = wide_of<T>(), size = sizeof(T);
    // Rows that lie side by side are one row per worker, and one worker's one row
    if ((a.per == 1 || (a.x_stride == a.D && a.out_stride == a.D && (!a.res || a.res_stride == a.D)))) {
        const long long workers = a.rows / a.per;
        if (a.per > 1) a.D *= a.per, a.rows = workers, a.per = 1, a.x_stride = a.out_stride = a.res_stride = a.D;
    }
    const bool vec = rows_aligned(a.x, a.x_stride, a.rows, size, 16) && rows_aligned(a.res, a.res_stride, a.rows, size, 16) &&
                     rows_aligned(a.out, a.out_stride, a.rows, size, 16) && (a.per == 1 || a.D % 4 == 0);
    a.vecs = vec ? (a.D + V - 1) / V : (a.per * a.D + 3) / 4;
    const long long items = vec ? a.rows * a.vecs : a.rows / a.per * a.vecs;
    constexpr int U = 2;
    const long long blocks = std::min<long long>((items + 255) / 256, 148 * 64);
    const dim3 grid((unsigned)blocks);
    if (vec) return a.res ? launch(false, dropout_kernel<T, V, U, true>, grid, 256, 0, st, a) : launch(false, dropout_kernel<T, V, U, false>, grid, 256, 0, st, a);
    return a.res ? launch(false, dropout_loose_kernel<T, true>, grid, 256, 0, st, a) : launch(false, dropout_loose_kernel<T, false>, grid, 256, 0, st, a);
}

}  // namespace
}  // namespace qs

using namespace qs;

extern "C" {

int qs_dropout(int R, int64_t N, int64_t D, const void* x, int type, int64_t x_stride, const void* residual, int64_t residual_stride, double p,
               uint64_t seed, uint64_t round, int worker, int layer, void* out, int64_t out_stride, void* cuda_stream) {
    const int size = size_of_type(type);
    if (R < 1 || R > 32 || N < 0 || D < 1 || !size || !(p >= 0.0 && p < 1.0) || round >= 1ull << 40 || worker < 0 || layer < 0 || layer > 65535)
        return QS_INVALID_ARG;
    if (N > (1ll << 30) || D > (1ll << 30) || N * D > (1ll << 34) || R * N > (1ll << 30)) return QS_TOO_LARGE;
    const int64_t rows = R * N;
    if (rows == 0) return QS_OK;
    if (!x || !out || x_stride < D || out_stride < D || (residual && residual_stride < D) || !aligned_to(x, size) || !aligned_to(residual, size) ||
        !aligned_to(out, size) || !beside(x, x_stride, out, out_stride, rows, D, size) ||
        !beside(residual, residual_stride, out, out_stride, rows, D, size)) return QS_INVALID_ARG;
    DropArgs a{};
    a.rows = rows; a.per = N; a.D = D; a.x = x; a.x_stride = x_stride; a.res = residual; a.res_stride = residual_stride; a.out = out;
    a.out_stride = out_stride;
    a.seed_lo = (uint32_t)seed; a.seed_hi = (uint32_t)(seed >> 32); a.round_lo = (uint32_t)round;
    a.word3 = (uint32_t)layer << 16 | (uint32_t)(round >> 32) << 8 | 2u;
    a.worker = (uint32_t)worker; a.threshold = (uint32_t)(p * 4294967296.0); a.c = (float)(1.0 / (1.0 - p));
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    return status_of(type == QS_F32 ? launch_dropout<float>(a, st) : type == QS_BF16 ? launch_dropout<__nv_bfloat16>(a, st) : launch_dropout<__half>(a, st));
}

}  // extern "C"
