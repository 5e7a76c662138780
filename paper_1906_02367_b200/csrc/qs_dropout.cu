// Dropout from the counter-based generator: no mask is stored, the backward pass draws the same words again.
//
//   out = residual + (word >= T ? c x : 0),   T = floor(p 2^32),  c = 1 / (1 - p)
//
// with one Philox4x32-10 word per element: key = the seed, counter = (element >> 2, worker, round's low half,
// layer << 16 | round's bits 32 to 39 << 8 | 2), word = out[element & 3]; 2 is this operator's stream beside those of
// the sparsifier and the quantizer.  A row is read and written once by vectors of 16 bytes, each with one or two draws of four
// words.  In fp32 memory sets the pace (6.7 TB/s); in 16 bits the generator does as much: ten rounds are about 20 of the 25
// instructions per element, and the multipliers and the logic units are each about half busy (5.0 to 5.3 TB/s).
#include <algorithm>

#include "qs_vec.cuh"

namespace qs {
namespace {

struct DropArgs {
    long long rows, per, D;                          // rows in all, rows of one worker, elements of a row
    const void* x; long long x_stride;
    const void* res; long long res_stride;
    void* out; long long out_stride;
    uint2 key[10];                                   // of the rounds
    uint32_t round_lo, word3, worker, threshold;
    float c;
    long long vecs, items;                           // work items of a row (vectors), or of a worker (groups of four); of all
};

// Philox4x32-10 with the ten round keys at hand: two wide products and two xors a round
__device__ __forceinline__ uint4 words_of(const DropArgs& a, uint32_t worker, uint32_t quad) {
    uint4 c = make_uint4(quad, a.worker + worker, a.round_lo, a.word3);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const unsigned long long p0 = (unsigned long long)0xD2511F53u * c.x, p1 = (unsigned long long)0xCD9E8D57u * c.z;
        c = make_uint4((uint32_t)(p1 >> 32) ^ c.y ^ a.key[i].x, (uint32_t)p1, (uint32_t)(p0 >> 32) ^ c.w ^ a.key[i].y, (uint32_t)p0);
    }
    return c;
}
__device__ __forceinline__ float dropped(const DropArgs& a, float x, uint32_t word) { return word >= a.threshold ? x * a.c : 0.0f; }

// Rows whose elements come in vectors of V, the first of each at a multiple of four elements of its worker
// FLAT: one row.  A vector per thread: what is in flight comes from many resident warps, and 32 registers let all of them in (8192 x
// 4096 in bf16 with a residual, words taken apart by elements: 44.0 us with eight blocks an SM, 46.2 with six; two vectors a thread 51;
// blocks that stay, with the next vector on its way, 75.  By pairs 41)
template <class T, int V, bool RES, bool FLAT>
__global__ void __launch_bounds__(256, 8) dropout_kernel(const DropArgs a) {
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i >= a.items) return;
    const long long row = FLAT ? 0 : i / a.vecs, at = (FLAT ? i : i - row * a.vecs) * V, w = FLAT || a.per == 1 ? row : row / a.per;
    const T* p = static_cast<const T*>(a.x) + row * a.x_stride + at;
    const T* q = static_cast<const T*>(a.res) + row * a.res_stride + at;
    T* o = static_cast<T*>(a.out) + row * a.out_stride + at;
    const bool whole = at + V <= a.D;
    Pack<T, V> x, res;
    if (whole) {
        x = *reinterpret_cast<const Pack<T, V>*>(p);
        if (RES) res = *reinterpret_cast<const Pack<T, V>*>(q);
    } else {                                         // the row's last elements
        x = pack_some<T, V>(p, a.D - at);
        if (RES) res = pack_some<T, V>(q, a.D - at);
    }
    const uint32_t quad = (uint32_t)(((FLAT ? 0 : (row - w * a.per) * a.D) + at) >> 2);
    float v[V];
    unpack(v, x);
#pragma unroll
    for (int j = 0; j < V / 4; ++j) {
        const uint4 r = words_of(a, (uint32_t)w, quad + j);
        const uint32_t word[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) v[4 * j + k] = dropped(a, v[4 * j + k], word[k]);
    }
    if (RES) {
        float t[V];
        unpack(t, res);
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] += t[j];
    }
    if (whole) {
        store_vec<V>(o, v);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (at + j < a.D) o[j] = from_float<T>(v[j]);
    }
}

// Any rows: a thread per draw of four words, whose elements may lie in two rows or more
template <class T, bool RES>
__global__ void __launch_bounds__(256) dropout_loose_kernel(const DropArgs a) {
    const long long items = a.items, count = a.per * a.D;
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i < items) {
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
    a.items = vec ? a.rows * a.vecs : a.rows / a.per * a.vecs;
    const dim3 grid((unsigned)((a.items + 255) / 256));                       // (2^34 elements a worker, 32 workers: 2^29 blocks)
    if (vec && a.rows == 1)
        return a.res ? launch(false, dropout_kernel<T, V, true, true>, grid, 256, 0, st, a) : launch(false, dropout_kernel<T, V, false, true>, grid, 256, 0, st, a);
    if (vec)
        return a.res ? launch(false, dropout_kernel<T, V, true, false>, grid, 256, 0, st, a) : launch(false, dropout_kernel<T, V, false, false>, grid, 256, 0, st, a);
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
    for (uint32_t i = 0; i < 10; ++i) a.key[i] = make_uint2((uint32_t)seed + i * 0x9E3779B9u, (uint32_t)(seed >> 32) + i * 0xBB67AE85u);
    a.round_lo = (uint32_t)round;
    a.word3 = (uint32_t)layer << 16 | (uint32_t)(round >> 32) << 8 | 2u;
    a.worker = (uint32_t)worker; a.threshold = (uint32_t)(p * 4294967296.0); a.c = (float)(1.0 / (1.0 - p));
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    return status_of(type == QS_F32 ? launch_dropout<float>(a, st) : type == QS_BF16 ? launch_dropout<__nv_bfloat16>(a, st) : launch_dropout<__half>(a, st));
}

}  // extern "C"
