// Embedding rows and their gradient.
//
//   forward    out[r, n, :] = scale * table[r][tok[r, n], :]
//   gradient   grad[r][v, :] = scale * sum over the places n with tok[r, n] = v of g[r, n, :]
//
// for R workers at once, each with its own table (a stretch of its row of the R x d batch) or a
// shared one.  The gradient is formed without atomic additions: the places are sorted by token
// (stable, so equal tokens stay in the order of their places) and each run is summed in that order.
#include "qs_lm.cuh"

namespace {

using namespace qs;

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
};

template <class TW, class TO>
__global__ void __launch_bounds__(256) embed_kernel(const EmbedArgs a) {
    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const long long r = row / a.N, t = a.tok.at(row);
        TO* out = static_cast<TO*>(a.out) + row * a.out_stride;
        const bool named = t >= 0 && t < a.V;
        if (t >= a.V && threadIdx.x == 0) flag_status(a.status, QS_INVALID_ARG);
        const TW* src = static_cast<const TW*>(a.table) + r * a.worker_stride + (named ? t : 0) * a.row_stride;
        const float other = t < 0 ? 0.0f : quiet_nan();
        for (long long i = threadIdx.x; i < a.D; i += 256)
            out[i] = from_float<TO>(named ? a.scale * to_float(src[i]) : other);
    }
}

template <class TW>
void launch_embed_to(const EmbedArgs& a, int out_type, int grid, cudaStream_t st) {
    if (out_type == QS_F32) embed_kernel<TW, float><<<grid, 256, 0, st>>>(a);
    else if (out_type == QS_BF16) embed_kernel<TW, __nv_bfloat16><<<grid, 256, 0, st>>>(a);
    else embed_kernel<TW, __half><<<grid, 256, 0, st>>>(a);
}

// ------------------------------------------------------------------ gradient: sort by token
constexpr int SORT_TILE = 1024;            // places per block, one per thread
constexpr int SORT_MAX_BITS = 9;

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
    // workspace: keys and places, two of each (R x N), and the digit counts (R x bins x tiles)
    uint32_t* key[2];
    uint32_t* pos[2];
    uint32_t* count;
    int tiles, bits;                       // tiles per worker, bits per digit
};

__device__ __forceinline__ uint32_t key_of(const GradArgs& a, long long i) {
    const long long t = a.tok.at(i);
    if (t >= a.V) flag_status(a.status, QS_INVALID_ARG);
    return (uint32_t)(t < 0 || t >= a.V ? a.V : t);      // places that name no row sort behind all rows
}

__global__ void __launch_bounds__(SORT_TILE) digit_count_kernel(const GradArgs a, int pass) {
    __shared__ uint32_t hist[1 << SORT_MAX_BITS];
    const int r = blockIdx.y, bins = 1 << a.bits;
    for (int b = threadIdx.x; b < bins; b += SORT_TILE) hist[b] = 0;
    __syncthreads();
    const long long n = (long long)blockIdx.x * SORT_TILE + threadIdx.x;
    if (n < a.N) {
        const uint32_t k = pass == 0 ? key_of(a, r * a.N + n) : a.key[pass & 1][r * a.N + n];
        atomicAdd(&hist[(k >> (pass * a.bits)) & (bins - 1)], 1u);
    }
    __syncthreads();
    for (int b = threadIdx.x; b < bins; b += SORT_TILE) a.count[((long long)r * bins + b) * a.tiles + blockIdx.x] = hist[b];
}

// exclusive sums over (digit, tile), one block per worker
__global__ void __launch_bounds__(1024) digit_scan_kernel(const GradArgs a) {
    __shared__ uint32_t part[1024];
    const long long len = (long long)(1 << a.bits) * a.tiles;
    uint32_t* c = a.count + blockIdx.x * len;
    const long long per = (len + 1023) / 1024, lo = threadIdx.x * per, hi = lo + per < len ? lo + per : len;
    uint32_t sum = 0;
    for (long long i = lo; i < hi; ++i) sum += c[i];
    part[threadIdx.x] = sum;
    __syncthreads();
    for (int o = 1; o < 1024; o <<= 1) {
        const uint32_t v = threadIdx.x >= o ? part[threadIdx.x - o] : 0u;
        __syncthreads();
        part[threadIdx.x] += v;
        __syncthreads();
    }
    uint32_t run = threadIdx.x ? part[threadIdx.x - 1] : 0u;
    for (long long i = lo; i < hi; ++i) {
        const uint32_t v = c[i];
        c[i] = run;
        run += v;
    }
}

__global__ void __launch_bounds__(SORT_TILE) digit_scatter_kernel(const GradArgs a, int pass) {
    extern __shared__ uint16_t warp_count[];             // 32 x bins
    const int r = blockIdx.y, bins = 1 << a.bits, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int b = threadIdx.x; b < 32 * bins; b += SORT_TILE) warp_count[b] = 0;
    __syncthreads();
    const long long n = (long long)blockIdx.x * SORT_TILE + threadIdx.x;
    const bool in = n < a.N;
    uint32_t k = 0, p = 0, d = (uint32_t)bins;
    if (in) {
        k = pass == 0 ? key_of(a, r * a.N + n) : a.key[pass & 1][r * a.N + n];
        p = pass == 0 ? (uint32_t)n : a.pos[pass & 1][r * a.N + n];
        d = (k >> (pass * a.bits)) & (bins - 1);
    }
    const uint32_t same = __match_any_sync(0xffffffffu, d);
    const int rank = __popc(same & ((1u << lane) - 1u));
    if (in && rank == 0) warp_count[warp * bins + d] = (uint16_t)__popc(same);
    __syncthreads();
    for (int b = threadIdx.x; b < bins; b += SORT_TILE) {
        uint32_t run = 0;
        for (int w = 0; w < 32; ++w) {
            const uint32_t v = warp_count[w * bins + b];
            warp_count[w * bins + b] = (uint16_t)run;
            run += v;
        }
    }
    __syncthreads();
    if (in) {
        const uint32_t to = a.count[((long long)r * bins + d) * a.tiles + blockIdx.x] + warp_count[warp * bins + d] + rank;
        a.key[(pass + 1) & 1][r * a.N + to] = k;
        a.pos[(pass + 1) & 1][r * a.N + to] = p;
    }
}

__global__ void __launch_bounds__(256) zero_rows_kernel(const GradArgs a) {
    for (long long row = blockIdx.x; row < a.R * a.V; row += gridDim.x) {
        float* dst = a.grad + (row / a.V) * a.worker_stride + (row % a.V) * a.row_stride;
        for (long long i = threadIdx.x; i < a.D; i += 256) dst[i] = 0.0f;
    }
}

// one block per place of the sorted list; the first place of a run sums the whole run
template <class TG>
__global__ void __launch_bounds__(256) run_sum_kernel(const GradArgs a, int side) {
    for (long long i = blockIdx.x; i < a.R * a.N; i += gridDim.x) {
        const long long r = i / a.N, first = r * a.N, end = first + a.N;
        const uint32_t k = a.key[side][i];
        if (k >= a.V || (i > first && a.key[side][i - 1] == k)) continue;
        float* dst = a.grad + r * a.worker_stride + (long long)k * a.row_stride;
        for (long long c = threadIdx.x; c < a.D; c += 256) {
            float sum = 0.0f;
            for (long long j = i; j < end && a.key[side][j] == k; ++j)
                sum += to_float(static_cast<const TG*>(a.g)[(first + a.pos[side][j]) * a.g_stride + c]);
            dst[c] = a.accumulate ? fmaf(a.scale, sum, dst[c]) : a.scale * sum;
        }
    }
}

int bits_for(long long v) {
    int b = 1;
    while ((1ll << b) < v) ++b;
    return b;
}

struct SortPlan {
    int passes, bits, tiles;
    int64_t words;
};
SortPlan sort_plan(int R, int64_t N, int64_t V) {
    SortPlan s;
    const int total = bits_for(V + 1);                   // keys 0 .. V
    s.passes = (total + SORT_MAX_BITS - 1) / SORT_MAX_BITS;
    s.bits = (total + s.passes - 1) / s.passes;
    s.tiles = (int)((N + SORT_TILE - 1) / SORT_TILE);
    s.words = 4 * (int64_t)R * N + (int64_t)R * (1 << s.bits) * s.tiles;
    return s;
}

bool bad_shape(int R, int64_t N, int64_t V, int64_t D) { return R < 1 || R > 32 || N < 0 || V < 1 || D < 1; }
bool too_large(int R, int64_t N, int64_t V, int64_t D) {
    return V > (1ll << 30) || N > (1ll << 30) / R || D > (1ll << 30);
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
    EmbedArgs a{N, V, D, Ids{tokens, token_type == QS_I64}, table, worker_stride, row_stride, scale, out, out_stride, status, R * N};
    const int grid = (int)(a.rows < 65536 ? a.rows : 65536);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (table_type == QS_F32) launch_embed_to<float>(a, out_type, grid, st);
    else if (table_type == QS_BF16) launch_embed_to<__nv_bfloat16>(a, out_type, grid, st);
    else launch_embed_to<__half>(a, out_type, grid, st);
    return launch_status();
}

int64_t qs_embed_grad_bytes(int R, int64_t N, int64_t V, int64_t D) {
    if (bad_shape(R, N, V, D)) return QS_INVALID_ARG;
    if (too_large(R, N, V, D)) return QS_TOO_LARGE;
    return 4 * sort_plan(R, N, V).words;
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
    const SortPlan p = sort_plan(R, N, V);
    if (N > 0 && (!tokens || !grad_out || !work || !aligned_to(tokens, token_type == QS_I64 ? 8 : 4) ||
                  !aligned_to(grad_out, size_of_type(grad_type)) || !aligned_to(work, 16))) return QS_INVALID_ARG;
    if (work_bytes < 4 * p.words) return QS_CAPACITY;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    uint32_t* w = static_cast<uint32_t*>(work);
    const int64_t m = R * N;
    GradArgs a{R, N, V, D, Ids{tokens, token_type == QS_I64}, grad_out, grad_stride, scale, accumulate, grad_table, worker_stride,
               row_stride, status, {w, w + m}, {w + 2 * m, w + 3 * m}, w + 4 * m, p.tiles, p.bits};
    const int64_t rows = R * V;
    if (!accumulate) zero_rows_kernel<<<(int)(rows < 65536 ? rows : 65536), 256, 0, st>>>(a);
    if (N > 0) {
        const dim3 grid(p.tiles, R);
        const size_t smem = sizeof(uint16_t) * 32 * (1 << p.bits);
        for (int pass = 0; pass < p.passes; ++pass) {
            digit_count_kernel<<<grid, SORT_TILE, 0, st>>>(a, pass);
            digit_scan_kernel<<<R, 1024, 0, st>>>(a);
            digit_scatter_kernel<<<grid, SORT_TILE, smem, st>>>(a, pass);
        }
        const int side = p.passes & 1, blocks = (int)(m < 65536 ? m : 65536);
        if (grad_type == QS_F32) run_sum_kernel<float><<<blocks, 256, 0, st>>>(a, side);
        else if (grad_type == QS_BF16) run_sum_kernel<__nv_bfloat16><<<blocks, 256, 0, st>>>(a, side);
        else run_sum_kernel<__half><<<blocks, 256, 0, st>>>(a, side);
    }
    return launch_status();
}

}  // extern "C"
