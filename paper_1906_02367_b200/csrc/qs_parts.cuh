// Sums over many rows, taken in two steps: blocks leave partial sums per column, which are joined in order.
#pragma once
#include "qs_gemm.cuh"

namespace qs {

// part: (workers, parts, D).  32 warps each sum a contiguous share of the parts
static __global__ void __launch_bounds__(1024) join_parts_kernel(const float* part, int parts, long long D, float* out, long long worker, int accumulate) {
    __shared__ float sh[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = blockIdx.y;
    const long long d = (long long)blockIdx.x * 32 + lane;
    const int per = (parts + 31) / 32, p0 = min(parts, warp * per), p1 = min(parts, p0 + per);
    after_launch();
    float s = 0.0f;
    if (d < D) {
        const float* p = part + (long long)r * parts * D + d;
#pragma unroll 4
        for (int i = p0; i < p1; ++i) s += p[i * D];
    }
    sh[warp][lane] = s;
    __syncthreads();
    if (warp || d >= D) return;
#pragma unroll
    for (int i = 1; i < 32; ++i) s += sh[i][lane];
    float* o = out + r * worker + d;
    *o = accumulate ? *o + s : s;
}
inline cudaError_t launch_join(bool after, const float* part, int parts, int R, long long D, float* out, long long worker, int accumulate, cudaStream_t st) {
    return launch(after, join_parts_kernel, dim3((unsigned)((D + 31) / 32), (unsigned)R), 1024, 0, st, part, parts, D, out, worker, accumulate);
}

inline int sm_count() {
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
        cudaGetLastError();
        return 0;
    }
    return sms;
}

}  // namespace qs
