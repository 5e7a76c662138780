// Sums over many rows, taken in two steps: blocks leave partial sums per column, which are joined.
#pragma once
#include "qs_gemm.cuh"

namespace qs {

// part: (workers, parts, D).  32 warps each sum a contiguous share of the parts, four sums side by side, and pairs of what they leave are added: a
// chain of the 32 was half of the error (weights' gradient of 509 x 257 in fp32: 1.45e-7, 1.0e-7 so)
static __global__ void __launch_bounds__(1024) join_parts_kernel(const float* part, int parts, long long D, float* out, long long worker, int accumulate) {
    __shared__ float sh[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = blockIdx.y;
    const long long d = (long long)blockIdx.x * 32 + lane;
    const int per = (parts + 31) / 32, p0 = min(parts, warp * per), p1 = min(parts, p0 + per);
    after_launch();
    float four[4] = {};
    if (d < D) {
        const float* p = part + (long long)r * parts * D + d;
        for (int i = p0; i < p1; i += 4) {           // (all four on their way before any is added)
            float v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = p[min(i + j, p1 - 1) * D];
#pragma unroll
            for (int j = 0; j < 4; ++j) four[j] += i + j < p1 ? v[j] : 0.0f;
        }
    }
    sh[warp][lane] = (four[0] + four[1]) + (four[2] + four[3]);
    __syncthreads();
    const float s = warp_sum_f(sh[lane][warp]);      // (a warp's column now: few registers, so that blocks fit beside the kernel before)
    const long long c = (long long)blockIdx.x * 32 + warp;
    if (lane || c >= D) return;
    float* o = out + r * worker + c;
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
