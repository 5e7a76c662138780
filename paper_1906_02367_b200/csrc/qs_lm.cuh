// Shared pieces of the language-model operators: element types, token ids, warp and block sums.
#pragma once
#include <cfloat>
#include <cmath>
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "../../include/qsparse.h"

namespace qs {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

__device__ __forceinline__ float neg_inf() { return __int_as_float(0xff800000); }
__device__ __forceinline__ float quiet_nan() { return __int_as_float(0x7fffffff); }

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
template <class T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

// token ids come as 32- or 64-bit integers
struct Ids {
    const void* p;
    int wide;
    __device__ __forceinline__ long long at(long long i) const {
        return wide ? static_cast<const long long*>(p)[i] : (long long)static_cast<const int*>(p)[i];
    }
};

__device__ __forceinline__ void flag_status(int* status, int code) {
    if (status) atomicCAS(status, 0, code);
}

__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// ------------------------------------------------------------------ host-side checks
inline int size_of_type(int type) { return type == QS_F32 ? 4 : (type == QS_BF16 || type == QS_F16) ? 2 : 0; }
inline bool aligned_to(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }
inline bool is_id_type(int t) { return t == QS_I32 || t == QS_I64; }
// of a call's own launches and copies: an error that another call left is not looked at
inline int status_of(cudaError_t e) {
    if (e == cudaSuccess) return QS_OK;
    cudaGetLastError();
    return QS_CUDA;
}
// A result may take an input's own place, row for row, or other columns of the same rows; any other overlap is refused
inline bool overlap(const void* z, int64_t stride, const void* g, int64_t g_stride, int64_t N, int64_t V, int size) {
    typedef __int128 wide;
    const wide z0 = reinterpret_cast<uintptr_t>(z), g0 = reinterpret_cast<uintptr_t>(g), row = (wide)stride * size, len = (wide)V * size;
    if (z0 == g0 && stride == g_stride) return false;
    const wide z1 = z0 + (N - 1) * row + len, g1 = g0 + (N - 1) * (wide)g_stride * size + len;
    if (z1 <= g0 || g1 <= z0) return false;
    if (stride != g_stride) return true;
    const wide apart = ((g0 - z0) % row + row) % row;            // from a row of z to the next row of g
    return apart < len || apart + len > row;
}
// AFTER: the kernel may start while the one before it still runs (it waits for that one's end itself)
template <class... P, class... A>
cudaError_t launch(bool after, void (*kernel)(P...), dim3 grid, unsigned threads, unsigned smem, cudaStream_t st, A... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = after ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

}  // namespace qs
