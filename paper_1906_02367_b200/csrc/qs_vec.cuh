// Elements of a row in vectors: V elements of type T by one access (V = 1: element by element), values in fp32.
#pragma once
#include <cuda_fp8.h>

#include "qs_lm.cuh"

namespace qs {

template <class T> constexpr int wide_of() { return 16 / (int)sizeof(T); }

template <class T, int V> struct alignas(sizeof(T) * V) Pack { T e[V]; };

// (accesses of 16 bytes at most: that is the alignment of what comes in vectors)
template <int V, class T>
__device__ __forceinline__ void load_vec(float (&v)[V], const T* p) {
    constexpr int W = V * (int)sizeof(T) <= 16 ? V : 16 / (int)sizeof(T);
#pragma unroll
    for (int i = 0; i < V; i += W) {
        const Pack<T, W> q = *reinterpret_cast<const Pack<T, W>*>(p + i);
#pragma unroll
        for (int j = 0; j < W; ++j) v[i + j] = to_float(q.e[j]);
    }
}
template <int V, class T>
__device__ __forceinline__ void store_vec(T* p, const float (&v)[V]) {
    constexpr int W = V * (int)sizeof(T) <= 16 ? V : 16 / (int)sizeof(T);
#pragma unroll
    for (int i = 0; i < V; i += W) {
        Pack<T, W> q;
#pragma unroll
        for (int j = 0; j < W; ++j) q.e[j] = from_float<T>(v[i + j]);
        *reinterpret_cast<Pack<T, W>*>(p + i) = q;
    }
}
template <class T, int V> __device__ __forceinline__ void unpack(float (&v)[V], const Pack<T, V>& q) {
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = to_float(q.e[j]);
}
template <int V> __device__ __forceinline__ void load_floats(float (&v)[V], const float* p) { load_vec<V>(v, p); }
// e4m3, rounded to nearest, magnitudes above 448 to 448, NaN kept
template <int V>
__device__ __forceinline__ void store_e4m3(uint8_t* p, const float (&v)[V]) {
    if constexpr (V == 1) {
        *p = (uint8_t)__nv_cvt_float_to_fp8(v[0], __NV_SATFINITE, __NV_E4M3);
    } else {
        Pack<uint16_t, V / 2> q;
#pragma unroll
        for (int i = 0; i < V; i += 2) q.e[i / 2] = (uint16_t)__nv_cvt_float2_to_fp8x2(make_float2(v[i], v[i + 1]), __NV_SATFINITE, __NV_E4M3);
        *reinterpret_cast<Pack<uint16_t, V / 2>*>(p) = q;
    }
}

__device__ __forceinline__ float warp_sum_f(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
}
// the largest value; a NaN among them stays
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float warp_max_f(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v = max_nan(v, __shfl_xor_sync(~0u, v, o));
    return v;
}

// whether rows of `count` vectors can be read by vectors of `bytes`: every row's start on that boundary
inline bool rows_aligned(const void* p, int64_t stride, int64_t rows, int size, int bytes) {
    return !p || (aligned_to(p, bytes) && (rows <= 1 || stride * size % bytes == 0));
}
// bytes [a, a + la) and [b, b + lb) share none
inline bool apart(const void* a, int64_t la, const void* b, int64_t lb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return !a || !b || la <= 0 || lb <= 0 || x + (uintptr_t)la <= y || y + (uintptr_t)lb <= x;
}
inline int64_t span(int64_t rows, int64_t stride, int64_t width, int size) { return rows > 0 && width > 0 ? ((rows - 1) * stride + width) * size : 0; }
// whether a result may lie where it does beside an input: nothing shared, the input's own place, or other columns of its rows
inline bool beside(const void* in, int64_t in_stride, const void* out, int64_t out_stride, int64_t rows, int64_t width, int size) {
    return !in || !out || rows <= 0 || width <= 0 || !overlap(in, in_stride, out, out_stride, rows, width, size);
}
// a pitch of one row says nothing: one that keeps wide accesses
inline int64_t pitch_of(int64_t rows, int64_t stride, int64_t width) { return rows > 1 ? stride : (width + 15) / 16 * 16; }

}  // namespace qs
