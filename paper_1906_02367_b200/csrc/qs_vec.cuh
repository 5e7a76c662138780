// Elements of a row in vectors: V elements of type T by one access (V = 1: element by element), values in fp32.
#pragma once
#include <cuda_fp8.h>

#include "qs_lm.cuh"

namespace qs {

template <class T> constexpr int wide_of() { return 16 / (int)sizeof(T); }

// V elements side by side.  Those of 16 bits are held and handled as pairs: element by element, taking the words apart and putting
// them together again was most of what the kernels around this did
template <class T, int V, bool PAIRS = sizeof(T) == 2 && V % 2 == 0> struct alignas(sizeof(T) * V) Pack { T e[V]; };
template <class T, int V> struct alignas(2 * V) Pack<T, V, true> { uint32_t w[V / 2]; };

template <class T> __device__ __forceinline__ uint32_t pack_two(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack_two<__nv_bfloat16>(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <> __device__ __forceinline__ uint32_t pack_two<__half>(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <class T> __device__ __forceinline__ float2 unpack_two(uint32_t w);
template <> __device__ __forceinline__ float2 unpack_two<__nv_bfloat16>(uint32_t w) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
template <> __device__ __forceinline__ float2 unpack_two<__half>(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }

template <class T, int V> __device__ __forceinline__ Pack<T, V> pack_of(const float* v) {
    Pack<T, V> q;
    if constexpr (sizeof(T) == 2 && V % 2 == 0) {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) q.w[i] = pack_two<T>(v[2 * i], v[2 * i + 1]);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) q.e[i] = from_float<T>(v[i]);
    }
    return q;
}
template <class T, int V> __device__ __forceinline__ void unpack(float* v, const Pack<T, V>& q) {
    if constexpr (sizeof(T) == 2 && V % 2 == 0) {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            const float2 f = unpack_two<T>(q.w[i]);
            v[2 * i] = f.x, v[2 * i + 1] = f.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = to_float(q.e[i]);
    }
}
// the elements [0, n) one by one, zeros behind them
template <class T, int V> __device__ __forceinline__ Pack<T, V> pack_some(const T* p, long long n) {
    float v[V];
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = j < n ? to_float(p[j]) : 0.0f;
    return pack_of<T, V>(v);
}

// (accesses of 16 bytes at most: that is the alignment of what comes in vectors)
template <int V, class T>
__device__ __forceinline__ void load_vec(float (&v)[V], const T* p) {
    constexpr int W = V * (int)sizeof(T) <= 16 ? V : 16 / (int)sizeof(T);
#pragma unroll
    for (int i = 0; i < V; i += W) unpack<T, W>(v + i, *reinterpret_cast<const Pack<T, W>*>(p + i));
}
template <int V, class T>
__device__ __forceinline__ void store_vec(T* p, const float (&v)[V]) {
    constexpr int W = V * (int)sizeof(T) <= 16 ? V : 16 / (int)sizeof(T);
#pragma unroll
    for (int i = 0; i < V; i += W) *reinterpret_cast<Pack<T, W>*>(p + i) = pack_of<T, W>(v + i);
}
template <int V> __device__ __forceinline__ void load_floats(float (&v)[V], const float* p) { load_vec<V>(v, p); }
// e4m3, rounded to nearest, magnitudes above 448 to 448, NaN kept
template <int V>
__device__ __forceinline__ void store_e4m3(uint8_t* p, const float (&v)[V]) {
    if constexpr (V == 1) {
        *p = (uint8_t)__nv_cvt_float_to_fp8(v[0], __NV_SATFINITE, __NV_E4M3);
    } else {
        uint32_t w[V / 4];                           // (V is 4 or 8)
#pragma unroll
        for (int i = 0; i < V; i += 4)
            w[i / 4] = (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(v[i], v[i + 1]), __NV_SATFINITE, __NV_E4M3) |
                       (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(v[i + 2], v[i + 3]), __NV_SATFINITE, __NV_E4M3) << 16;
        if constexpr (V == 8) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t*>(p) = w[0];
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

}  // namespace qs
