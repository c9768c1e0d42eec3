// What the epilogues of the product kernels share: 32 consecutive entries of a row, a thread's own, to and from memory.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>
#include <string.h>

namespace gvq {

template <typename T> __device__ __forceinline__ T from_f(float x);
template <> __device__ __forceinline__ float from_f(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f(float x) { return __float2half_rn(x); }
template <typename T> __device__ __forceinline__ float to_f(T x);
template <> __device__ __forceinline__ float to_f(float x) { return x; }
template <> __device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
template <> __device__ __forceinline__ float to_f(__half x) { return __half2float(x); }

// The first n of 32 entries (n <= 0: none), in 16-byte pieces where they are aligned.
template <typename T>
__device__ __forceinline__ void store_row32(T *dst, const float (&v)[32], int n)
{
    constexpr int PER = 16 / (int)sizeof(T);
    T e[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) e[i] = from_f<T>(v[i]);
    if (n >= 32 && (reinterpret_cast<uintptr_t>(dst) & 15u) == 0) {
#pragma unroll
        for (int i = 0; i < 32 / PER; ++i) {
            uint4 q;
            memcpy(&q, e + i * PER, 16);
            reinterpret_cast<uint4 *>(dst)[i] = q;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i)
            if (i < n) dst[i] = e[i];
    }
}
template <typename T>
__device__ __forceinline__ void load_row32(const T *src, float (&v)[32], int n)
{
    constexpr int PER = 16 / (int)sizeof(T);
    T e[32];
    if (n >= 32 && (reinterpret_cast<uintptr_t>(src) & 15u) == 0) {
#pragma unroll
        for (int i = 0; i < 32 / PER; ++i) {
            const uint4 q = reinterpret_cast<const uint4 *>(src)[i];
            memcpy(e + i * PER, &q, 16);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) e[i] = i < n ? src[i] : from_f<T>(0.0f);
    }
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = to_f(e[i]);
}

}  // namespace gvq
