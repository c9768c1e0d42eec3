// What the epilogues of the product kernels share: a 32 x 32 piece of an accumulator goes from "a thread has a row"
// (how tensor memory is read) to "a warp has a row" through shared memory, so that global memory is read and written
// along rows: 64 or 128 bytes of one or two rows an instruction, where a thread's own row would touch 32 lines.
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
// Two entries of a 16-bit type in a word, rounded by one conversion; and back.
template <typename T> __device__ __forceinline__ uint32_t pack2(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2<__half>(float a, float b)
{
    const __half2 h = __floats2half2_rn(a, b);
    uint32_t w;
    memcpy(&w, &h, 4);
    return w;
}
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    uint32_t w;
    memcpy(&w, &h, 4);
    return w;
}
__device__ __forceinline__ float2 unpack_half2(uint32_t w)
{
    __half2 h;
    memcpy(&h, &w, 4);
    return __half22float2(h);
}

constexpr int kPiecePitch = 36;                              // words: 16-byte stores of eight lanes hit all banks
constexpr int kPieceBytes = 32 * kPiecePitch * 4;            // a warp's staging area

// Thread `lane` holds row `lane` of the piece.
__device__ __forceinline__ void stage_piece(float *buf, int lane, const float (&v)[32])
{
    __syncwarp();                                            // the last piece has been read
#pragma unroll
    for (int i = 0; i < 8; ++i)
        *reinterpret_cast<float4 *>(buf + lane * kPiecePitch + 4 * i) = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
    __syncwarp();
}

// A piece as a TMA store reads it: 32 rows of 128 bytes, 16-byte chunk j of row r at place j ^ (r % 8).  Thread `lane` holds
// row `lane`: 64 entries of a 16-bit type, or 32 floats.
__device__ __forceinline__ void stage_swizzled(unsigned char *buf, int lane, const float (&v)[32])
{
#pragma unroll
    for (int j = 0; j < 8; ++j)
        *reinterpret_cast<float4 *>(buf + lane * 128 + ((j ^ (lane & 7)) << 4)) =
            make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
}
template <typename T>
__device__ __forceinline__ void stage_swizzled16(unsigned char *buf, int lane, const float (&a)[32], const float (&b)[32])
{
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int e = (8 * j + 2 * i) & 31;
            w[i] = j < 4 ? pack2<T>(a[e], a[e + 1]) : pack2<T>(b[e], b[e + 1]);
        }
        *reinterpret_cast<uint4 *>(buf + lane * 128 + ((j ^ (lane & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// Writes the piece's rows x cols entries (both at most 32) at dst, rows ld entries apart.  PAIR: two entries a lane, for
// 16-bit types whose rows start at 4-byte boundaries.
template <typename T>
__device__ __forceinline__ void store_piece(const float *buf, int lane, T *dst, int64_t ld, int rows, int cols)
{
    if (sizeof(T) == 2 && (ld & 1) == 0 && (reinterpret_cast<uintptr_t>(dst) & 3u) == 0) {
        const int c = (lane & 15) * 2;
#pragma unroll 8
        for (int r = lane >> 4; r < rows; r += 2) {
            const float2 x = *reinterpret_cast<const float2 *>(buf + r * kPiecePitch + c);
            T *d = dst + (int64_t)r * ld + c;
            if constexpr (sizeof(T) == 2) {
                if (c + 1 < cols) *reinterpret_cast<uint32_t *>(d) = pack2<T>(x.x, x.y);
                else if (c < cols) *d = from_f<T>(x.x);
            }
        }
    } else {
#pragma unroll 4
        for (int r = 0; r < rows; ++r)
            if (lane < cols) dst[(int64_t)r * ld + lane] = from_f<T>(buf[r * kPiecePitch + lane]);
    }
}

}  // namespace gvq
