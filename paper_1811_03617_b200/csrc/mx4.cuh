// Microscaled 4-bit floating point (the block format of gvq.h, "microscaled 4-bit"): the arithmetic of one block,
// shared by the kernels that quantize.
//
// A block is 32 consecutive entries, a quad of lanes holds it, eight entries a lane.  Its scale is the smallest
// power of two 2^(s - 127), s >= 0, with max |x| <= 6 * scale: with max |x| = m 2^e that is 2^(e - 2) for m <= 1.5 and
// 2^(e - 1) above, i.e. an addition that carries out of the mantissa exactly when it exceeds 1.5.  Dividing by a power
// of two is exact, so the codes depend on no rounding but the one they are defined by.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

namespace gvq {
namespace mx4 {

constexpr int kBlock = 32;                 // entries of a block
constexpr int kTileRows = 128, kTileBlocks = 4, kTileBytes = 512;   // one tile of scale bytes

__host__ __device__ inline int64_t blocks(int64_t cols) { return (cols + kBlock - 1) / kBlock; }
__host__ __device__ inline int64_t tiles_of(int64_t n, int per) { return (n + per - 1) / per; }
// Place of (row, block) in the scale bytes of a matrix with `kt` tiles along its blocks.
__host__ __device__ inline int64_t scale_at(int64_t row, int64_t block, int64_t kt)
{
    return ((row >> 7) * kt + (block >> 2)) * kTileBytes + (row & 31) * 16 + ((row >> 5) & 3) * 4 + (block & 3);
}

__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b, float c)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// Scale byte of a block from max |x| (NaN and infinity: 255).
__device__ __forceinline__ uint32_t scale_byte(float amax)
{
    const uint32_t b = __float_as_uint(amax) & 0x7FFFFFFFu;
    const int s = (int)((b + 0x3FFFFFu) >> 23) - 2;
    return b >= 0x7F800000u ? 255u : (uint32_t)max(s, 0);
}
// 1 / scale.  For a block without a value the factor is 0 and the caller's entries are replaced by 0 first.
__device__ __forceinline__ float inv_scale(uint32_t s) { return __uint_as_float((254u - s) << 23); }
__device__ __forceinline__ float scale_value(uint32_t s)
{
    return s == 255u ? __uint_as_float(0x7FC00000u) : s == 0u ? __uint_as_float(0x00400000u) : __uint_as_float(s << 23);
}

// Eight signed values on or near the grid to eight codes (nearest, ties to the even code), the first in the low bits.
__device__ __forceinline__ uint32_t codes8(const float (&v)[8])
{
    uint32_t r;
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
        "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
        : "=r"(r)
        : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}

// The row's part of the random numbers: hash24's two 64-bit rounds (gvq.h), the first of them done by the host.
__host__ __device__ inline uint64_t mix64(uint64_t z)
{
    z ^= z >> 30; z *= 0xBF58476D1CE4E5B9ull;
    z ^= z >> 27; z *= 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}
__host__ __device__ inline uint64_t seed_word(uint64_t seed, uint32_t node)
{
    return mix64(seed + 0x9E3779B97F4A7C15ull * ((uint64_t)node + 1));
}
__device__ __forceinline__ uint64_t row_word(uint64_t seed_w, int64_t row)
{
    return mix64(seed_w ^ (0xD1B54A32D192ED03ull * (uint64_t)(row + 1)));
}
// The columns 2p and 2p + 1 of a row have the low and the high half of a 32-bit word x ^ (x >> 16); this is x.
__device__ __forceinline__ uint32_t pair_word(uint64_t h, uint32_t p)
{
    uint32_t x = (uint32_t)(h >> 32) ^ ((uint32_t)h + 0x9E3779B9u * (p + 1));
    x ^= x >> 16; x *= 0x7FEB352Du;
    x ^= x >> 15;
    return x * 0x846CA68Bu;
}
// Stochastic rounding of r = |x| / scale to the grid: (floor(65536 r / step) + u) >> 16 steps.  For r >= 1 a step is bit 22
// of r's float pattern, so u is added 16 places below it and the rest is cut off; below 1, where the grid keeps the
// step 0.5 of [1, 2), the same is done to r + 1 (rounded toward zero, which keeps every bit that floor(65536 r / step)
// depends on).  Integer and comparison instructions run at half the rate of fp32 arithmetic and are what this costs: the
// comparison is a multiplication that saturates, and the halves of a word are taken from its last mixing step.
__device__ __forceinline__ float round_up_or_down(float r, uint32_t u)
{
    float c;      // 1 below 1, 0 from there on: 2^126 (1 - r), saturated
    asm("fma.rn.sat.f32 %0, %1, 0fFE800000, 0f7E800000;" : "=f"(c) : "f"(r));
    const float t = __fadd_rz(r, c);
    return __uint_as_float((__float_as_uint(t) + u * 64u) & 0xFFC00000u) - c;
}
__device__ __forceinline__ float with_sign(float mag, float x)
{
    return __uint_as_float(__float_as_uint(mag) | (__float_as_uint(x) & 0x80000000u));
}
// Eight entries of a lane -> signed grid values (what the codes stand for, over the scale).
// p0: column pair of the first entry.
template <bool SR>
__device__ __forceinline__ void grid8(float (&v)[8], float inv, uint64_t h, uint32_t p0)
{
    if (SR) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t x = pair_word(h, p0 + i), y = x >> 16;
            v[2 * i] = with_sign(round_up_or_down(fabsf(v[2 * i]) * inv, (x ^ y) & 0xFFFFu), v[2 * i]);
            v[2 * i + 1] = with_sign(round_up_or_down(fabsf(v[2 * i + 1]) * inv, y), v[2 * i + 1]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= inv;
    }
}
// A block without a value (s = 255) has codes 0.  Kept as a branch: it is hardly ever taken, and eight selects are not free.
__device__ __forceinline__ void clear_invalid(float (&v)[8], uint32_t s)
{
    if (s == 255u) {
        asm volatile("");
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 0.0f;
    }
}
__device__ __forceinline__ float quad_max(float m)
{
    m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, 1));
    return max_nan(m, __shfl_xor_sync(0xffffffffu, m, 2));
}
__device__ __forceinline__ float amax8(const float (&v)[8])
{
    float m = max_nan(fabsf(v[0]), fabsf(v[1]));
#pragma unroll
    for (int i = 2; i < 8; i += 2) m = max_nan(m, fabsf(v[i]), fabsf(v[i + 1]));
    return m;
}

}  // namespace mx4
}  // namespace gvq
