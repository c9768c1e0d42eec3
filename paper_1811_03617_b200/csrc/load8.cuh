// Eight consecutive entries of a row that starts anywhere, as they lie in memory; a matrix's chunks of entries dealt out to a grid.
#pragma once
#include <stdint.h>

namespace gvq {

template <typename T> struct Raw8 { uint4 q[sizeof(T) / 2]; };

// Entries from the n-th on are 0 (n <= 0: nothing is read).  VEC: p is at a 16-byte boundary.  Elsewhere the 16-byte words that
// hold the entries are read, each of which has one of them at least, and shifted together: reading entry by entry asks for every
// sector eight times.
template <bool VEC, typename T>
__device__ __forceinline__ Raw8<T> load8(const T *p, int n)
{
    constexpr int G = (int)sizeof(T) / 2, W = 4 * G;      // 16-byte words, words of the result
    Raw8<T> r;
    if (VEC && n >= 8) {
        if (sizeof(T) == 4 && (reinterpret_cast<uintptr_t>(p) & 31) == 0) {      // a whole sector (two halves ask for it twice)
            asm volatile("ld.global.nc.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=r"(r.q[0].x), "=r"(r.q[0].y), "=r"(r.q[0].z), "=r"(r.q[0].w), "=r"(r.q[G - 1].x), "=r"(r.q[G - 1].y),
                           "=r"(r.q[G - 1].z), "=r"(r.q[G - 1].w) : "l"(p));
            return r;
        }
#pragma unroll
        for (int i = 0; i < G; ++i) r.q[i] = __ldg(reinterpret_cast<const uint4 *>(p) + i);
        return r;
    }
    const uintptr_t at = reinterpret_cast<uintptr_t>(p), from = at & ~(uintptr_t)15, end = at + (n < 8 ? n : 8) * sizeof(T);
    const uint32_t off = VEC ? 0u : (uint32_t)(at & 15);
    uint32_t w[W + 4];
#pragma unroll
    for (int i = 0; i < G + (VEC ? 0 : 1); ++i) {
        const bool there = n > 0 && from + 16 * i < end;
        const uint4 q = there ? __ldg(reinterpret_cast<const uint4 *>(from) + i) : make_uint4(0, 0, 0, 0);
        w[4 * i] = q.x; w[4 * i + 1] = q.y; w[4 * i + 2] = q.z; w[4 * i + 3] = q.w;
    }
    if (!VEC && (off & 8)) {
#pragma unroll
        for (int i = 0; i < W + 2; ++i) w[i] = w[i + 2];
    }
    if (!VEC && (off & 4)) {
#pragma unroll
        for (int i = 0; i < W + 1; ++i) w[i] = w[i + 1];
    }
    if (!VEC && sizeof(T) == 2 && (off & 2)) {
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
    }
    if (n < 8) {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            if (sizeof(T) == 4) { if (i >= n) w[i] = 0; }
            else if (2 * i >= n) w[i] = 0;
            else if (2 * i + 1 >= n) w[i] &= 0xFFFFu;
        }
    }
#pragma unroll
    for (int i = 0; i < G; ++i) r.q[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    return r;
}

// f(row, chunk) of every chunk of `rows` rows of `chunks` of them, the grid's threads side by side.  One division a
// thread: what a step adds is the same for all.
template <typename F>
__device__ __forceinline__ void for_chunks(int64_t rows, uint32_t chunks, F f)
{
    const uint32_t first = blockIdx.x * 256 + threadIdx.x, step = gridDim.x * 256, dr = step / chunks, dc = step - dr * chunks;
    int64_t r = first / chunks;
    uint32_t c = first - (uint32_t)r * chunks;
    while (r < rows) {
        f(r, (int)c);
        r += dr;
        c += dc;
        if (c >= chunks) { c -= chunks; ++r; }
    }
}

}  // namespace gvq
