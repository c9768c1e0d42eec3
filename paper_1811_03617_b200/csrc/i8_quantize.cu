// Quantization to 8-bit integers with a scale a row, and back (gvq.h, "8-bit integers").
//
//  i8_rows_kernel     along the rows, read once: a row stays in the registers of the threads that share it
//  i8_strip_kernel    along the columns, read once: a strip of columns stays in the shared memory of a cluster
//  i8_both_kernel     both of these in one launch
//  i8_max_kernel, i8_tile_kernel   along columns too long for that: largest magnitudes first, then tile by tile
//  i8_dequantize_kernel
//
// Measured, from memory, in us (the bytes at the copy rate): rows of 8192 x 4096 bf16 20.0 nearest, 28 stochastic (15.4), fp32 28 and 32
// (25.7); columns of 2048 x 4096 bf16 in strips 9.9 and 12.6 (3.8); columns of 8192 x 4096 bf16, gone through twice, 30 and 41 (15.4), fp32
// 60 and 70 (25.7); 777 x 1083 rows 3.3, columns 6.5, both 8.1 (0.4).  Of large ones instructions take as long as memory: of the nearest codes
// the conversions, maxima and packing, of the stochastic ones the random words, 10 integer instructions for two entries.  Small ones
// are a launch and the way to memory and back.
//
// With a = max(max |x|, 2^-100) and r the largest float with r a <= 127, a code is x r to the nearest whole number, rounded from
// the exact product: one fused multiply-add to 1.5 * 2^23 leaves it in the low bits, two's complement.  Stochastic rounding adds 14
// random bits below floor(2^14 x r), which the same instruction leaves there when it rounds down (2^14 * 127 < 2^22).
#include "gvq_internal.h"
#include "load8.cuh"
#include "mx4.cuh"
#include "row32.cuh"
#include "sm100_ptx.cuh"

namespace gvq {
namespace {

constexpr float kMagic = 12582912.0f;               // 1.5 * 2^23: its pattern's low 22 bits are 0
constexpr int kMaxRows = 512;      // of a CTA of i8_max_kernel
// i8_strip_kernel: CTAs of a cluster, threads, words from row to row, most rows of a CTA (106 KB of shared memory: two CTAs an SM)
constexpr int kCluster = 4, kStripThreads = 512, kStripPitch = 36, kStripRows = 752;
// i8_both_kernel: up to so many CTAs one at a time has an SM (us, bf16, one, two, a launch each: 512 x 4096, 192 CTAs, 5.2, 6.0, 9.2; 2048 x
// 1024, 192, 6.2, 7.9, 10.2; 777 x 1083, 263, 8.1, 9.9, 9.2; 1000 x 4096, 378, 11.3, 9.2, 12.1; 2048 x 2048, 640, 14.3, 9.7, 13.2), and
// so many are made in one launch at all (2048 x 4096, 768, 22.3, 15.1, 15.1; 1000 x 8192, 1256, 24.2, 16.4, 14.3).
constexpr int64_t kFewBlocks = 296, kBothBlocks = 768;

__host__ __device__ inline int64_t pitch_of(int64_t cols) { return (cols + 15) / 16 * 16; }
inline int64_t row_blocks(int64_t rows) { return (rows + kMaxRows - 1) / kMaxRows; }

// A row's factor and scale from the pattern of its largest magnitude.  A row that holds a NaN or an infinity has factor 0,
// and the caller's entries are replaced by 0.
struct RowScale { float r, scale; };
__device__ __forceinline__ RowScale row_scale(uint32_t top)
{
    RowScale s;
    if (top >= 0x7F800000u) { s.r = 0.0f; s.scale = __uint_as_float(0x7FC00000u); return s; }
    const float a = fmaxf(__uint_as_float(top), 7.888609052210118e-31f);      // 2^-100
    s.r = __fdiv_rd(127.0f, a);
    s.scale = __fdiv_rn(a, 127.0f);
    return s;
}
// Eight codes.  `r` is the row's factor, times 2^14 for stochastic rounding; p0: column pair of the first entry.
template <bool SR>
__device__ __forceinline__ uint2 codes_of(const float (&v)[8], float r, uint64_t h, uint32_t p0)
{
    uint32_t c[8];
    if (SR) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t x = mx4::pair_word(h, p0 + i), y = x >> 16;
            c[2 * i] = (__float_as_uint(__fmaf_rd(v[2 * i], r, kMagic)) + (((x ^ y) & 0xFFFFu) >> 2)) >> 14;
            c[2 * i + 1] = (__float_as_uint(__fmaf_rd(v[2 * i + 1], r, kMagic)) + (y >> 2)) >> 14;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i] = __float_as_uint(__fmaf_rn(v[i], r, kMagic));
    }
    uint2 q;
    q.x = __byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410);
    q.y = __byte_perm(__byte_perm(c[4], c[5], 0x0040), __byte_perm(c[6], c[7], 0x0040), 0x5410);
    return q;
}

template <typename T>
__device__ __forceinline__ void unpack8(const Raw8<T> &r, float (&v)[8])
{
    T e[8];
    memcpy(e, &r, sizeof(r));
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = to_f(e[i]);
}
// Pattern of the largest magnitude: patterns without their sign order like the magnitudes, infinity and NaN above all.
template <typename T>
__device__ __forceinline__ uint32_t top8(const Raw8<T> &r)
{
    if constexpr (sizeof(T) == 4) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            m = max(m, max(r.q[i].x & 0x7FFFFFFFu, r.q[i].y & 0x7FFFFFFFu));
            m = max(m, max(r.q[i].z & 0x7FFFFFFFu, r.q[i].w & 0x7FFFFFFFu));
        }
        return m;
    } else {      // two at a time
        const uint32_t m = __vmaxu2(__vmaxu2(r.q[0].x & 0x7FFF7FFFu, r.q[0].y & 0x7FFF7FFFu), __vmaxu2(r.q[0].z & 0x7FFF7FFFu, r.q[0].w & 0x7FFF7FFFu));
        const uint16_t top = (uint16_t)max(m & 0xFFFFu, m >> 16);
        T e;
        memcpy(&e, &top, 2);
        return __float_as_uint(to_f(e));
    }
}

struct QuantParams {
    const void *x;
    int64_t rows, cols, ld;
    uint64_t seed_w;            // mix64 of (seed, node)
    int8_t *codes, *codes_t;    // along the rows, along the columns; null: not wanted
    float *scales, *scales_t;
    int cluster, rows_per;      // of strips: CTAs that share one, rows of a CTA (a multiple of 16)
    int strip_blocks;           // of i8_both_kernel: CTAs for strips
    uint32_t *col_top;          // [row_blocks][cols]: patterns of magnitudes
    int row_blocks;             // CTAs along the rows of i8_max_kernel
    int ct;                     // tiles along the columns
};

// A CTA of NT threads: G of them share a row, KEEP groups of eight entries a thread in registers; longer rows are read again from L2.
template <typename T, bool SR, int G, int NT, bool VEC>
__device__ __forceinline__ void quantize_rows_of(const QuantParams &prm, uint32_t block)
{
    constexpr int KEEP = 4, ROWS = NT / G;
    __shared__ uint32_t tops[NT / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, in_row = ROWS == 1 ? threadIdx.x : threadIdx.x % G;
    const int64_t row = (int64_t)block * ROWS + (ROWS == 1 ? 0 : threadIdx.x / G);
    const bool there = row < prm.rows;
    const T *x = static_cast<const T *>(prm.x) + (there ? row : 0) * prm.ld;
    const int64_t pitch = pitch_of(prm.cols), groups = there ? pitch / 8 : 0;
    auto load = [&](int64_t at) { return load8<VEC>(x + at * 8, (int)min((int64_t)8, prm.cols - at * 8)); };
    Raw8<T> kept[KEEP];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
        const int64_t at = in_row + i * G;
        if (at < groups) kept[i] = load(at);
    }
#pragma unroll
    for (int i = 0; i < KEEP; ++i)
        if (in_row + i * G < groups) top = max(top, top8(kept[i]));
    for (int64_t at = in_row + KEEP * G; at < groups; at += G) top = max(top, top8(load(at)));
    top = __reduce_max_sync(0xffffffffu, top);
    if (G > 32) {
        if (lane == 0) tops[warp] = top;
        __syncthreads();
        constexpr int WARPS = G / 32;
        top = 0;
#pragma unroll
        for (int i = 0; i < WARPS; ++i) top = max(top, tops[(ROWS == 1 ? 0 : warp / WARPS * WARPS) + i]);
    }
    const RowScale s = row_scale(top);
    const bool fine = top < 0x7F800000u;
    const uint64_t h = SR ? mx4::row_word(prm.seed_w, row) : 0;
    const float r = SR ? s.r * 16384.0f : s.r;
    auto write = [&](int64_t at, const Raw8<T> &raw) {
        float v[8];
        unpack8(raw, v);
        *reinterpret_cast<uint2 *>(prm.codes + row * pitch + at * 8) = fine ? codes_of<SR>(v, r, h, (uint32_t)(at * 4)) : make_uint2(0, 0);
    };
#pragma unroll
    for (int i = 0; i < KEEP; ++i)
        if (in_row + i * G < groups) write(in_row + i * G, kept[i]);
    for (int64_t at = in_row + KEEP * G; at < groups; at += G) write(at, load(at));
    if (there && in_row == 0) prm.scales[row] = s.scale;
}
template <typename T, bool SR, int G, bool VEC>
__global__ void __launch_bounds__(G < 256 ? 256 : G) i8_rows_kernel(const QuantParams prm)
{
    ptx::launch_dependents();
    ptx::grid_dependency_wait();
    quantize_rows_of<T, SR, G, (G < 256 ? 256 : G), VEC>(prm, blockIdx.x);
}

// Largest magnitudes of eight columns over rows, as patterns: kept as they come, two columns of a 16-bit type a word.
template <typename T> struct Tops8 {
    static constexpr int N = 2 * (int)sizeof(T);
    uint32_t m[N];
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < N; ++i) m[i] = 0;
    }
    __device__ __forceinline__ void add(const Raw8<T> &r)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint4 q = r.q[i / 4];
            const uint32_t w = i % 4 == 0 ? q.x : i % 4 == 1 ? q.y : i % 4 == 2 ? q.z : q.w;
            m[i] = sizeof(T) == 4 ? max(m[i], w & 0x7FFFFFFFu) : __vmaxu2(m[i], w & 0x7FFF7FFFu);
        }
    }
    __device__ __forceinline__ void across(int lanes)      // of the lanes that are `lanes` apart (a power of two, a constant)
    {
#pragma unroll
        for (int d = 16; d >= lanes; d >>= 1) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const uint32_t o = __shfl_xor_sync(0xffffffffu, m[i], d);
                m[i] = sizeof(T) == 4 ? max(m[i], o) : __vmaxu2(m[i], o);
            }
        }
    }
    __device__ __forceinline__ uint32_t column(int i) const      // (a constant)
    {
        if (sizeof(T) == 4) return m[i % N];
        const uint16_t u = (uint16_t)(i & 1 ? m[i / 2 % N] >> 16 : m[i / 2 % N] & 0xFFFFu);
        T e;
        memcpy(&e, &u, sizeof(e) < 2 ? sizeof(e) : 2);
        return __float_as_uint(to_f(e));
    }
};

// Sixteen rows from r on of column c, whose entries are the `part`-th of the words: a 16-byte piece of the output's row c.
template <typename T, bool SR>
__device__ __forceinline__ void column_run(const QuantParams &prm, const uint32_t (&w)[16], int part, const RowScale &s, int64_t c, int64_t r,
                                           int64_t pitch_t)
{
    if (c >= prm.cols) return;
    const uint64_t h = SR ? mx4::row_word(prm.seed_w, c) : 0;
    uint2 q[2];
#pragma unroll
    for (int o = 0; o < 2; ++o) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t word = w[8 * o + e];
            if (sizeof(T) == 4) v[e] = __uint_as_float(word);
            else {
                T t;
                const uint16_t u = (uint16_t)(part ? word >> 16 : word & 0xFFFFu);
                memcpy(&t, &u, sizeof(t) < 2 ? sizeof(t) : 2);
                v[e] = to_f(t);
            }
        }
        q[o] = s.scale == s.scale ? codes_of<SR>(v, SR ? s.r * 16384.0f : s.r, h, (uint32_t)((r + 8 * o) >> 1)) : make_uint2(0, 0);
    }
    *reinterpret_cast<uint4 *>(prm.codes_t + c * pitch_t + r) = make_uint4(q[0].x, q[0].y, q[1].x, q[1].y);
}

// A cluster of up to four CTAs has a strip of 128 bytes of every row, rows_per rows a CTA (all of its columns' entries): it is read once
// into shared memory, the columns' largest magnitudes go round the cluster, and a thread takes 16 entries of a column (of two columns
// of a 16-bit type, so that a word is read once); eight lanes write 128 bytes of an output row.  Rows lie 4 words further apart than
// they are long and another 4 words on every 16 rows, so that eight lanes' 16-byte words, and the words of 4 columns in 8 runs of 16
// rows, lie in different banks.
template <typename T, bool SR, bool VEC>
__device__ __forceinline__ void quantize_strip(const QuantParams &prm, uint32_t block)
{
    constexpr int SC = 128 / (int)sizeof(T), L = SC / 8, RP = kStripThreads / L, WARPS = kStripThreads / 32;   // columns, lanes a row, rows a pass
    extern __shared__ uint4 smem_q[];
    uint32_t *tile = reinterpret_cast<uint32_t *>(smem_q);
    __shared__ uint32_t tops[WARPS][SC], of_cta[SC];
    __shared__ RowScale of_col[SC];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int cluster = prm.cluster, rank = block % cluster;
    const int64_t c0 = (int64_t)(block / cluster) * SC, r0 = (int64_t)rank * prm.rows_per;
    const T *x = static_cast<const T *>(prm.x);
    auto at = [&](int row) { return tile + row * kStripPitch + (row >> 4) * 4; };

    const int g = tid % L, n = (int)max((int64_t)0, min((int64_t)8, prm.cols - (c0 + g * 8)));
    Tops8<T> m;
    m.clear();
    constexpr int U = 16 / (int)sizeof(T);
    for (int p = tid / L; p < prm.rows_per; p += RP * U) {
        Raw8<T> raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t r = r0 + p + u * RP;
            raw[u] = load8<VEC>(x + r * prm.ld + c0 + g * 8, r < prm.rows && p + u * RP < prm.rows_per ? n : 0);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            m.add(raw[u]);
            if (p + u * RP < prm.rows_per) {
#pragma unroll
                for (int q = 0; q < (int)sizeof(T) / 2; ++q)
                    *reinterpret_cast<uint4 *>(at(p + u * RP) + g * (int)sizeof(T) * 2 + q * 4) = raw[u].q[q];
            }
        }
    }
    __syncwarp();
    m.across(L);
    if (lane < L) {
#pragma unroll
        for (int i = 0; i < 8; ++i) tops[warp][lane * 8 + i] = m.column(i);
    }
    __syncthreads();
    if (tid < SC) {
        uint32_t t = 0;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) t = max(t, tops[w][tid]);
        of_cta[tid] = t;
    }
    if (cluster > 1) ptx::cluster_sync(); else __syncthreads();
    if (tid < SC) {
        uint32_t t = of_cta[tid];
        if (cluster > 1) {
            const uint32_t from = ptx::smem_u32(of_cta + tid);
            t = 0;
#pragma unroll
            for (int i = 0; i < kCluster; ++i)
                if (i < cluster) t = max(t, __float_as_uint(ptx::load_cluster1(ptx::cluster_address(from, i))));
        }
        const RowScale s = row_scale(t);
        of_col[tid] = s;
        if (rank == 0 && c0 + tid < prm.cols) prm.scales_t[c0 + tid] = s.scale;
    }
    __syncthreads();
    const int64_t pitch_t = pitch_of(prm.rows);
    constexpr int PER = 4 / (int)sizeof(T);                 // columns of a word: 1 or 2
    const int runs = prm.rows_per / 16, items = (runs + 7) / 8 * 8;    // groups of eight runs, times eight groups of four words
    for (int it = warp; it < items; it += WARPS) {
        const int blk = it / 8 * 8 + (lane & 7), cw = it % 8 * 4 + (lane >> 3);
        const int64_t r = r0 + blk * 16;
        if (blk < runs && r < pitch_t) {
            uint32_t w[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) w[i] = at(blk * 16 + i)[cw];
#pragma unroll
            for (int part = 0; part < PER; ++part)
                column_run<T, SR>(prm, w, part, of_col[cw * PER + part], c0 + cw * PER + part, r, pitch_t);
        }
    }
    if (cluster > 1) ptx::cluster_sync();      // (its neighbours have read this CTA's maxima)
}
template <typename T, bool SR, bool VEC>
__global__ void __launch_bounds__(kStripThreads) i8_strip_kernel(const QuantParams prm)
{
    ptx::launch_dependents();
    ptx::grid_dependency_wait();
    quantize_strip<T, SR, VEC>(prm, blockIdx.x);
}
// Both in one launch, which a small matrix waits for as long as for its data: the strips first, rows on CTAs of the same size.  AT_ONCE:
// CTAs of an SM; two have 64 registers a thread and spill some.
template <typename T, bool SR, bool VEC, int AT_ONCE>
__global__ void __launch_bounds__(kStripThreads, AT_ONCE) i8_both_kernel(const QuantParams prm)
{
    ptx::launch_dependents();
    ptx::grid_dependency_wait();
    const int block = (int)blockIdx.x - prm.strip_blocks;
    if (block < 0) quantize_strip<T, SR, VEC>(prm, blockIdx.x);
    else if (prm.cols <= 1024) quantize_rows_of<T, SR, 32, kStripThreads, VEC>(prm, block);
    else if (prm.cols <= 4096) quantize_rows_of<T, SR, 128, kStripThreads, VEC>(prm, block);
    else quantize_rows_of<T, SR, kStripThreads, kStripThreads, VEC>(prm, block);
}

// A CTA: kMaxRows rows of a strip of 128 bytes.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) i8_max_kernel(const QuantParams prm)
{
    constexpr int SC = 128 / (int)sizeof(T), L = SC / 8, RP = 256 / L;      // columns, lanes a row, rows a pass
    __shared__ uint32_t tops[8][SC];
    ptx::launch_dependents();
    ptx::grid_dependency_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = threadIdx.x % L;
    const int strips = (int)((prm.cols + SC - 1) / SC), rb = blockIdx.x / strips;
    const int64_t c0 = (int64_t)(blockIdx.x - rb * strips) * SC;
    const int64_t r0 = (int64_t)rb * kMaxRows, r1 = min(prm.rows, r0 + kMaxRows);
    const int n = (int)max((int64_t)0, min((int64_t)8, prm.cols - (c0 + g * 8)));
    const T *x = static_cast<const T *>(prm.x) + c0 + g * 8;
    Tops8<T> m;
    m.clear();
    constexpr int U = 16 / (int)sizeof(T);
    for (int64_t r = r0 + threadIdx.x / L; r < r1; r += RP * U) {
        Raw8<T> raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = load8<VEC>(x + (r + u * RP) * prm.ld, r + u * RP < r1 ? n : 0);
#pragma unroll
        for (int u = 0; u < U; ++u) m.add(raw[u]);
    }
    __syncwarp();
    m.across(L);
    if (lane < L) {
#pragma unroll
        for (int i = 0; i < 8; ++i) tops[warp][lane * 8 + i] = m.column(i);
    }
    __syncthreads();
    if (threadIdx.x < SC && c0 + threadIdx.x < prm.cols) {
        uint32_t t = 0;
#pragma unroll
        for (int w = 0; w < 8; ++w) t = max(t, tops[w][threadIdx.x]);
        prm.col_top[(int64_t)rb * prm.cols + c0 + threadIdx.x] = t;
    }
}

// 16 bytes to shared memory without a register, zeros after the first `bytes` of them.
__device__ __forceinline__ void copy16(void *to, const void *from, int bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(ptx::smem_u32(to)), "l"(from), "r"(bytes) : "memory");
}
// A CTA: a tile of 128 x 128 entries, from the end: what i8_max_kernel has read last is in L2 (of 8192 x 4096 bf16 a fifth comes from memory again).  Shared memory and what follows as above.
template <typename T, bool SR, bool VEC>
__global__ void __launch_bounds__(256) i8_tile_kernel(const QuantParams prm)
{
    constexpr int W = 128 * (int)sizeof(T) / 4, PITCH = W + 4;    // words of a row of the tile
    extern __shared__ uint4 smem_q[];
    uint32_t *tile = reinterpret_cast<uint32_t *>(smem_q);
    __shared__ RowScale of_col[128];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    ptx::launch_dependents();
    ptx::grid_dependency_wait();
    const int tile_at = gridDim.x - 1 - blockIdx.x, rtile = tile_at / prm.ct, ctile = tile_at - rtile * prm.ct;
    const int64_t r0 = (int64_t)rtile * 128, c0 = (int64_t)ctile * 128;
    const T *x = static_cast<const T *>(prm.x);
    auto at = [&](int row) { return tile + row * PITCH + (row >> 4) * 4; };

    // warp w, iteration it: rows 16 w + 2 it + (lane >> 4); copies that need no registers, all of them on their way at once
    const int cl = (lane & 15) * 8;
    const int ncol = (int)max((int64_t)0, min((int64_t)8, prm.cols - (c0 + cl)));    // this lane's valid entries
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int row = 16 * warp + 2 * i + (lane >> 4);
        uint32_t *to = at(row) + (lane & 15) * (int)sizeof(T) * 2;
        const int64_t r = r0 + row;
        if constexpr (VEC) {
#pragma unroll
            for (int q = 0; q < (int)sizeof(T) / 2; ++q) {
                const int bytes = r < prm.rows ? max(0, min(16, ncol * (int)sizeof(T) - 16 * q)) : 0;
                // (where nothing is read the address is x's own)
                copy16(to + q * 4, bytes ? reinterpret_cast<const char *>(x + r * prm.ld + c0 + cl) + 16 * q : prm.x, bytes);
            }
        } else {
            const Raw8<T> raw = load8<false>(x + r * prm.ld + c0 + cl, r < prm.rows ? ncol : 0);
#pragma unroll
            for (int q = 0; q < (int)sizeof(T) / 2; ++q) *reinterpret_cast<uint4 *>(to + q * 4) = raw.q[q];
        }
    }
    uint32_t top = 0;
    if (tid < 128 && c0 + tid < prm.cols) {
        const uint32_t *from = prm.col_top + c0 + tid;
        int b = 0;
        for (; b + 8 <= prm.row_blocks; b += 8) {
            uint32_t t[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) t[i] = __ldcg(from + (int64_t)(b + i) * prm.cols);
#pragma unroll
            for (int i = 0; i < 8; ++i) top = max(top, t[i]);
        }
        for (; b < prm.row_blocks; ++b) top = max(top, __ldcg(from + (int64_t)b * prm.cols));
    }
    if (tid < 128) {
        const RowScale s = row_scale(top);
        of_col[tid] = s;
        if (rtile == 0 && c0 + tid < prm.cols) prm.scales_t[c0 + tid] = s.scale;
    }
    if (VEC) asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    constexpr int PER = 4 / (int)sizeof(T);                 // columns of a word: 1 or 2
    const int64_t pitch_t = pitch_of(prm.rows);
    const int blk = lane & 7;
#pragma unroll 1
    for (int cw = warp * 4 + (lane >> 3); cw < W; cw += 32) {
        uint32_t w[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) w[i] = at(blk * 16 + i)[cw];
        if (r0 + blk * 16 < pitch_t) {
#pragma unroll
            for (int part = 0; part < PER; ++part)
                column_run<T, SR>(prm, w, part, of_col[cw * PER + part], c0 + cw * PER + part, r0 + blk * 16, pitch_t);
        }
    }
}

// Four entries a thread.  8192 x 4096 in 34 us, where the bytes take 26 at the copy rate.
template <bool VEC>
__global__ void __launch_bounds__(256) i8_dequantize_kernel(const int8_t *codes, const float *scales, int64_t rows, int64_t cols, float *out,
                                                            int64_t ld)
{
    ptx::launch_dependents();
    ptx::grid_dependency_wait();
    const int64_t pitch = pitch_of(cols);
    for_chunks(rows, (uint32_t)((cols + 3) / 4), [&](int64_t r, int chunk) {
        const int64_t c = (int64_t)chunk * 4;
        const char4 q = *reinterpret_cast<const char4 *>(codes + r * pitch + c);
        const float s = __ldg(scales + r), v[4] = {q.x * s, q.y * s, q.z * s, q.w * s};
        float *to = out + r * ld + c;
        if (VEC && c + 4 <= cols) *reinterpret_cast<float4 *>(to) = make_float4(v[0], v[1], v[2], v[3]);
        else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (c + i < cols) to[i] = v[i];
        }
    });
}

template <typename T, bool SR, bool VEC>
cudaError_t quantize_rows(cudaStream_t st, const QuantParams &prm)
{
    // a row's threads: as few as keep it in registers, where there are rows enough (us, bf16: 8192 x 1024 with 32 threads a row 6.9, 128
    // 12.5, 256 18.9; 8192 x 4096 with 128 20.0, 256 25.5; 16 x 4096 with 128 2.5, 256 2.2; 2048 x 8192 with 256 11.2, 1024 34;
    // 2000 x 16384 with 512 23, 1024 39; 300 x 32768, which only 1024 keep, 11.2, 256 that read it twice 15.8)
    auto grid = [&](int rows) { return (int)((prm.rows + rows - 1) / rows); };
    if (prm.cols <= 1024) return ptx::launch_chained<i8_rows_kernel<T, SR, 32, VEC>>(prm, grid(8), 256, 0, 1, st);
    if (prm.cols <= 4096 && prm.rows > 512) return ptx::launch_chained<i8_rows_kernel<T, SR, 128, VEC>>(prm, grid(2), 256, 0, 1, st);
    if (prm.cols <= 8192) return ptx::launch_chained<i8_rows_kernel<T, SR, 256, VEC>>(prm, grid(1), 256, 0, 1, st);
    if (prm.cols <= 16384) return ptx::launch_chained<i8_rows_kernel<T, SR, 512, VEC>>(prm, grid(1), 512, 0, 1, st);
    return ptx::launch_chained<i8_rows_kernel<T, SR, 1024, VEC>>(prm, grid(1), 1024, 0, 1, st);
}
// Sets how a matrix's columns are quantized in strips, whether they are.
template <typename T, bool VEC>
bool cut_strips(QuantParams &prm)
{
    constexpr int SC = 128 / (int)sizeof(T);
    const int64_t strips = (prm.cols + SC - 1) / SC;
    // more CTAs where a strip does not fit one, or where it is long and there are SMs for them (bf16, 700 x 8192 11.4 us, two 7.9, four
    // 13.6; 450 x 4096 4.6, 6.4, 7.4; rows at any place take longer to read: 777 x 1083 two 7.5, four 6.5)
    int cluster = 1;
    auto per = [&] { return (prm.rows + 16 * cluster - 1) / (16 * cluster) * 16; };
    while (cluster < kCluster && (per() > kStripRows || (strips * cluster <= 128 && per() > (VEC ? 512 : 256)))) cluster *= 2;
    if (per() > kStripRows) return false;
    prm.cluster = cluster;
    prm.rows_per = (int)per();
    prm.strip_blocks = (int)(strips * cluster);
    return true;
}
inline size_t strip_smem(const QuantParams &prm) { return (size_t)(prm.rows_per * kStripPitch + prm.rows_per / 16 * 4) * 4; }

template <typename T, bool SR, bool VEC>
cudaError_t quantize_cols(cudaStream_t st, QuantParams prm)
{
    constexpr int SC = 128 / (int)sizeof(T);
    if (cut_strips<T, VEC>(prm))
        return ptx::launch_chained<i8_strip_kernel<T, SR, VEC>>(prm, prm.strip_blocks, kStripThreads, strip_smem(prm), prm.cluster, st);
    const cudaError_t e = ptx::launch_chained<i8_max_kernel<T, VEC>>(prm, (int)(prm.row_blocks * ((prm.cols + SC - 1) / SC)), 256, 0, 1, st);
    if (e != cudaSuccess) return e;
    const int tiles = (int)(mx4::tiles_of(pitch_of(prm.rows), 128) * prm.ct);
    const size_t smem = (128 * (128 * sizeof(T) / 4 + 4) + 32) * 4;
    return ptx::launch_chained<i8_tile_kernel<T, SR, VEC>>(prm, tiles, 256, smem, 1, st);
}

template <typename T, bool SR, bool VEC>
cudaError_t quantize_as(cudaStream_t st, QuantParams prm)
{
    if (prm.codes && prm.codes_t && cut_strips<T, VEC>(prm)) {
        const int rows = prm.cols <= 1024 ? kStripThreads / 32 : prm.cols <= 4096 ? kStripThreads / 128 : 1;      // of a CTA
        const int64_t blocks = prm.strip_blocks + (prm.rows + rows - 1) / rows;
        if (blocks <= kBothBlocks) {
            const int grid = (int)((blocks + prm.cluster - 1) / prm.cluster * prm.cluster);
            if (blocks <= kFewBlocks)
                return ptx::launch_chained<i8_both_kernel<T, SR, VEC, 1>>(prm, grid, kStripThreads, strip_smem(prm), prm.cluster, st);
            return ptx::launch_chained<i8_both_kernel<T, SR, VEC, 2>>(prm, grid, kStripThreads, strip_smem(prm), prm.cluster, st);
        }
    }
    if (prm.codes) {
        const cudaError_t e = quantize_rows<T, SR, VEC>(st, prm);
        if (e != cudaSuccess) return e;
    }
    return prm.codes_t ? quantize_cols<T, SR, VEC>(st, prm) : cudaSuccess;
}

template <typename T, bool SR>
cudaError_t quantize_as(cudaStream_t st, const QuantParams &prm, bool vec)
{
    return vec ? quantize_as<T, SR, true>(st, prm) : quantize_as<T, SR, false>(st, prm);
}

}  // namespace

int64_t i8_scratch_bytes(int64_t rows, int64_t cols) { return rows <= kCluster * kStripRows ? 0 : row_blocks(rows) * cols * 4; }

cudaError_t launch_i8_quantize(cudaStream_t st, const void *x, int dtype, int64_t rows, int64_t cols, int64_t ld, bool stochastic,
                               uint64_t seed, uint32_t node, int8_t *codes, float *scales, int8_t *codes_t, float *scales_t, void *scratch)
{
    QuantParams prm = {};
    prm.x = x;
    prm.rows = rows; prm.cols = cols; prm.ld = ld;
    prm.seed_w = mx4::seed_word(seed, node);
    prm.codes = codes; prm.codes_t = codes_t;
    prm.scales = scales; prm.scales_t = scales_t;
    prm.row_blocks = (int)row_blocks(rows);
    prm.col_top = static_cast<uint32_t *>(scratch);
    const bool vec = (reinterpret_cast<uintptr_t>(x) & 15u) == 0 && ld * (dtype == GVQ_F32 ? 4 : 2) % 16 == 0;
    prm.ct = (int)mx4::tiles_of(pitch_of(cols), 128);
    if (dtype == GVQ_F32) return stochastic ? quantize_as<float, true>(st, prm, vec) : quantize_as<float, false>(st, prm, vec);
    if (dtype == GVQ_BF16) return stochastic ? quantize_as<__nv_bfloat16, true>(st, prm, vec) : quantize_as<__nv_bfloat16, false>(st, prm, vec);
    return stochastic ? quantize_as<__half, true>(st, prm, vec) : quantize_as<__half, false>(st, prm, vec);
}

cudaError_t launch_i8_dequantize(cudaStream_t st, int num_sms, const int8_t *codes, const float *scales, int64_t rows, int64_t cols,
                                 float *out, int64_t ld)
{
    const int64_t blocks = (rows * ((cols + 3) / 4) + 255) / 256, most = (int64_t)num_sms * 8;
    const int grid = (int)(blocks < most ? blocks : most);
    if ((reinterpret_cast<uintptr_t>(out) & 15u) == 0 && ld % 4 == 0) i8_dequantize_kernel<true><<<grid, 256, 0, st>>>(codes, scales, rows, cols, out, ld);
    else i8_dequantize_kernel<false><<<grid, 256, 0, st>>>(codes, scales, rows, cols, out, ld);
    return cudaGetLastError();
}

}  // namespace gvq
