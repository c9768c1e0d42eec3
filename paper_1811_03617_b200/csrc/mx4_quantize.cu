// Quantization to microscaled 4-bit floating point, and back (gvq.h, "microscaled 4-bit").
//
//  mx4_quantize_kernel            a matrix, along its rows and / or along its columns (the transposed operand), read once
//  mx4_quantize_rows_kernel       a matrix along its rows only, where they start at 16-byte boundaries
//  mx4_quantize_aggregate_kernel  every node's slices, and the sum over the nodes of what the codes stand for
//  mx4_dequantize_kernel          codes back to values, summed over the nodes
#include "gvq_internal.h"
#include "mx4.cuh"
#include "row32.cuh"
#include "sm100_ptx.cuh"

namespace gvq {
namespace {

using namespace mx4;

// Eight consecutive entries as they lie in memory.
template <typename T> struct Raw8 { uint4 q[sizeof(T) / 2]; };

// 32 bytes at a 32-byte boundary that are read once.
__device__ __forceinline__ void load32(const void *p, uint4 &a, uint4 &b)
{
    asm volatile("ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(a.x), "=r"(a.y), "=r"(a.z), "=r"(a.w), "=r"(b.x), "=r"(b.y), "=r"(b.z), "=r"(b.w) : "l"(p) : "memory");
}
template <typename T>
__device__ __forceinline__ Raw8<T> load8(const T *p, int n, bool vec)
{
    Raw8<T> r;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.q[i] = make_uint4(0, 0, 0, 0);
    if (n >= 8 && vec) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.q[i] = __ldcs(reinterpret_cast<const uint4 *>(p) + i);
    } else if (n > 0) {
        T e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = i < n ? p[i] : T(0.0f);
        memcpy(&r, e, sizeof(r));
    }
    return r;
}
template <typename T>
__device__ __forceinline__ void unpack8(const Raw8<T> &r, float (&v)[8])
{
    T e[8];
    memcpy(e, &r, sizeof(r));
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = to_f(e[i]);
}

struct QuantParams {
    const void *x;
    int64_t rows, cols, ld;
    uint64_t seed_w;            // mix64 of (seed, node)
    uint8_t *codes, *scales;    // along the rows; null: not wanted
    uint8_t *codes_t, *scales_t;   // along the columns
    int vec;                    // rows start at 16-byte (1) or 32-byte (2) boundaries
    int ct;                     // tiles along the columns
    // of the row kernel: a CTA has rows_per_cta rows of a chunk of columns, chunk_blocks blocks (by_chunk: 2^32 over that, up)
    int64_t padded_rows;
    int rows_per_cta, chunks, chunk_blocks;
    uint32_t by_chunk;
};

// Max |x| of the entries in four words (NaN and infinity come out as themselves or as a NaN).
template <typename T>
__device__ __forceinline__ float amax_words(const uint32_t (&w)[8 * sizeof(T)])
{
    constexpr int N = 8 * (int)sizeof(T);
    if constexpr (sizeof(T) == 4) {
        float m = max_nan(fabsf(__uint_as_float(w[0])), fabsf(__uint_as_float(w[1])));
#pragma unroll
        for (int i = 2; i < N; i += 2) m = max_nan(m, fabsf(__uint_as_float(w[i])), fabsf(__uint_as_float(w[i + 1])));
        return m;
    } else {      // patterns without their sign order like the magnitudes, two at a time
        uint32_t m = __vmaxu2(w[0] & 0x7FFF7FFFu, w[1] & 0x7FFF7FFFu);
#pragma unroll
        for (int i = 2; i < N; i += 2) m = __vimax3_u16x2(m, w[i] & 0x7FFF7FFFu, w[i + 1] & 0x7FFF7FFFu);
        const uint16_t top = (uint16_t)max(m & 0xFFFFu, m >> 16);
        T e;
        memcpy(&e, &top, 2);
        return to_f(e);
    }
}

// Thirty-two entries that a lane holds in words -> its block's scale byte and 16 bytes of codes.
template <typename T, bool SR>
__device__ __forceinline__ uint4 quantize_block(const uint32_t (&w)[8 * sizeof(T)], uint64_t h, uint32_t p0, uint32_t &s)
{
    s = scale_byte(amax_words<T>(w));
    const float inv = inv_scale(min(s, 253u));
    uint32_t code[4];
#pragma unroll
    for (int o = 0; o < 4; ++o) {
        float v[8];
        T e[8];
        memcpy(e, w + o * 2 * sizeof(T), sizeof(e));
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = to_f(e[i]);
        clear_invalid(v, s);
        grid8<SR>(v, inv, h, p0 + 4 * o);
        code[o] = codes8(v);
    }
    return make_uint4(code[0], code[1], code[2], code[3]);
}

// One CTA: a tile of 128 x 128 entries, which is one tile of scale bytes of either form, read once (16 lanes have a row,
// 16 or 32 bytes each).  With COLS it goes through shared memory in its own type, rows 4 words longer than they are so that
// eight lanes' 16-byte words of eight rows lie in different banks.
//   ROWS alone   a quad of lanes quantizes a block as it comes
//   both         a lane takes a row's block from shared memory; the codes go out through shared memory, 64 bytes of a row
//   COLS         a thread takes 32 entries of a column (two columns of a 16-bit type at a time, so that a word is read once);
//                another eight words per 32 rows put the four blocks of eight columns that a warp works on in different
//                banks, and a warp's four lanes write 64 bytes of one output row
// Bound by instructions, 8 to 15 an entry and form, most of them integer ones at half rate (a quad a block in "both" cost 4 us
// more at the size below).  8192 x 4096 bf16 on the GPU, inputs from memory, us, floor in bytes 13 a form and 16 for both:
// columns 19.5 nearest and 29.5 stochastic, both 27 and 49; fp32 (floor 23 and 26) 34, 39, 41 and 57.
// (Of fp32 both ways two CTAs fit an SM; held to the registers of three it takes 57.0 us stochastic, to those of two 58.3.)
template <typename T, bool SR, bool ROWS, bool COLS>
__global__ void __launch_bounds__(256, COLS ? 3 : 4) mx4_quantize_kernel(const QuantParams prm)
{
    constexpr int W = 128 * (int)sizeof(T) / 4, PITCH = W + 4;    // words of a row of the tile
    extern __shared__ uint4 smem_q[];
    uint32_t *tile = reinterpret_cast<uint32_t *>(smem_q);          // [128][PITCH] + skew, when COLS
    uint4 *row_codes = reinterpret_cast<uint4 *>(tile + 128 * PITCH + 32);   // [128][5], when both: four blocks' codes
    __shared__ __align__(16) uint8_t sc[2][kTileBytes];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    ptx::launch_dependents();
    ptx::grid_dependency_wait();
    const int rtile = blockIdx.x / prm.ct, ctile = blockIdx.x - rtile * prm.ct;
    const int64_t r0 = (int64_t)rtile * 128, c0 = (int64_t)ctile * 128;
    const T *x = static_cast<const T *>(prm.x);
    const int64_t pitch = 16 * blocks(prm.cols), pitch_t = 16 * blocks(prm.rows);

    // warp w, iteration it: rows 16 w + 2 it + (lane >> 4)
    const int cl = (lane & 15) * 8;
    const int ncol = (int)min((int64_t)8, prm.cols - (c0 + cl));    // this lane's valid entries (<= 0: none)
    uint64_t h_own = 0;
    if (ROWS && !COLS && SR) h_own = row_word(prm.seed_w, r0 + 16 * warp + (lane & 15));
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        Raw8<T> raw[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t r = r0 + 16 * warp + 2 * (4 * half + i) + (lane >> 4);
            raw[i] = load8(x + r * prm.ld + c0 + cl, r < prm.rows ? ncol : 0, prm.vec);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int rl = 16 * warp + 2 * (4 * half + i) + (lane >> 4);
            if (COLS) {
#pragma unroll
                for (int q = 0; q < (int)sizeof(T) / 2; ++q)
                    *reinterpret_cast<uint4 *>(tile + rl * PITCH + (rl >> 5) * 8 + (lane & 15) * (int)sizeof(T) * 2 + q * 4) = raw[i].q[q];
            }
            if (ROWS && !COLS) {
                float v[8];
                unpack8(raw[i], v);
                const float amax = quad_max(amax8(v));
                const uint32_t s = scale_byte(amax);
                uint64_t h = 0;
                if (SR) h = __shfl_sync(0xffffffffu, h_own, rl & 15);
                clear_invalid(v, s);
                grid8<SR>(v, inv_scale(min(s, 253u)), h, (uint32_t)((c0 + cl) >> 1));
                const int64_t r = r0 + rl, b = (c0 + cl) >> 5;
                if (r < prm.rows && b < blocks(prm.cols))
                    *reinterpret_cast<uint32_t *>(prm.codes + r * pitch + ((c0 + cl) >> 1)) = codes8(v);
                if ((lane & 3) == 0) sc[0][(rl & 31) * 16 + (rl >> 5) * 4 + ((lane & 15) >> 2)] = (uint8_t)s;
            }
        }
    }
    __syncthreads();
    if (ROWS && COLS) {
        const int g = warp >> 1, rl = 32 * g + lane;
        const uint64_t h = SR ? row_word(prm.seed_w, r0 + rl) : 0;
#pragma unroll 1
        for (int b = 2 * (warp & 1); b < 2 * (warp & 1) + 2; ++b) {
            uint32_t w[W / 4], s;
#pragma unroll
            for (int i = 0; i < W / 16; ++i) {
                const uint4 q = *reinterpret_cast<const uint4 *>(tile + rl * PITCH + g * 8 + b * (W / 4) + 4 * i);
                w[4 * i] = q.x; w[4 * i + 1] = q.y; w[4 * i + 2] = q.z; w[4 * i + 3] = q.w;
            }
            row_codes[rl * 5 + b] = quantize_block<T, SR>(w, h, (uint32_t)(c0 >> 1) + 16 * b, s);
            sc[0][(rl & 31) * 16 + g * 4 + b] = (uint8_t)s;
        }
    }
    if (COLS) {
        constexpr int PER = 4 / (int)sizeof(T);                 // columns of a word: 1 or 2
        const int blk = lane & 3;
#pragma unroll 1
        for (int cw = warp * 8 + (lane >> 2); cw < W; cw += 64) {
            uint32_t w[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) w[i] = tile[(blk * 32 + i) * PITCH + blk * 8 + cw];
#pragma unroll
            for (int part = 0; part < PER; ++part) {
                const int cl2 = cw * PER + part;
                const int64_t c = c0 + cl2, b = (r0 >> 5) + blk;
                auto entry = [&](int i) -> float {
                    if (sizeof(T) == 4) return __uint_as_float(w[i]);
                    T e;
                    const uint16_t u = (uint16_t)(part ? w[i] >> 16 : w[i] & 0xFFFFu);
                    memcpy(&e, &u, sizeof(e) < 2 ? sizeof(e) : 2);
                    return to_f(e);
                };
                float amax = 0.0f;
#pragma unroll
                for (int i = 0; i < 32; i += 2) amax = max_nan(amax, fabsf(entry(i)), fabsf(entry(i + 1)));
                const uint32_t s = scale_byte(amax);
                const float inv = inv_scale(min(s, 253u));
                uint64_t h = 0;
                if (SR) h = row_word(prm.seed_w, c);
                uint32_t code[4];
#pragma unroll
                for (int o = 0; o < 4; ++o) {
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = entry(8 * o + e);
                    clear_invalid(v, s);
                    grid8<SR>(v, inv, h, (uint32_t)((r0 + blk * 32 + 8 * o) >> 1));
                    code[o] = codes8(v);
                }
                if (c < prm.cols && b < blocks(prm.rows))
                    *reinterpret_cast<uint4 *>(prm.codes_t + c * pitch_t + b * 16) = make_uint4(code[0], code[1], code[2], code[3]);
                sc[1][(cl2 & 31) * 16 + (cl2 >> 5) * 4 + blk] = (uint8_t)s;
            }
        }
        __syncthreads();
    }
    if (ROWS && COLS) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int at = tid + 256 * i;
            const int64_t r = r0 + (at >> 2), b = (c0 >> 5) + (at & 3);
            if (r < prm.rows && b < blocks(prm.cols)) *reinterpret_cast<uint4 *>(prm.codes + r * pitch + b * 16) = row_codes[(at >> 2) * 5 + (at & 3)];
        }
    }
    // the tile's scale bytes, whole (entries past the matrix are zeros, whose scale byte is 0)
    if (ROWS && tid < 32)
        reinterpret_cast<uint4 *>(prm.scales + ((int64_t)rtile * prm.ct + ctile) * kTileBytes)[tid] =
            reinterpret_cast<const uint4 *>(sc[0])[tid];
    if (COLS && tid >= 32 && tid < 64)
        reinterpret_cast<uint4 *>(prm.scales_t + ((int64_t)ctile * tiles_of(prm.rows, 128) + rtile) * kTileBytes)[tid - 32] =
            reinterpret_cast<const uint4 *>(sc[1])[tid - 32];
}

// Along the rows only: a lane has a whole block, so that what belongs to a block (its largest entry, its scale, its row's
// random word) costs a lane once and no shuffles; its 16 bytes of codes lie next to its neighbours'.  With a quad for a
// block, as in the tile kernel, those were half of 13 instructions an entry, and instructions are what bounds this: 8192 x 4096
// bf16 nearest 16.6 us on the GPU (floor 13; 13.4 of an input that L2 still holds), stochastic 26; fp32 30.5 and 29.5 (floor 23).
// Loads of 32 bytes, whole sectors, where rows start at such boundaries; with 16 bytes each sector is asked for twice (17.3, 26.3;
// 36 and 38).
template <typename T, bool SR>
__global__ void __launch_bounds__(256) mx4_quantize_rows_kernel(const QuantParams prm)
{
    constexpr int W = 8 * (int)sizeof(T);          // words of a block
    ptx::launch_dependents();
    ptx::grid_dependency_wait();
    const int chunk = blockIdx.x % prm.chunks;
    const int64_t row0 = (int64_t)(blockIdx.x / prm.chunks) * prm.rows_per_cta;
    const int64_t nb = blocks(prm.cols), kt = tiles_of(nb, kTileBlocks);
    const int b0 = chunk * prm.chunk_blocks, n_b = (int)min((int64_t)prm.chunk_blocks, kt * kTileBlocks - b0);   // padded
    const int items = prm.rows_per_cta * n_b;
    const T *x = static_cast<const T *>(prm.x);
    for (int it = threadIdx.x; it < items; it += 256) {
        // (it < 2^16: exact)
        const int r = n_b == prm.chunk_blocks ? (int)__umulhi((uint32_t)it, prm.by_chunk) : it / n_b;
        const int64_t row = row0 + r, b = b0 + it - r * n_b;
        if (row >= prm.padded_rows) break;
        uint32_t s = 0;
        if (row < prm.rows && b < nb) {
            uint32_t w[W];
            const T *from = x + row * prm.ld + b * kBlock;
            const int n = (int)min((int64_t)kBlock, prm.cols - b * kBlock);
            if (n == kBlock && prm.vec == 2) {
#pragma unroll
                for (int i = 0; i < W / 8; ++i) {
                    uint4 q, u;
                    load32(from + i * 32 / sizeof(T), q, u);
                    w[8 * i] = q.x; w[8 * i + 1] = q.y; w[8 * i + 2] = q.z; w[8 * i + 3] = q.w;
                    w[8 * i + 4] = u.x; w[8 * i + 5] = u.y; w[8 * i + 6] = u.z; w[8 * i + 7] = u.w;
                }
            } else if (n == kBlock) {
#pragma unroll
                for (int i = 0; i < W / 4; ++i) {
                    const uint4 q = __ldcs(reinterpret_cast<const uint4 *>(from) + i);
                    w[4 * i] = q.x; w[4 * i + 1] = q.y; w[4 * i + 2] = q.z; w[4 * i + 3] = q.w;
                }
            } else {
                T e[kBlock];
#pragma unroll
                for (int i = 0; i < kBlock; ++i) e[i] = i < n ? from[i] : T(0.0f);
                memcpy(w, e, sizeof(w));
            }
            reinterpret_cast<uint4 *>(prm.codes)[row * nb + b] = quantize_block<T, SR>(w, SR ? row_word(prm.seed_w, row) : 0, (uint32_t)(b * 16), s);
        }
        prm.scales[scale_at(row, b, kt)] = (uint8_t)s;      // (past the matrix: 0)
    }
}

struct AggParams {
    int d, n_nodes;
    uint64_t seed_w[GVQ_MAX_NODES];
    const int32_t *tile_layer, *tile_row0, *layer_S;
    const int64_t *layer_off, *layer_soff;
    NodePtrs<const float> g;
    NodePtrs<uint8_t> codes, scales;
    float *out;                 // may be null
    int n_tiles, n_tails;       // the CTAs after the tiles' sum the tails
    int shares;                 // CTAs that share a tile's rounds, where there are few tiles (464,432 entries, 8 nodes: 12.3 us -> 8.0)
    const int64_t *tail_off;
    const int32_t *tail_len;
};

// A quad of lanes takes a block of a slice and goes through the nodes: eight entries a lane, read once, quantized, and
// what the codes stand for added (fp32, n ascending; code times power of two is exact, so the only rounding is the
// sum's).  OUT: the codes and scale bytes are wanted.  Of four nodes' row words each lane of the quad mixes one.
// Bound by instructions, a third of them the random words': 14.7 million entries of 16 nodes, stochastic, 188 us a call in a long
// loop (copying the same bytes: 153), 205 in a burst of three, whose first call's way to the GPU is in it.  Nearest 171.  With the
// codes, 125 MB more, 250 and 224.  One launch for slices and tails: a small layout's 3.1 us are its launch.
template <bool SR, bool OUT>
__global__ void __launch_bounds__(256, 4) mx4_quantize_aggregate_kernel(const __grid_constant__ AggParams prm)
{
    ptx::launch_dependents();
    ptx::grid_dependency_wait();
    if ((int)blockIdx.x >= prm.n_tiles * prm.shares) {
        const int tail = blockIdx.x - prm.n_tiles * prm.shares, len = prm.tail_len[tail];
        const int64_t off = prm.tail_off[tail];
        for (int e = threadIdx.x; e < len; e += 256) {
            float acc = prm.g.p[0][off + e];
            for (int n = 1; n < prm.n_nodes; ++n) acc += prm.g.p[n][off + e];
            prm.out[off + e] = acc;
        }
        return;
    }
    const int t = blockIdx.x / prm.shares, share = blockIdx.x - t * prm.shares, layer = prm.tile_layer[t], row0 = prm.tile_row0[t];
    const int rows = min(kDecompressRows, prm.layer_S[layer] - row0);
    const int d = prm.d, nb = (d + kBlock - 1) / kBlock;
    const int64_t base = prm.layer_off[layer] + (int64_t)row0 * d, slice0 = prm.layer_soff[layer] + row0;
    const int64_t kt = tiles_of(nb, kTileBlocks);
    const int lane4 = threadIdx.x & 3;
    // every thread of a warp makes the same number of rounds: the shuffles below need the whole quad
    const int n_items = rows * nb, rounds = (n_items + 63) / 64;
    for (int it = share; it < rounds; it += prm.shares) {
        const int item = it * 64 + (threadIdx.x >> 2);
        const bool in = item < n_items;
        const int row = in ? item / nb : 0, b = in ? item - row * nb : 0;
        const int j = b * kBlock + lane4 * 8;                    // first entry of this lane in the slice
        const bool in0 = in && j < d, in1 = in && j + 4 < d;     // d is a multiple of 4
        const int64_t at = base + (int64_t)row * d + j;
        const int64_t slice = slice0 + row;
        float acc[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = 0.0f;
        constexpr int U = 4;                                     // nodes whose loads are in flight together
        for (int n0 = 0; n0 < prm.n_nodes; n0 += U) {
            float4 x[U][2];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                x[u][0] = x[u][1] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (n0 + u < prm.n_nodes) {
                    const float4 *src = reinterpret_cast<const float4 *>(prm.g.p[n0 + u] + at);
                    if (in0) x[u][0] = __ldcs(src);
                    if (in1) x[u][1] = __ldcs(src + 1);
                }
            }
            uint64_t h_own = 0;
            if (SR) h_own = row_word(prm.seed_w[min(n0 + lane4, prm.n_nodes - 1)], slice);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (n0 + u >= prm.n_nodes) break;
                const int n = n0 + u;
                float v[8] = {x[u][0].x, x[u][0].y, x[u][0].z, x[u][0].w, x[u][1].x, x[u][1].y, x[u][1].z, x[u][1].w};
                const uint32_t s = scale_byte(quad_max(amax8(v)));
                if (OUT) clear_invalid(v, s);      // (the sum takes its NaN from the scale)
                const uint64_t h = SR ? __shfl_sync(0xffffffffu, h_own, (threadIdx.x & 28) + u) : 0;
                grid8<SR>(v, inv_scale(min(s, 253u)), h, (uint32_t)(j >> 1));
                if (OUT || !SR) {
                    const uint32_t code = codes8(v);
                    if (OUT && in && prm.codes.p[n]) {
                        *reinterpret_cast<uint32_t *>(prm.codes.p[n] + (slice * nb + b) * 16 + lane4 * 4) = code;
                        if (lane4 == 0) prm.scales.p[n][scale_at(slice, b, kt)] = (uint8_t)s;
                    }
                    if (!SR) {   // nearest: the grid value is what the code stands for
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const uint32_t c = code >> (4 * e);
                            const uint32_t m = c & 7u;
                            const float mag = m < 2u ? 0.5f * (float)m : __uint_as_float((m + 252u) << 22);
                            v[e] = with_sign(mag, __uint_as_float(c << 28));
                        }
                    }
                }
                const float sv = scale_value(s);
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[e] = fmaf(v[e], sv, acc[e]);
            }
        }
        if (prm.out) {
            float4 *dst = reinterpret_cast<float4 *>(prm.out + at);
            if (in0) dst[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
            if (in1) dst[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
        }
    }
}

// Scale bytes past the last slice or block of an operand that the kernel above writes entry by entry: zeros.
__global__ void mx4_clear_scale_padding_kernel(NodePtrs<uint8_t> scales, int64_t S, int nb)
{
    const int64_t kt = tiles_of(nb, kTileBlocks), rt = tiles_of(S, kTileRows);
    uint8_t *s = scales.p[blockIdx.y];
    if (!s) return;
    const int64_t total = rt * kt * kTileBytes;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += (int64_t)gridDim.x * blockDim.x) {
        const int64_t tile = i / kTileBytes;
        const int in = (int)(i - tile * kTileBytes);
        const int64_t row = (tile / kt) * kTileRows + ((in >> 2) & 3) * 32 + (in >> 4), b = (tile % kt) * kTileBlocks + (in & 3);
        if (row >= S || b >= nb) s[i] = 0;
    }
}

struct DeqParams {
    int n_nodes;
    int64_t rows, cols;         // of the quantized matrix
    int64_t ld;                 // of the output; ignored when a layout gives the rows' places
    int d;
    int n_layers;
    const int64_t *layer_off, *layer_soff;
    const int32_t *layer_S;
    NodePtrs<const uint8_t> codes, scales;
    float *out;
    int vec;
};

// A lane takes eight entries of a row, one after the other every node's: four code bytes and the block's scale byte.  8192 x 4096
// 33 us (floor 23); the sum of 16 nodes' 14.7 million entries 123 us (floor 28): bound by the index arithmetic in 64 bits and by
// four-byte loads.
template <bool LAYOUT>
__global__ void __launch_bounds__(256) mx4_dequantize_kernel(const __grid_constant__ DeqParams prm)
{
    const int64_t nb = blocks(prm.cols), kt = tiles_of(nb, kTileBlocks);
    const int64_t total = prm.rows * nb * 4;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / (nb * 4), piece = i - row * (nb * 4), b = piece >> 2;
        const int64_t sc = scale_at(row, b, kt);
        float acc[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = 0.0f;
        for (int n = 0; n < prm.n_nodes; ++n) {
            const uint32_t code = __ldcs(reinterpret_cast<const uint32_t *>(prm.codes.p[n]) + i);
            const float sv = scale_value(prm.scales.p[n][sc]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t c = code >> (4 * e), m = c & 7u;
                const float mag = m < 2u ? 0.5f * (float)m : __uint_as_float((m + 252u) << 22);
                acc[e] = fmaf(with_sign(mag, __uint_as_float(c << 28)), sv, acc[e]);
            }
        }
        const int64_t col = piece * 8;
        float *dst;
        if (LAYOUT) {
            int lo = 0, hi = prm.n_layers - 1;   // the layer of this slice: the last one that starts at or before it
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (prm.layer_soff[mid] <= row) lo = mid; else hi = mid - 1;
            }
            dst = prm.out + prm.layer_off[lo] + (row - prm.layer_soff[lo]) * prm.d + col;
        } else {
            dst = prm.out + row * prm.ld + col;
        }
        if (prm.vec && col + 8 <= prm.cols) {
            reinterpret_cast<float4 *>(dst)[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
            reinterpret_cast<float4 *>(dst)[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (col + e < prm.cols) dst[e] = acc[e];
        }
    }
}

template <typename T, bool SR, bool ROWS, bool COLS>
cudaError_t launch_quantize_as(cudaStream_t st, const QuantParams &prm)
{
    const unsigned grid = (unsigned)(prm.ct * tiles_of(prm.rows, 128));
    const size_t smem = COLS ? 128 * (128 * sizeof(T) + 16) + 128 + (ROWS ? 128 * 80 : 0) : 0;
    return ptx::launch_chained<mx4_quantize_kernel<T, SR, ROWS, COLS>>(prm, (int)grid, 256, smem, 1, st);
}
template <typename T, bool SR>
cudaError_t launch_quantize_forms(cudaStream_t st, const QuantParams &prm)
{
    if (prm.codes && !prm.codes_t && prm.vec) {
        QuantParams p = prm;
        const int64_t padded = tiles_of(blocks(prm.cols), kTileBlocks) * kTileBlocks;
        p.chunk_blocks = (int)min(padded, (int64_t)1024);
        p.chunks = (int)tiles_of(padded, 1024);
        p.by_chunk = (uint32_t)((((uint64_t)1 << 32) + p.chunk_blocks - 1) / p.chunk_blocks);
        p.rows_per_cta = max(1, 1024 / p.chunk_blocks);
        p.padded_rows = tiles_of(prm.rows, kTileRows) * kTileRows;
        const int64_t grid = p.chunks * tiles_of(p.padded_rows, p.rows_per_cta);
        if (grid <= INT32_MAX) return ptx::launch_chained<mx4_quantize_rows_kernel<T, SR>>(p, (int)grid, 256, 0, 1, st);
    }
    if (prm.codes && prm.codes_t) return launch_quantize_as<T, SR, true, true>(st, prm);
    if (prm.codes) return launch_quantize_as<T, SR, true, false>(st, prm);
    return launch_quantize_as<T, SR, false, true>(st, prm);
}
template <typename T>
cudaError_t launch_quantize_rounding(cudaStream_t st, const QuantParams &prm, bool stochastic)
{
    return stochastic ? launch_quantize_forms<T, true>(st, prm) : launch_quantize_forms<T, false>(st, prm);
}

}  // namespace

cudaError_t launch_mx4_quantize(cudaStream_t st, const void *x, int dtype, int64_t rows, int64_t cols, int64_t ld,
                                bool stochastic, uint64_t seed, uint32_t node, uint8_t *codes, uint8_t *scales,
                                uint8_t *codes_t, uint8_t *scales_t)
{
    QuantParams prm;
    prm.ct = (int)tiles_of(cols, 128);
    prm.x = x; prm.rows = rows; prm.cols = cols; prm.ld = ld;
    prm.seed_w = seed_word(seed, node);
    prm.codes = codes; prm.scales = scales; prm.codes_t = codes_t; prm.scales_t = scales_t;
    const size_t size = dtype == GVQ_F32 ? 4 : 2;
    const auto starts_at = [&](unsigned bytes) { return reinterpret_cast<uintptr_t>(x) % bytes == 0 && (rows == 1 || (ld * size) % bytes == 0); };
    prm.vec = starts_at(32) ? 2 : starts_at(16) ? 1 : 0;
    if (dtype == GVQ_F32) return launch_quantize_rounding<float>(st, prm, stochastic);
    if (dtype == GVQ_BF16) return launch_quantize_rounding<__nv_bfloat16>(st, prm, stochastic);
    return launch_quantize_rounding<__half>(st, prm, stochastic);
}

cudaError_t launch_mx4_quantize_aggregate(cudaStream_t st, int num_sms, int d, int64_t S, const TileTable &tiles, const LayerTables &lt,
                                          const NodePtrs<const float> &g, int n_nodes, uint32_t node0, bool stochastic,
                                          uint64_t seed, float *out, const NodePtrs<uint8_t> *codes,
                                          const NodePtrs<uint8_t> *scales)
{
    AggParams prm;
    prm.n_tiles = tiles.n_tiles;
    prm.n_tails = out ? lt.n_tails : 0;
    if (prm.n_tiles + prm.n_tails == 0) return cudaSuccess;
    prm.tail_off = lt.tail_off; prm.tail_len = lt.tail_len;
    prm.d = d; prm.n_nodes = n_nodes;
    for (int n = 0; n < n_nodes; ++n) prm.seed_w[n] = seed_word(seed, node0 + (uint32_t)n);
    for (int n = 0; n < GVQ_MAX_NODES; ++n) {
        prm.codes.p[n] = codes ? codes->p[n] : nullptr;
        prm.scales.p[n] = scales ? scales->p[n] : nullptr;
    }
    prm.tile_layer = tiles.layer; prm.tile_row0 = tiles.row0; prm.layer_S = lt.S;
    prm.layer_off = lt.off; prm.layer_soff = lt.soff;
    prm.g = g; prm.out = out;
    if (codes && S > 0) {
        mx4_clear_scale_padding_kernel<<<dim3(32, n_nodes), 256, 0, st>>>(prm.scales, S, (d + kBlock - 1) / kBlock);
        cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    prm.shares = tiles.n_tiles > 0 ? max(1, min((d + kBlock - 1) / kBlock, 4 * num_sms / tiles.n_tiles)) : 1;
    const int n = prm.n_tiles * prm.shares + prm.n_tails;
    if (stochastic) return codes ? ptx::launch_chained<mx4_quantize_aggregate_kernel<true, true>>(prm, n, 256, 0, 1, st)
                                 : ptx::launch_chained<mx4_quantize_aggregate_kernel<true, false>>(prm, n, 256, 0, 1, st);
    return codes ? ptx::launch_chained<mx4_quantize_aggregate_kernel<false, true>>(prm, n, 256, 0, 1, st)
                 : ptx::launch_chained<mx4_quantize_aggregate_kernel<false, false>>(prm, n, 256, 0, 1, st);
}

cudaError_t launch_mx4_dequantize(cudaStream_t st, int num_sms, const NodePtrs<const uint8_t> &codes,
                                  const NodePtrs<const uint8_t> &scales, int n_nodes, int64_t rows, int64_t cols, float *out,
                                  int64_t ld, const LayerTables *lt, int n_layers)
{
    if (rows == 0 || cols == 0) return cudaSuccess;
    DeqParams prm;
    prm.n_nodes = n_nodes; prm.rows = rows; prm.cols = cols; prm.ld = ld; prm.d = (int)cols;
    prm.n_layers = n_layers;
    prm.layer_off = lt ? lt->off : nullptr; prm.layer_soff = lt ? lt->soff : nullptr; prm.layer_S = lt ? lt->S : nullptr;
    prm.codes = codes; prm.scales = scales; prm.out = out;
    prm.vec = (reinterpret_cast<uintptr_t>(out) & 15u) == 0 && (lt ? cols % 4 == 0 : (rows == 1 || ld % 4 == 0));
    const int64_t items = rows * blocks(cols) * 4;
    const int grid = (int)min((int64_t)num_sms * 16, (items + 255) / 256);
    if (lt) mx4_dequantize_kernel<true><<<grid, 256, 0, st>>>(prm);
    else mx4_dequantize_kernel<false><<<grid, 256, 0, st>>>(prm);
    return cudaGetLastError();
}

}  // namespace gvq
