// Products on the tcgen05 tensor path of 16-bit or 8-bit integer operands,  D[m][n] = sum_k A[m][k] B[n][k],  with what
// follows a product done where its sums are read back: scales, the gated block's activation and product.  Kernel and host
// side shared by product_i8.cu, gated_product.cu and gated_gradient.cu, each of which makes the forms it needs.
//
// Operands come by TMA (128-byte swizzle, zero fill outside), K-major (a row of the contraction is contiguous) or MN-major (a
// row across it is; 16-bit types only).  A stage is 128 bytes of contraction of either: 64 entries of 16 bits or 128 of 8, four
// MMAs.  Tiles are CG * 128 rows of A x BN rows of B.
//   CG = 2, BN = 256, 128   a pair of CTAs on two SMs; each holds its own 128 rows of A and half of B's rows, the even one issues
//                      MMAs that read both: 64 (96) bytes a clock and SM from L2, where a CTA alone on 128 x 128 would ask for 128.
//                      Gated: B's first half are rows of the gate's weights (the even CTA's), the second of the other
//                      projection's, so that the accumulator holds both values of an output.
//   CG = 1, BN = 64    one CTA: products too small to give every SM a large tile.  Gated: 32 rows of either matrix.
//   CG = 1, FEW        few rows (tokens): they become B, the tile as narrow as they are (BN = 16, 32 or 64) against rows_a rows
//                      of weights, as many as spread them evenly over the SMs (the MMA takes 128; what the others hold is not
//                      looked at).  Gated: rows_a rows of either matrix, one below the other, so that a step of the contraction is
//                      one MMA; the two sums of an output meet in shared memory.
// Where CG = 1 leaves SMs without a tile, a cluster of up to eight CTAs shares a tile's contraction; each leaves its sums in its
// shared memory, and they add them up across the cluster, always in the same order.
//   warp 0      producer, one lane
//   warp 1      MMA issuer, one lane (the order of issue is the order of execution)
//   warps 2-9   epilogue: accumulator -> registers -> staging -> output along its rows
// Accumulators alternate between two column ranges of tensor memory.  Every mbarrier wait is bounded.
//
// What bounds it, measured: large tiles the tensor pipe (8192 x 16384 x 4096 in 8 bits 338 us, 3.25 POP/s, twice the measured bf16 rate;
// the gated block 8192 x 8192 x 4096 in bf16 687 us, 1.60 PFLOP/s, where the library's product of the same size alone takes 675); short
// contractions the epilogue (8192 x 4096 x 512 in 8 bits 31 us of which 15 are the tiles; gated 57, of which 40; instructions, and the
// exponentials' and quotients' unit); few tokens the weights' way from memory (1 x 4096 x 8192 gated 26 us, 5.2 TB/s); small ones
// the chain of a launch, 1 us to the first stage, 0.2 us a stage and 1 to 2 us for the outputs (333 x 1024 x 512 gated 5.5 us).
#pragma once
#include "activation.cuh"
#include "gvq_internal.h"
#include "row32.cuh"
#include "sm100_ptx.cuh"

#include <type_traits>

namespace gvq {
namespace product {

using namespace ptx;

constexpr int NTHREADS = 320;
constexpr int kHalves = 2;             // epilogue warps that share a quarter of the tile's rows, every other 32 columns each
constexpr int kJoinPitch = 129;        // (a row's words of 16 bytes, eight lanes' of them, lie in different banks)
constexpr int kWindow = 12;            // words of a lane's sector of shared memory: 8, and 4 that spread the lanes over the banks
constexpr int kBox = 8192;             // an MN-major box: 64 entries (128 bytes) x 64 steps of the contraction
constexpr uint32_t A_BYTES = 128 * 128;

enum { k16 = 0, kI8 = 1 };             // kinds of operands

struct Params {
    CUtensorMap a[4], b[4];            // see the producer
    int64_t M, N;                      // rows of A (of one half), rows of B, as far as there are outputs
    int tiles_m, tiles_n;              // tiles_m: of both halves
    int half_tiles;                    // tiles_m of one half: two products with B in common are one, A's and the outputs' halves apart
    int n_stages, seg_stages, segments;     // stages of a tile's contraction, of one of its segments (all alike), segments
    int n_last;                        // MMAs of a segment's last stage
    int parts;                         // CTAs (a cluster) that share a tile's contraction; with more than one, a tile a cluster
    int group;                         // tiles along M that are gone through before the next along N
    int rows_a, stages;                // FEW: rows of a matrix that a tile has (a multiple of 8); stages that there is room for
    void *out[3];                      // the product of either half; or the block's output, its gate and its other projection
    int64_t ld[3];
    int align[3];                      // bytes at whose multiples the outputs' rows start: 32, 16 or less
    int dtype, act, bf16;              // outputs' type; activation; operands' type, of 16 bits
    const float *scale_m[2], *scale_n[2];   // of 8-bit operands
    const float *unscale;              // of 16-bit operands that are held times a power of two: the sums' factor; null: 1
    int32_t *error_word;
    int wait_kcycles, test_drop;
    int a_mn;                          // of two problems in a launch: this one's A is MN-major
};
// Two products of the same form in one launch, each on CTAs of its own.
struct Pair {
    Params p[2];
    int blocks;                        // CTAs of the first
};

__device__ __forceinline__ const Params &params_of(const Params &p, int) { return p; }
__device__ __forceinline__ const Params &params_of(const Pair &p, int which) { return p.p[which]; }

template <int CG, int BN, bool FEW> struct Shape {
    static constexpr uint32_t B_BYTES = BN / CG * 128, LOADED = A_BYTES + B_BYTES;
    static constexpr uint32_t ROOM = FEW ? 168 * 1024 : 200 * 1024;   // for the stages
    static constexpr int MOST = 16, STAGES = FEW ? MOST : (int)(ROOM / LOADED) < 8 ? (int)(ROOM / LOADED) : 8;
    // sums on their way to other threads: of few rows behind the stages (and behind what the MMA reads past the last of them, 128 rows
    // of A that may be fewer), else where the stages were
    static constexpr uint32_t JOIN = BN / 4 * kJoinPitch * 16, JOIN_AT = FEW ? ROOM + A_BYTES : 0;
    static constexpr uint32_t ALL = FEW ? (JOIN_AT + JOIN + 1023) / 1024 * 1024 : STAGES * LOADED;
    static constexpr uint32_t TMEM = 2 * BN <= 32 ? 32 : 2 * BN <= 64 ? 64 : 2 * BN <= 128 ? 128 : 2 * BN <= 256 ? 256 : 512;
    // of an epilogue warp: a sector a lane (tiles of few rows have no use for them), and its columns' scales
    static constexpr uint32_t PIECE = FEW ? 0 : 32 * kWindow * 4, STAGING = PIECE + 512;
    static constexpr size_t SMEM = (size_t)ALL + 4 * kHalves * STAGING + 512 + 1024;
    static_assert(LOADED % 1024 == 0 && SMEM <= 232448, "room");
    static_assert(CG == 2 || JOIN_AT + JOIN <= ALL, "room to join parts");
};

template <int CG>
__device__ __forceinline__ void mma_i8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    if (CG == 2)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// signed 8-bit x signed 8-bit -> 32-bit integers
__host__ __device__ constexpr uint32_t idesc_i8(int m, int n)
{
    return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

// A lane's entries of a row to global memory in the output's type.
__device__ __forceinline__ void store_one(void *out, int dtype, int64_t at, float x)
{
    if (dtype == GVQ_F32) static_cast<float *>(out)[at] = x;
    else if (dtype == GVQ_BF16) static_cast<__nv_bfloat16 *>(out)[at] = from_f<__nv_bfloat16>(x);
    else static_cast<__half *>(out)[at] = from_f<__half>(x);
}
__device__ __forceinline__ uint32_t pack_as(int dtype, float a, float b)
{
    return dtype == GVQ_BF16 ? pack2<__nv_bfloat16>(a, b) : pack2<__half>(a, b);
}
// Four entries of a row; `wide`: rows of the output start at 16-byte boundaries.
__device__ __forceinline__ void store_four(void *out, int dtype, int64_t at, int64_t step, const float (&x)[4], int n, bool wide)
{
    if (wide && n >= 4) {
        if (dtype == GVQ_F32) *reinterpret_cast<float4 *>(static_cast<float *>(out) + at) = make_float4(x[0], x[1], x[2], x[3]);
        else *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(out) + at) = make_uint2(pack_as(dtype, x[0], x[1]), pack_as(dtype, x[2], x[3]));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < n) store_one(out, dtype, at + e * step, x[e]);
    }
}
// A sector of 32 bytes; a lane's 32 columns of a row that starts at one.
__device__ __forceinline__ void store32(void *p, const uint32_t (&w)[8])
{
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
}
__device__ __forceinline__ void store_row(void *out, int dtype, int64_t at, const float (&v)[32])
{
    uint32_t w[8];
    if (dtype == GVQ_F32) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(v[8 * j + i]);
            store32(static_cast<float *>(out) + at + 8 * j, w);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = pack_as(dtype, v[16 * j + 2 * i], v[16 * j + 2 * i + 1]);
            store32(static_cast<uint16_t *>(out) + at + 16 * j, w);
        }
    }
}
// Bytes lo to hi of a sector at `from` (shared memory) to the same places from `to` on; both are even.
__device__ __forceinline__ void store_bytes(char *to, const uint32_t *from, int lo, int hi)
{
    auto move = [&](auto unit) {
        using U = decltype(unit);
        *reinterpret_cast<U *>(to + lo) = *reinterpret_cast<const U *>(reinterpret_cast<const char *>(from) + lo);
        lo += (int)sizeof(U);
    };
    if ((lo & 2) && lo + 2 <= hi) move(uint16_t{});
    if ((lo & 4) && lo + 4 <= hi) move(uint32_t{});
    if ((lo & 8) && lo + 8 <= hi) move(uint2{});
    if (hi - lo >= 16) move(uint4{});
    if (hi - lo >= 8) move(uint2{});
    if (hi - lo >= 4) move(uint32_t{});
    if (hi - lo >= 2) move(uint16_t{});
}
// `cols` columns of a warp's rows, which start anywhere; value(c, x) gives the lane's 16 entries from column c on.  L2 takes a 32-byte
// sector in parts at a fraction of the rate at which it takes it whole, so only whole ones are written but for a row's first and last
// of the strip: 64 bytes at a time are shifted in registers by the row's offset within a sector (by 16, 8, 4 and 2 bytes), and what
// they begin of the next sector waits.
template <typename F>
__device__ __forceinline__ void store_strip(uint32_t *win, int lane, int dtype, void *out, int64_t at, int64_t ld, int rows, int cols, F value)
{
    const int size = dtype == GVQ_F32 ? 4 : 2, bytes = cols * size;
    char *to = static_cast<char *>(out) + (at + lane * ld) * size;
    const int phase = (int)(reinterpret_cast<uintptr_t>(to) & 31u), words = phase >> 2;
    to -= phase;
    const uint32_t shift = phase & 2 ? 16 : 0;
    const bool fine = __any_sync(0xffffffffu, phase & 15);
    uint32_t kept[7] = {}, last = 0;      // words of a sector that is not whole, the word before the next
    auto sector = [&](int place, const uint32_t (&x)[8]) {
        const int lo = max(0, phase - place), hi = min(32, phase + bytes - place);
        if (lane >= rows || lo >= hi) return;
        if (lo == 0 && hi == 32) store32(to + place, x);
        else {
            uint32_t *own = win + lane * kWindow;
            *reinterpret_cast<uint4 *>(own) = make_uint4(x[0], x[1], x[2], x[3]);
            *reinterpret_cast<uint4 *>(own + 4) = make_uint4(x[4], x[5], x[6], x[7]);
            store_bytes(to + place, own, lo, hi);
        }
    };
    int place = 0;
#pragma unroll 1
    for (int c = 0; c < cols; c += 64 / size, place += 64) {
        uint32_t y[23], x[8];
        float v[16];
        __syncwarp();      // (sums are read by a warp's lanes together)
        value(c, v);
        if (size == 4) {
#pragma unroll
            for (int k = 0; k < 16; ++k) y[k] = __float_as_uint(v[k]);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) y[k] = pack_as(dtype, v[2 * k], v[2 * k + 1]);
            value(c + 16, v);
#pragma unroll
            for (int k = 0; k < 8; ++k) y[8 + k] = pack_as(dtype, v[2 * k], v[2 * k + 1]);
        }
#pragma unroll
        for (int k = 16; k < 23; ++k) y[k] = 0;
        auto up = [&](int d) {
            const bool by = phase & (4 * d);
#pragma unroll
            for (int k = 22; k >= 0; --k) y[k] = by ? (k >= d ? y[k - d] : 0u) : y[k];
        };
        if (fine) {
            const uint32_t before = last;
            last = y[15];
#pragma unroll
            for (int k = 15; k >= 0; --k) y[k] = __funnelshift_l(k ? y[k - 1] : before, y[k], shift);
            up(1);
            up(2);
        }
        up(4);
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = k < 7 && k < words ? kept[k < 7 ? k : 0] : y[k];
        sector(place, x);
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = y[8 + k];
        sector(place + 32, x);
#pragma unroll
        for (int k = 0; k < 7; ++k) kept[k] = y[16 + k];
    }
    uint32_t x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = k < 7 && k < words ? kept[k < 7 ? k : 0] : last >> 16;      // (of an odd row, an entry that is left)
    sector(place, x);
}

// A tile's place: tiles go through groups of `group` tiles along M, so that the operands of the tiles at work at a time lie
// in L2.
__device__ __forceinline__ void place(const Params &prm, int tile, int &tm, int &tn)
{
    const int per = prm.group * prm.tiles_n, g = tile / per, r = tile - g * per;
    const int m = min(prm.group, prm.tiles_m - g * prm.group);
    tn = r / m;
    tm = g * prm.group + r - tn * m;
}

// The segment of a stage.
__device__ __forceinline__ int segment_of(const Params &prm, int st)
{
    return (st >= prm.seg_stages) + (st >= 2 * prm.seg_stages) + (st >= 3 * prm.seg_stages);
}

// A sum of codes times its scales, of A's row and of B's: the tokens' before the weights', so that a token's results have the same bits in
// every form.
template <bool FEW>
__device__ __forceinline__ float scaled(int sum, float of_a, float of_b)
{
    const float x = __int2float_rn(sum);
    return FEW ? x * of_b * of_a : x * of_a * of_b;
}

// Sums that lie in the shared memory of the P CTAs of a cluster (of this one): added up, four columns of a row a thread at a time, the
// parts in order, and then what the epilogue does with them.  Lanes lie along what is contiguous in the output.  tid: this thread's
// place among the `threads` that do this in each CTA, whole warps.
template <int KIND, int BN, bool FEW, bool GATED, int P>
__device__ __forceinline__ void join_parts(const Params &prm, const float4 *join, int part, int tm, int tn, int tid, int threads)
{
    constexpr int HN = GATED && !FEW ? BN / 2 : BN;
    const int half = tm >= prm.half_tiles, hm = tm - half * prm.half_tiles, per = FEW ? prm.rows_a : 128;
    const int64_t m0 = (int64_t)hm * per, n0 = (int64_t)tn * HN;
    const int rows = (int)min((int64_t)per, prm.M - m0), cols = (int)min((int64_t)HN, prm.N - n0);
    const int quads = (cols + 3) / 4, inner = FEW ? rows : quads, total = rows * quads;
    uint32_t from[P];
    if constexpr (P > 1) {
#pragma unroll
        for (int p = 0; p < P; ++p) from[p] = cluster_address(smem_u32(join), p);
    }
    auto one = [&](int it) {
        const int o = it / inner, i = it - o * inner, c4 = FEW ? o : i, r = FEW ? i : o;
        const int n = cols - c4 * 4;
        const int64_t m = m0 + r, col = n0 + c4 * 4;
        auto value = [&](int which, float (&y)[4]) {
            const int at = (c4 + (FEW ? 0 : which * HN / 4)) * kJoinPitch + r + (FEW ? which * prm.rows_a : 0);
            float4 x[P];
#pragma unroll
            for (int p = 0; p < P; ++p) x[p] = P > 1 ? load_cluster(from[p] + at * 16) : join[at];
            if constexpr (KIND == kI8) {
                int s[4] = {0, 0, 0, 0};
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    s[0] += __float_as_int(x[p].x); s[1] += __float_as_int(x[p].y);
                    s[2] += __float_as_int(x[p].z); s[3] += __float_as_int(x[p].w);
                }
                const float sm = prm.scale_m[FEW ? which : 0][m];
                const float *sn = prm.scale_n[FEW ? 0 : which] + col;
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = e < n ? scaled<FEW>(s[e], sm, sn[e]) : 0.0f;
            } else {
#pragma unroll
                for (int p = 1; p < P; ++p) { x[0].x += x[p].x; x[0].y += x[p].y; x[0].z += x[p].z; x[0].w += x[p].w; }
                const float f = !GATED && prm.unscale ? __ldcg(prm.unscale) : 1.0f;
                y[0] = x[0].x * f; y[1] = x[0].y * f; y[2] = x[0].z * f; y[3] = x[0].w * f;
            }
        };
        auto store = [&](int k, const float (&y)[4]) {
            const int64_t ld = prm.ld[k];
            store_four(prm.out[k], prm.dtype, FEW ? m + col * ld : m * ld + col, FEW ? ld : 1, y, n, !FEW && prm.align[k] >= 16);
        };
        if constexpr (GATED) {
            float g[4], u[4], h[4];
            value(0, g);
            value(1, u);
#pragma unroll
            for (int e = 0; e < 4; ++e) h[e] = activation(prm.act, g[e]) * u[e];
            store(0, h);
            if (prm.out[1]) { store(1, g); store(2, u); }
        } else {
            float y[4];
            value(0, y);
            store(half, y);
        }
    };
    // (a warp's lanes go round together: what follows are barriers and a dealloc that its lanes take as one)
#pragma unroll 1
    for (int it0 = part * threads + (tid & ~31); it0 < total; it0 += P * threads) {
        const int it = it0 + (tid & 31);
        if (it < total) one(it);
        __syncwarp();
    }
}
// The epilogue's warps alone: all of them have come here, and whether `ok` held for all.
__device__ __forceinline__ bool epilogue_and(bool ok)
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, 1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"((uint32_t)ok), "n"(32 * 4 * kHalves) : "memory");
    return r != 0;
}

template <int KIND, int CG, int BN, bool FEW, bool A_MN, bool B_MN, bool GATED, bool PAIR = false>
__global__ void __launch_bounds__(NTHREADS, 1) product_kernel(const __grid_constant__ std::conditional_t<PAIR, Pair, Params> all)
{
    using S = Shape<CG, BN, FEW>;
    constexpr int KS = KIND == kI8 ? 128 : 64;                        // entries of the contraction a stage
    constexpr bool SIDE = GATED && !FEW;                              // both matrices lie side by side in B
    constexpr int HN = SIDE ? BN / 2 : BN;                            // columns of the output a tile has
    constexpr int BL = BN / CG;                                       // rows of B that this CTA holds
    static_assert(!(KIND == kI8 && (A_MN || B_MN)) && (!B_MN || BL % 64 == 0) && !(FEW && (CG == 2 || B_MN || PAIR)) && !(GATED && A_MN), "forms");
    int block = blockIdx.x, blocks = gridDim.x, which = 0;
    if constexpr (PAIR) {
        which = block >= all.blocks;
        blocks = which ? blocks - all.blocks : all.blocks;
        if (which) block -= all.blocks;
    }
    const Params &prm = params_of(all, which);
    const bool a_mn = PAIR ? prm.a_mn : A_MN;
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    unsigned char *staging = smem + S::ALL;
    float4 *join = reinterpret_cast<float4 *>(smem + S::JOIN_AT);     // [BN / 4][kJoinPitch]: four columns of a row
    uint64_t *bars = reinterpret_cast<uint64_t *>(staging + 4 * kHalves * S::STAGING);
    const uint32_t a_bytes = FEW ? prm.rows_a * 128 : A_BYTES, stage_bytes = (FEW && GATED ? 2 : 1) * a_bytes + S::B_BYTES;
    const uint32_t n_stage = FEW ? prm.stages : S::STAGES;
    uint64_t *full = bars, *empty = full + S::STAGES;                 // [STAGES]
    uint64_t *d_full = empty + S::STAGES;                             // [2] accumulator complete
    uint64_t *d_empty = d_full + 2;                                   // [2] accumulator read
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(d_empty + 2);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = CG == 2 ? (int)cluster_rank() : 0;
    const int parts = CG == 1 ? prm.parts : 1, part = parts > 1 ? (int)cluster_rank() : 0;
    if (threadIdx.x == 0) {
        for (int i = 0; i < S::STAGES; ++i) { mbar_init(full + i, 1); mbar_init(empty + i, 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(d_full + i, 1); mbar_init(d_empty + i, 4 * kHalves * CG); }
        *abort_flag = 0;
        const_cast<int *>(abort_flag)[2] = prm.wait_kcycles;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc<CG>(tmem_slot, S::TMEM);
    tc_fence_before();
    if (CG == 2) cluster_sync(); else __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    launch_dependents();
    const int n_tiles = prm.tiles_m * prm.tiles_n;
    const int first = block / (CG * parts), stride = blocks / (CG * parts);
    const int st0 = prm.n_stages * part / parts, st1 = prm.n_stages * (part + 1) / parts;    // this CTA's stages
    if constexpr (FEW) {
        // weights on their way to L2 while the launch before this one ends (nothing is read yet that it may write)
        if (warp == 0 && elect_one()) {
            int tm, tn;
            place(prm, first, tm, tn);
            for (int st = st0; st < min(st1, st0 + (int)n_stage); ++st) {
                const int seg = segment_of(prm, st), k = (st - seg * prm.seg_stages) * KS, m0 = tm * prm.rows_a;
                prefetch_2d(prm.a + seg, A_MN ? m0 : k, A_MN ? k : m0);
                if (A_MN && a_bytes > kBox) prefetch_2d(prm.a + seg, m0 + 64, k);
                if (GATED) prefetch_2d(prm.a + 1, k, m0);
            }
        }
        __syncwarp();
    }
    grid_dependency_wait();      // what earlier launches wrote is visible from here on
    bool failed = false;

    if (warp == 0) {
        // ------------------------------------------------------------------ producer
        if (elect_one()) {
            fence_proxy_async_global();      // what plain stores of earlier launches wrote is read by TMA
            uint32_t c = 0, s = 0, phase = 1;
            for (int tile = first; tile < n_tiles && !failed; tile += stride) {
                int tm, tn;
                place(prm, tile, tm, tn);
                const int half = tm >= prm.half_tiles;
                const int m0 = (tm - half * prm.half_tiles) * (FEW ? prm.rows_a : 128 * CG) + 128 * rank;
                const int n0 = SIDE ? tn * HN : tn * BN + BL * rank;
                for (int st = st0; st < st1; ++st, ++c) {
                    if (!mbar_poll(empty + s, phase, abort_flag)) { failed = true; break; }
                    const bool drop = prm.test_drop && blockIdx.x == 0 && c == 0;   // test hook: this stage never arrives
                    if (!drop) {
                        // a contraction of segments has a map of either operand for each; two halves have their own of A
                        const int seg = segment_of(prm, st);
                        const CUtensorMap *map_a = prm.a + half * prm.segments + seg;
                        const int k = (st - seg * prm.seg_stages) * KS;
                        unsigned char *dst = smem + s * stage_bytes, *dst_b = dst + stage_bytes - S::B_BYTES;
                        if (rank == 0) mbar_arrive_expect_tx(full + s, CG * stage_bytes);
                        const uint32_t bar = CG == 2 ? in_leader(full + s) : 0;
                        auto load = [&](unsigned char *to, const CUtensorMap *map, bool mn, int at) {
                            if (CG == 2) tma_load_2d_pair(to, map, mn ? at : k, mn ? k : at, bar);
                            else tma_load_2d(to, map, mn ? at : k, mn ? k : at, full + s);
                        };
                        load(dst, map_a, a_mn, m0);
                        if (a_mn && (!FEW || a_bytes > kBox)) load(dst + kBox, map_a, true, m0 + 64);
                        if (FEW && GATED) load(dst + a_bytes, prm.a + 1, false, m0);
                        if constexpr (SIDE && CG == 2) load(dst_b, prm.b + rank, false, n0);
                        else if constexpr (SIDE) {
                            load(dst_b, prm.b, false, n0);
                            load(dst_b + HN * 128, prm.b + 1, false, n0);
                        } else if constexpr (B_MN) {
#pragma unroll
                            for (int i = 0; i < BL / 64; ++i) load(dst_b + i * kBox, prm.b + seg, true, n0 + 64 * i);
                        } else load(dst_b, prm.b + seg, false, n0);
                    }
                    if (++s == n_stage) { s = 0; phase ^= 1; }
                }
            }
            if (failed && rank == 0) {   // give the copies already in flight a bounded chance to land before the CTA exits
                for (uint32_t i = c > n_stage ? c - n_stage : 0; i < c; ++i)
                    for (int it = 0; it < 100000 && !mbar_try_wait(full + i % n_stage, (i / n_stage) & 1); ++it) {}
            }
        }
        failed = __any_sync(0xffffffffu, failed);
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer
        if (rank == 0 && elect_one()) {
            uint32_t s = 0, phase = 0, t = 0;
            const uint32_t base = smem_u32(smem);
            const uint64_t a0 = a_mn ? make_mn_desc(base, kBox) : make_b_desc(base);
            const uint64_t b0 = B_MN ? make_mn_desc(base + stage_bytes - S::B_BYTES, kBox)
                                     : make_b_desc(base + stage_bytes - S::B_BYTES);
            // 32 bytes of a K-major row, or 16 rows of 128 bytes of an MN-major box
            const uint32_t IA = a_mn ? 16 * 128 / 16 : 2;
            constexpr uint32_t IB = B_MN ? 16 * 128 / 16 : 2;
            const uint32_t idesc = KIND == kI8 ? idesc_i8(128 * CG, BN)
                                               : make_idesc_f16(128 * CG, BN, a_mn, B_MN) | (prm.bf16 ? (1u << 7) | (1u << 10) : 0u);
            for (int tile = first; tile < n_tiles && !failed; tile += stride, ++t) {
                const uint32_t buf = t & 1, d = tmem + buf * BN;
                if (t > 1) {
                    if (!mbar_poll(d_empty + buf, ((t >> 1) - 1) & 1, abort_flag)) { failed = true; break; }
                    tc_fence_after();
                }
                int left = prm.seg_stages - (st0 - segment_of(prm, st0) * prm.seg_stages);      // stages of the segment
                for (int st = st0; st < st1; ++st) {
                    if (!mbar_poll(full + s, phase, abort_flag)) { failed = true; break; }
                    tc_fence_after();
                    const uint64_t da = a0 + s * (stage_bytes >> 4), db = b0 + s * (stage_bytes >> 4);
                    auto issue = [&](int n_mma) {      // (a constant, except in a short last stage)
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (k < n_mma) {
                                if (KIND == kI8) mma_i8<CG>(d, da + k * IA, db + k * IB, idesc, st > st0 || k > 0);
                                else tc_mma_f16<CG>(d, da + k * IA, db + k * IB, idesc, st > st0 || k > 0);
                            }
                    };
                    if (--left == 0) {
                        left = prm.seg_stages;
                        issue(prm.n_last);
                    } else issue(4);
                    if (CG == 2) tc_commit_pair(empty + s); else tc_commit(empty + s);
                    if (st == st1 - 1) { if (CG == 2) tc_commit_pair(d_full + buf); else tc_commit(d_full + buf); }
                    if (++s == n_stage) { s = 0; phase ^= 1; }
                }
            }
        }
        failed = __any_sync(0xffffffffu, failed);
    } else {
        // ------------------------------------------------------------------ epilogue
        const int q = warp & 3, side = (warp - 2) >> 2;      // a quarter of the rows; pieces of 32 columns side, side + 2, ...
        const uint32_t lane_base = (uint32_t)(32 * q) << 16;
        unsigned char *mine = staging + (warp - 2) * S::STAGING;
        float *scales = reinterpret_cast<float *>(mine + S::PIECE);      // of the columns: [matrix][piece][32]
        uint32_t t = 0;
        const int dtype = prm.dtype;
        constexpr int PW = HN < 32 ? HN : 32, NP = HN / PW;  // columns of a piece, pieces of a tile
        constexpr bool SCALED = KIND == k16 && !GATED;
        const float unscale = SCALED && prm.unscale ? __ldcg(prm.unscale) : 1.0f;
        for (int tile = first; tile < n_tiles; tile += stride, ++t) {
            int tm, tn;
            place(prm, tile, tm, tn);
            const int half = tm >= prm.half_tiles;
            const int64_t m0 = (int64_t)(tm - half * prm.half_tiles) * (FEW ? prm.rows_a : 128 * CG) + 128 * rank + 32 * q, n0 = (int64_t)tn * HN;
            const int rows = (int)max((int64_t)0, min((int64_t)(FEW ? min(32, prm.rows_a - 32 * q) : 32), prm.M - m0));
            // 8-bit operands: the scale of this lane's row, and those of the columns, which every lane reads
            constexpr int NS = (NP + kHalves - 1) / kHalves;
            float sm = 0.0f;
            if constexpr (KIND == kI8 && !(FEW && GATED)) {
                if (lane < rows) sm = __ldg(prm.scale_m[0] + m0 + lane);
#pragma unroll
                for (int i = 0; i < (SIDE ? 2 : 1); ++i)
#pragma unroll
                    for (int j = 0; j < NS; ++j) {
                        const int64_t n = n0 + 32 * (NS * side + j) + lane;
                        scales[(i * NS + j) * 32 + lane] = n < prm.N ? __ldg(prm.scale_n[i] + n) : 0.0f;
                    }
                __syncwarp();
            }
            const uint32_t buf = t & 1;
            bool ok = mbar_poll(d_full + buf, (t >> 1) & 1, abort_flag);
            // (those that go on to wait for one another below have to agree)
            ok = FEW && GATED && parts == 1 ? epilogue_and(ok) : __all_sync(0xffffffffu, ok);
            if (!ok) { failed = true; break; }
            tc_fence_after();
            const uint32_t acc = tmem + lane_base + buf * BN;
            if (parts > 1 || (FEW && GATED)) {           // sums that other threads take up
                if constexpr (CG == 1) {
#pragma unroll 1
                    for (int c = 16 * side; c < BN; c += 16 * kHalves) {
                        float v[16];
                        tmem_ld16_wait(acc + c, v);
#pragma unroll
                        for (int i = 0; i < 16; i += 4)
                            join[(c + i) / 4 * kJoinPitch + 32 * q + lane] = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                    }
                    if constexpr (FEW && GATED) {
                        if (parts == 1) {
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) mbar_arrive(d_empty + buf);
                            epilogue_and(true);
                            join_parts<KIND, BN, FEW, GATED, 1>(prm, join, 0, tm, tn, threadIdx.x - 64, 32 * 4 * kHalves);
                            epilogue_and(true);      // (the next tile's sums take their place)
                        }
                    }
                }
                continue;
            }
            // the sums of one matrix's piece p = 2 j + side
            auto sums = [&](int which, int j, float (&v)[32]) {
                const uint32_t from = acc + (SIDE ? which * HN : 0) + 32 * (NS * side + j);
                if constexpr (PW == 32) tmem_ld32_wait(from, v);
                else {
                    float w[16];
                    tmem_ld16_wait(from, w);
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = i < 16 ? w[i] : 0.0f;
                }
                if constexpr (KIND == kI8) {
                    const float4 *of = reinterpret_cast<const float4 *>(scales + ((SIDE ? which : 0) * NS + j) * 32);
#pragma unroll
                    for (int i = 0; i < PW; i += 4) {
                        const float4 x = of[i / 4];
                        v[i] = scaled<FEW>(__float_as_int(v[i]), sm, x.x);
                        v[i + 1] = scaled<FEW>(__float_as_int(v[i + 1]), sm, x.y);
                        v[i + 2] = scaled<FEW>(__float_as_int(v[i + 2]), sm, x.z);
                        v[i + 3] = scaled<FEW>(__float_as_int(v[i + 3]), sm, x.w);
                    }
                }
                if constexpr (SCALED) {
#pragma unroll
                    for (int i = 0; i < PW; ++i) v[i] *= unscale;
                }
            };
            if constexpr (FEW) {       // rows of A run along the output's rows: a warp's lanes do too
#pragma unroll 1
                for (int j = 0; j < NS && NS * side + j < NP; ++j) {
                    const int64_t n = n0 + 32 * (NS * side + j);
                    const int cols = (int)min((int64_t)PW, prm.N - n);
                    if (rows <= 0 || cols <= 0) break;
                    float v[32];
                    __syncwarp();
                    sums(0, j, v);
                    if (lane < rows) {
#pragma unroll
                        for (int i = 0; i < PW; ++i)
                            if (i < cols) store_one(prm.out[half], dtype, m0 + lane + (n + i) * prm.ld[half], v[i]);
                    }
                }
            } else {
                // this warp's columns, side by side
                const int64_t n = n0 + 32 * NS * side;
                const int cols = (int)min((int64_t)32 * min(NS, NP - NS * side), prm.N - n);
                const bool all = SIDE && prm.out[1];
                const bool direct = prm.align[half] == 32 && (!all || (prm.align[1] == 32 && prm.align[2] == 32));
                if (rows > 0 && cols > 0) {
                    int j = 0;
                    if (direct) {
#pragma unroll 1
                        for (; 32 * (j + 1) <= cols; ++j) {
                            float v[32];
                            __syncwarp();
                            sums(0, j, v);
                            auto store = [&](int slot, const float (&x)[32]) {
                                if (lane < rows) store_row(prm.out[slot], dtype, (m0 + lane) * prm.ld[slot] + n + 32 * j, x);
                            };
                            if constexpr (SIDE) {
                                float u[32];
                                sums(1, j, u);
                                if (all) {
                                    store(1, v);
                                    store(2, u);
                                }
                                activate(prm.act, v, u);
                                store(0, v);
                            } else store(half, v);
                        }
                    }
                    const int left = cols - 32 * j;
                    if (left > 0) {
                        // 16 sums of one matrix from column c of the strip on
                        auto sixteen = [&](int which, int c, float (&x)[16]) {
                            tmem_ld16_wait(acc + (SIDE ? which * HN : 0) + 32 * NS * side + c, x);
                            if constexpr (KIND == kI8) {
                                const float *of = scales + (SIDE ? which : 0) * NS * 32 + c;
#pragma unroll
                                for (int i = 0; i < 16; ++i) x[i] = scaled<FEW>(__float_as_int(x[i]), sm, of[i]);
                            }
                            if constexpr (SCALED) {
#pragma unroll
                                for (int i = 0; i < 16; ++i) x[i] *= unscale;
                            }
                        };
#pragma unroll 1
                        for (int slot = all ? 2 : half; slot >= (SIDE ? 0 : half); --slot)
                            store_strip(reinterpret_cast<uint32_t *>(mine), lane, dtype, prm.out[slot], m0 * prm.ld[slot] + n + 32 * j,
                                        prm.ld[slot], rows, left, [&](int c, float (&x)[16]) {
                                            sixteen(SIDE && slot == 2 ? 1 : 0, 32 * j + c, x);
                                            if constexpr (SIDE) {
                                                if (slot == 0) {
                                                    float u[16];
                                                    sixteen(1, 32 * j + c, u);
                                                    activate(prm.act, x, u);
                                                }
                                            }
                                        });
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) { if (CG == 2) mbar_arrive_cluster(in_leader(d_empty + buf)); else mbar_arrive(d_empty + buf); }
        }
    }

    if constexpr (CG == 1) {
        if (parts > 1) {
            cluster_sync();
            if (!failed) {
                int tm, tn;
                place(prm, first, tm, tn);
                if (parts == 2) join_parts<KIND, BN, FEW, GATED, 2>(prm, join, part, tm, tn, threadIdx.x, NTHREADS);
                else if (parts == 4) join_parts<KIND, BN, FEW, GATED, 4>(prm, join, part, tm, tn, threadIdx.x, NTHREADS);
                else join_parts<KIND, BN, FEW, GATED, 8>(prm, join, part, tm, tn, threadIdx.x, NTHREADS);
            }
        }
    }
    if (failed) {
        *abort_flag = 1;
        if (lane == 0) atomicExch(prm.error_word, 120 + warp);
    }
    tc_fence_before();
    __syncwarp();
    // (the other CTAs of a cluster use this one's barriers and memory until here)
    if (CG == 2 || parts > 1) cluster_sync(); else __syncthreads();
    tc_fence_after();
    __syncwarp();
    if (warp == 1) tmem_dealloc<CG>(tmem, S::TMEM);
}

// ---------------------------------------------------------------------------------------------------- host side
inline int tiles_of(int64_t n, int per) { return (int)((n + per - 1) / per); }

template <int KIND, int CG, int BN, bool FEW, bool A_MN, bool B_MN, bool GATED>
cudaError_t launch(cudaStream_t st, int num_sms, const Params &prm)
{
    using S = Shape<CG, BN, FEW>;
    const int cluster = CG * prm.parts;
    const int64_t tiles = (int64_t)prm.tiles_m * prm.tiles_n;
    return launch_chained<product_kernel<KIND, CG, BN, FEW, A_MN, B_MN, GATED>>(
        prm, cluster * (int)(tiles < num_sms / cluster ? tiles : num_sms / cluster), NTHREADS, S::SMEM, cluster, st);
}

template <int KIND, int CG, int BN, bool B_MN>
cudaError_t launch_pair(cudaStream_t st, const Pair &pair, const int (&blocks)[2])
{
    using S = Shape<CG, BN, false>;
    const int parts = pair.p[0].parts > pair.p[1].parts ? pair.p[0].parts : pair.p[1].parts;
    return launch_chained<product_kernel<KIND, CG, BN, false, false, B_MN, false, true>>(pair, blocks[0] + blocks[1], NTHREADS, S::SMEM,
                                                                                     CG * parts, st);
}

// A matrix [rows][cols] of 16-bit or 8-bit entries, rows ld entries apart and starting at 16-byte boundaries: boxes of 128 bytes of
// a row by `box_rows` rows.
inline bool encode(EncodeTiledFn enc, CUtensorMap *map, int kind, const void *p, int64_t rows, int64_t cols, int64_t ld, int box_rows)
{
    const int size = kind == kI8 ? 1 : 2;
    cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    cuuint64_t strides[1] = {(cuuint64_t)(ld * size)};
    cuuint32_t box[2] = {(cuuint32_t)(128 / size), (cuuint32_t)box_rows};
    cuuint32_t estr[2] = {1, 1};
    return enc(map, kind == kI8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, const_cast<void *>(p), dims, strides,
               box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Output `slot`, rows ld entries apart.
inline void set_output(Params &prm, int slot, void *out, int dtype, int64_t ld)
{
    prm.out[slot] = out;
    prm.ld[slot] = ld;
    const uint64_t at = reinterpret_cast<uintptr_t>(out) | (uint64_t)(ld * (dtype == GVQ_F32 ? 4 : 2));
    prm.align[slot] = at % 32 == 0 ? 32 : at % 16 == 0 ? 16 : 1;
}

// How a product of M rows of tokens and N outputs is cut up.
struct Cut {
    bool few;          // the tokens are B: A and B, M and N change places
    int cg, bn;        // of the kernel
    int rows_a, parts;
    double time;       // expected, in microseconds
};

// Parts of a contraction of n stages where a CTA has a tile alone: as many as there are SMs for, of `least` stages at least.  Clusters
// of four fill 128 of 148 SMs and those of eight fewer (the SMs of a cluster lie together); one more than fit takes a wave of its
// own (8 x 2048 x 1024 gated in 37 clusters of four 14 us, in 32 of them 8).
inline int parts_of(int num_sms, int64_t tiles, int n, int least)
{
    int parts = 1;
    while (parts < 8 && tiles * 2 * parts <= (parts == 1 ? num_sms : parts == 2 ? num_sms * 7 / 8 : num_sms * 2 / 3) &&
           n >= 2 * parts * least)
        parts *= 2;
    return parts;
}
// What bringing parts together takes, in microseconds.
inline double join_cost(int parts) { return parts > 1 ? 1.2 + 0.3 * parts : 0.0; }

// Tiles: of the forms, the one with the least time in microseconds by what was measured: a tile's stages, its epilogue where that
// takes longer than another tile's stages, and once what a launch, the pipeline's start and the last epilogue take.  (In 8 bits, us, with
// 256, 128 and 64 columns: 777 x 515 x 1083 9.5, 7.7, 6.5; 512 x 4096 x 4096 16.2, 12.3, 17.4; 2048 x 8192 x 4096 47, 53, 94;
// 8192 x 16384 x 4096 344, 424, 705; 300 x 300 x 8192 24, 17, 16, with four parts of 64 columns 9.2.)
struct Form { int cg, bn; double stage, epilogue, once; };
static const Form kForms[3] = {{2, 256, 0.29, 3.6, 6.2}, {2, 128, 0.21, 2.6, 4.7}, {1, 64, 0.21, 1.4, 3.8}};
inline Cut cut_tiles(int num_sms, int64_t M, int64_t N, bool gated, int n, int halves)
{
    Cut best = {};
    for (const Form &f : kForms) {
        const int64_t tiles = (int64_t)halves * tiles_of(M, 128 * f.cg) * tiles_of(N, f.bn / (gated ? 2 : 1));
        const int slots = num_sms / f.cg;
        const int most = f.cg == 1 ? parts_of(num_sms, tiles, n, 4) : 1;
        for (int parts = 1; parts <= most; parts *= 2) {
            const double own = f.stage * ((n + parts - 1) / parts), more = own > f.epilogue ? own : f.epilogue;
            const double t = f.once + own + join_cost(parts) + more * (double)((tiles * parts + slots - 1) / slots - 1);
            if (!best.cg || t < best.time) best = {false, f.cg, f.bn, 128, parts, t};
        }
    }
    return best;
}

// Two products in one launch: each on SMs of its own, so that both end at about the same time.  dx and both weights' gradients of a
// block, with the slopes: 777 x 515 x 1029 21.5 us in one launch, 27.0 in two; 2048 x 1024 x 2048 35.4 and 43.1; 1024 x 1024 x 4096 40.5
// and 54; 8192 x 4096 x 8192, where either fills the SMs seven times and more, takes two.
struct PairCut {
    Cut c[2];
    int blocks[2];
    double time;
};
struct Extent { int64_t M, N; int n, halves; };      // of a product; n: stages of its contraction
inline PairCut cut_pair(int num_sms, const Extent (&e)[2])
{
    PairCut best = {};
    for (const Form &f : kForms) {
        int64_t tiles[2];
        double own[2], more[2];
        for (int i = 0; i < 2; ++i) tiles[i] = (int64_t)e[i].halves * tiles_of(e[i].M, 128 * f.cg) * tiles_of(e[i].N, f.bn);
        // parts of the one's contraction and of the other's: one, or as many as a cluster has CTAs
        for (int cluster = 1; cluster <= (f.cg == 1 ? 8 : 1); cluster *= 2) {
            const int slots = (cluster <= 2 ? num_sms : cluster == 4 ? num_sms * 7 / 8 : num_sms * 2 / 3) / (f.cg * cluster) * cluster;
            for (int which = cluster == 1 ? 0 : 1; which < (cluster == 1 ? 1 : 4); ++which) {      // (bit i: of product i)
                const int parts[2] = {which & 1 ? cluster : 1, which & 2 ? cluster : 1};
                bool fits = true;
                for (int i = 0; i < 2; ++i) {
                    fits = fits && (parts[i] == 1 || (e[i].n >= 4 * parts[i] && tiles[i] * parts[i] < slots));
                    own[i] = f.stage * ((e[i].n + parts[i] - 1) / parts[i]) + join_cost(parts[i]);
                    more[i] = own[i] > f.epilogue ? own[i] : f.epilogue;
                }
                // rounds of the first's tiles; past eight of them two launches are as good
                for (int rounds = 1; fits && rounds <= (parts[0] > 1 ? 1 : 8) && rounds <= tiles[0]; ++rounds) {
                    const int64_t first = ((tiles[0] * parts[0] + rounds - 1) / rounds + cluster - 1) / cluster * cluster;
                    if (first >= slots) continue;
                    const int64_t need = (tiles[1] * parts[1] + cluster - 1) / cluster * cluster, second = need < slots - first ? need : slots - first;
                    if (parts[1] > 1 && second < need) continue;
                    const double a = own[0] + more[0] * (rounds - 1);
                    const double b = own[1] + more[1] * (double)((tiles[1] * parts[1] + second - 1) / second - 1);
                    const double t = f.once + (a > b ? a : b);
                    if (!best.time || t < best.time)
                        best = {{{false, f.cg, f.bn, 128, parts[0], t}, {false, f.cg, f.bn, 128, parts[1], t}},
                                {(int)first * f.cg, (int)second * f.cg}, t};
                }
            }
        }
    }
    return best;
}

// Few tokens: the weights' rows are spread over the SMs, step rows at a time.  A stage takes its bytes' time or, where they are few, that
// of its four MMAs.  (In 8 bits, us: 16 x 4096 -> 16384 with 112 rows a tile 17.4, 96 21.7, 64 20.4, 32 31.9; 1 x 2048 -> 1000 with 96
// rows 6.4, of four parts 4.8, of eight 5.2; 40 x 4096 -> 4096 with 64 rows 11.5, of two parts 9.2.)
inline Cut cut_few(int num_sms, int64_t M, int64_t N, bool gated, int n, int step)
{
    const int na = gated ? 2 : 1;
    Cut best = {};
    best.few = true;
    best.cg = 1;
    best.bn = M <= 16 ? 16 : M <= 32 ? 32 : 64;
    double least = 0;
    for (int rows = step; rows * na <= 128; rows += step) {
        const int64_t tiles = (int64_t)tiles_of(N, rows) * tiles_of(M, best.bn);
        const int most = parts_of(num_sms, tiles, n, 2);
        const double bytes = rows * na * 128 / 44e3, stage = bytes > 0.21 ? bytes : 0.21;
        for (int parts = 1; parts <= most; parts *= 2) {
            const double t = stage * ((n + parts - 1) / parts) * (double)((tiles * parts + num_sms - 1) / num_sms) + join_cost(parts);
            if (!best.rows_a || t <= least) { best.rows_a = rows; best.parts = parts; least = t; }
        }
    }
    return best;
}

// n: stages of the contraction; step: of rows_a.
inline Cut cut(int num_sms, int64_t M, int64_t N, bool gated, int n, int step = 8)
{
    return M <= 64 ? cut_few(num_sms, M, N, gated, n, step) : cut_tiles(num_sms, M, N, gated, n, 1);
}
inline int stages_of(int64_t K, int kind) { return tiles_of(K, kind == kI8 ? 128 : 64); }

// Fills in how the product is gone through.  out_n: columns of the output a tile has; K: of a segment of the contraction.
inline void divide(Params &prm, const Cut &c, int kind, bool gated, int64_t K, int segments, int halves)
{
    const int ks = kind == kI8 ? 128 : 64;
    prm.rows_a = c.few ? c.rows_a : 128;
    prm.half_tiles = tiles_of(prm.M, c.few ? c.rows_a : 128 * c.cg);
    prm.tiles_m = prm.half_tiles * halves;
    prm.tiles_n = tiles_of(prm.N, gated && !c.few ? c.bn / 2 : c.bn);
    prm.seg_stages = tiles_of(K, ks);
    prm.segments = segments;
    prm.n_stages = prm.seg_stages * segments;
    prm.n_last = (int)((K - (int64_t)(prm.seg_stages - 1) * ks + ks / 4 - 1) / (ks / 4));
    prm.group = prm.tiles_m < 8 ? prm.tiles_m : 8;
    prm.parts = c.parts;
    if (halves == 1) prm.half_tiles = prm.tiles_m;
    const int stage = (gated ? 2 : 1) * c.rows_a * 128 + c.bn * 128, room = Shape<1, 16, true>::ROOM / stage;
    prm.stages = room < Shape<1, 16, true>::MOST ? room : Shape<1, 16, true>::MOST;      // (of few rows)
}

}  // namespace product
}  // namespace gvq
