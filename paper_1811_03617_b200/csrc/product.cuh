// Products on the tcgen05 tensor path of 16-bit or 8-bit integer operands,  D[m][n] = sum_k A[m][k] B[n][k],  with what
// follows a product done where its sums are read back: scales, the gated block's activation and product.  Kernel and host
// side shared by product_i8.cu, gated_product.cu and gated_gradient.cu, each of which makes the forms it needs.
//
// Operands come by TMA (128-byte swizzle, zero fill outside), K-major (a row of the contraction is contiguous) or MN-major (a
// row across it is; 16-bit types only).  A stage is 128 bytes of contraction of either: 64 entries of 16 bits or 128 of 8, four
// MMAs.  Tiles are CG * 128 rows of A x BN rows of B.
//   CG = 2, BN = 256   a pair of CTAs on two SMs; each holds its own 128 rows of A and half of B's rows, the even one issues
//                      MMAs that read both: 64 bytes a clock and SM from L2, half of what a CTA alone on 128 x 128 would ask for.
//                      Gated: B's first half are rows of the gate's weights (the even CTA's), the second of the other
//                      projection's, so that the accumulator holds both values of 128 outputs.
//   CG = 1, BN = 64    one CTA: products too small to give every SM a large tile.  Gated: 32 rows of either matrix.
//   CG = 1, NA tiles   few rows (tokens): they become B, the tile as narrow as they are (BN = 16, 32 or 64) against NA * 128 rows
//                      of weights; gated: NA = 2, a tile of either matrix.
// Where CG = 1 leaves SMs without a tile, a cluster of up to eight CTAs shares a tile's contraction; each leaves its sums in its
// shared memory, where the stages were, and they add them up across the cluster, always in the same order.
//   warp 0      producer, one lane
//   warp 1      MMA issuer, one lane (the order of issue is the order of execution)
//   warps 2-5   epilogue: accumulator -> registers -> staging -> output along its rows
// Accumulators alternate between two column ranges of tensor memory.  Every mbarrier wait is bounded.
#pragma once
#include "activation.cuh"
#include "gvq_internal.h"
#include "row32.cuh"
#include "sm100_ptx.cuh"

namespace gvq {
namespace product {

using namespace ptx;

constexpr int NTHREADS = 192;
constexpr int kJoinPitch = 129;        // (a row's words of 16 bytes, eight lanes' of them, lie in different banks)
constexpr int kBox = 8192;             // an MN-major box: 64 entries (128 bytes) x 64 steps of the contraction
constexpr uint32_t A_BYTES = 128 * 128;

enum { k16 = 0, kI8 = 1 };             // kinds of operands

struct Params {
    CUtensorMap a[2], b[2];            // see the producer
    CUtensorMap o[3];                  // outputs, boxes of 128 bytes x 32 rows (where tma_out says so)
    int64_t M, N;                      // rows of A (of one half), rows of B, as far as there are outputs
    int tiles_m, tiles_n;              // tiles_m: of both halves
    int half_tiles;                    // tiles_m of one half: two products with B in common are one, A's and the outputs' halves apart
    int n_stages, seg_stages, n_last;  // stages of a tile's contraction, of its first segment; MMAs of a segment's last stage
    int parts;                         // CTAs (a cluster) that share a tile's contraction; with more than one, a tile a cluster
    int group;                         // tiles along M that are gone through before the next along N
    int swapped;                       // rows of A run along the output's rows
    void *out[3];                      // the product of either half; or the block's output, its gate and its other projection
    int64_t ld[3];
    int tma_out;                       // a bit an output
    int dtype, act, bf16;              // outputs' type; activation; operands' type, of 16 bits
    const float *scale_m[2], *scale_n[2];   // of 8-bit operands
    int32_t *error_word;
    int wait_kcycles, test_drop;
};

template <int CG, int BN, int NA> struct Shape {
    static constexpr uint32_t B_BYTES = BN / CG * 128;
    static constexpr uint32_t LOADED = NA * A_BYTES + B_BYTES, STAGE = LOADED;
    static constexpr int STAGES = CG == 2 ? 6 : (int)(200 * 1024 / STAGE) < 8 ? (int)(200 * 1024 / STAGE) : 8;
    static constexpr uint32_t ACC = NA * BN;                          // columns of an accumulator
    static constexpr uint32_t TMEM = 2 * ACC <= 32 ? 32 : 2 * ACC <= 64 ? 64 : 2 * ACC <= 128 ? 128 : 2 * ACC <= 256 ? 256 : 512;
    static constexpr uint32_t STAGING = CG == 2 || (BN == 64 && NA == 1) ? 8192 : 1024;   // of an epilogue warp; a few rows have no use for it
    static constexpr size_t SMEM = (size_t)STAGE * STAGES + 4 * STAGING + 256 + 1024;
    static_assert(STAGE % 1024 == 0 && 2 * ACC <= TMEM && SMEM <= 232448, "room");
    static_assert(CG == 2 || (size_t)ACC / 4 * kJoinPitch * 16 <= (size_t)STAGE * STAGES, "room to join parts");
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
// 32 columns of a 64-column piece of a 16-bit type, as a TMA store reads it (see stage_swizzled16).
__device__ __forceinline__ void stage_half16(unsigned char *buf, int lane, int half, int dtype, const float (&v)[32])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack_as(dtype, v[8 * j + 2 * i], v[8 * j + 2 * i + 1]);
        *reinterpret_cast<uint4 *>(buf + lane * 128 + (((4 * half + j) ^ (lane & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
    }
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

// The CTAs of a cluster of P add up a tile's entries, four columns of a row a thread at a time, the parts in order, and do what
// the epilogue does with them.  Lanes lie along what is contiguous in the output.
template <int KIND, int BN, int NA, bool GATED, int P>
__device__ __forceinline__ void join_parts(const Params &prm, const float4 *join, int part, int tm, int tn)
{
    constexpr int HN = GATED && NA == 1 ? BN / 2 : BN;
    const int half = tm >= prm.half_tiles, hm = tm - half * prm.half_tiles;
    const int64_t m0 = (int64_t)hm * 128, n0 = (int64_t)tn * HN;
    const int rows = (int)min((int64_t)128, prm.M - m0), cols = (int)min((int64_t)HN, prm.N - n0);
    const int quads = (cols + 3) / 4, inner = prm.swapped ? rows : quads;
    uint32_t from[P];
#pragma unroll
    for (int p = 0; p < P; ++p) from[p] = cluster_address(smem_u32(join), p);
    auto sum = [&](int c4, int r, float (&y)[4]) {
        float4 x[P];
#pragma unroll
        for (int p = 0; p < P; ++p) x[p] = load_cluster(from[p] + (c4 * kJoinPitch + r) * 16);
        if constexpr (KIND == kI8) {
            int s[4] = {0, 0, 0, 0};
#pragma unroll
            for (int p = 0; p < P; ++p) {
                s[0] += __float_as_int(x[p].x); s[1] += __float_as_int(x[p].y);
                s[2] += __float_as_int(x[p].z); s[3] += __float_as_int(x[p].w);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = __int2float_rn(s[e]);
        } else {
#pragma unroll
            for (int p = 1; p < P; ++p) { x[0].x += x[p].x; x[0].y += x[p].y; x[0].z += x[p].z; x[0].w += x[p].w; }
            y[0] = x[0].x; y[1] = x[0].y; y[2] = x[0].z; y[3] = x[0].w;
        }
    };
#pragma unroll 2
    for (int it = part * NTHREADS + threadIdx.x; it < rows * quads; it += P * NTHREADS) {
        const int o = it / inner, i = it - o * inner, c4 = prm.swapped ? o : i, r = prm.swapped ? i : o;
        const int n = cols - c4 * 4;
        const int64_t m = m0 + r, col = n0 + c4 * 4;
        auto scaled = [&](int which, float (&y)[4]) {
            sum(c4 + which * (NA == 1 ? HN : BN) / 4, r, y);
            if constexpr (KIND == kI8) {
                const float sm = prm.scale_m[NA == 2 ? which : 0][m];
                const float *sn = prm.scale_n[GATED && NA == 1 ? which : 0] + col;
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = e < n ? y[e] * sm * sn[e] : 0.0f;
            }
        };
        auto store = [&](int k, const float (&y)[4]) {
            const int64_t ld = prm.ld[k];
            store_four(prm.out[k], prm.dtype, prm.swapped ? m + col * ld : m * ld + col, prm.swapped ? ld : 1, y, n,
                       !prm.swapped && (prm.tma_out >> k & 1));
        };
        if constexpr (GATED) {
            float g[4], u[4], h[4];
            scaled(0, g);
            scaled(1, u);
#pragma unroll
            for (int e = 0; e < 4; ++e) h[e] = activation(prm.act, g[e]) * u[e];
            store(0, h);
            if (prm.out[1]) { store(1, g); store(2, u); }
        } else {
            float y[4];
            scaled(0, y);
            store(half, y);
        }
    }
}

template <int KIND, int CG, int BN, int NA, bool A_MN, bool B_MN, bool GATED>
__global__ void __launch_bounds__(NTHREADS, 1) product_kernel(const __grid_constant__ Params prm)
{
    using S = Shape<CG, BN, NA>;
    constexpr int KS = KIND == kI8 ? 128 : 64;                        // entries of the contraction a stage
    constexpr bool SIDE = GATED && NA == 1;                           // both matrices lie side by side in B
    constexpr int HN = SIDE ? BN / 2 : BN;                            // columns of the output a tile has
    constexpr int UP = NA == 2 ? BN : HN;                             // accumulator columns from the gate to the other projection
    constexpr int BL = BN / CG;                                       // rows of B that this CTA holds
    static_assert(!(KIND == kI8 && (A_MN || B_MN)) && (!B_MN || BL % 64 == 0) && (NA == 1 || (CG == 1 && GATED)), "forms");
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    unsigned char *staging = smem + (size_t)S::STAGE * S::STAGES;
    float4 *join = reinterpret_cast<float4 *>(smem);                  // [ACC / 4][kJoinPitch]: four columns of a row
    uint64_t *bars = reinterpret_cast<uint64_t *>(staging + 4 * S::STAGING);
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
        for (int i = 0; i < 2; ++i) { mbar_init(d_full + i, 1); mbar_init(d_empty + i, 4 * CG); }
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
    grid_dependency_wait();      // what earlier launches wrote is visible from here on
    bool failed = false;

    const int n_tiles = prm.tiles_m * prm.tiles_n;
    const int first = blockIdx.x / (CG * parts), stride = gridDim.x / (CG * parts);
    const int st0 = prm.n_stages * part / parts, st1 = prm.n_stages * (part + 1) / parts;    // this CTA's stages

    if (warp == 0) {
        // ------------------------------------------------------------------ producer
        if (elect_one()) {
            fence_proxy_async_global();      // what plain stores of earlier launches wrote is read by TMA
            uint32_t c = 0, s = 0, phase = 1;
            for (int tile = first; tile < n_tiles && !failed; tile += stride) {
                int tm, tn;
                place(prm, tile, tm, tn);
                const int half = tm >= prm.half_tiles;
                const int m0 = (tm - half * prm.half_tiles) * 128 * CG + 128 * rank;
                const int n0 = SIDE ? tn * HN : tn * BN + BL * rank;
                for (int st = st0; st < st1; ++st, ++c) {
                    if (!mbar_poll(empty + s, phase, abort_flag)) { failed = true; break; }
                    const bool drop = prm.test_drop && blockIdx.x == 0 && c == 0;   // test hook: this stage never arrives
                    if (!drop) {
                        // a contraction of two segments has a map of either operand for each; two halves one of A
                        const int seg = st >= prm.seg_stages;
                        const int k = (st - seg * prm.seg_stages) * KS;
                        unsigned char *dst = smem + s * S::STAGE, *dst_b = dst + NA * A_BYTES;
                        if (rank == 0) mbar_arrive_expect_tx(full + s, CG * S::LOADED);
                        const uint32_t bar = CG == 2 ? in_leader(full + s) : 0;
                        auto load = [&](unsigned char *to, const CUtensorMap *map, bool mn, int at) {
                            if (CG == 2) tma_load_2d_pair(to, map, mn ? at : k, mn ? k : at, bar);
                            else tma_load_2d(to, map, mn ? at : k, mn ? k : at, full + s);
                        };
#pragma unroll
                        for (int i = 0; i < NA; ++i) {
                            const CUtensorMap *map = prm.a + (NA == 2 ? i : half + seg);
                            load(dst + i * A_BYTES, map, A_MN, m0);
                            if (A_MN) load(dst + i * A_BYTES + kBox, map, A_MN, m0 + 64);
                        }
                        if constexpr (SIDE && CG == 2) load(dst_b, prm.b + rank, false, n0);
                        else if constexpr (SIDE) {
                            load(dst_b, prm.b, false, n0);
                            load(dst_b + HN * 128, prm.b + 1, false, n0);
                        } else if constexpr (B_MN) {
#pragma unroll
                            for (int i = 0; i < BL / 64; ++i) load(dst_b + i * kBox, prm.b + seg, true, n0 + 64 * i);
                        } else load(dst_b, prm.b + seg, false, n0);
                    }
                    if (++s == S::STAGES) { s = 0; phase ^= 1; }
                }
            }
            if (failed && rank == 0) {   // give the copies already in flight a bounded chance to land before the CTA exits
                for (uint32_t i = c > S::STAGES ? c - S::STAGES : 0; i < c; ++i)
                    for (int it = 0; it < 100000 && !mbar_try_wait(full + i % S::STAGES, (i / S::STAGES) & 1); ++it) {}
            }
        }
        failed = __any_sync(0xffffffffu, failed);
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer
        if (rank == 0 && elect_one()) {
            uint32_t s = 0, phase = 0, t = 0;
            const uint32_t base = smem_u32(smem);
            const uint64_t a0 = A_MN ? make_mn_desc(base, kBox) : make_b_desc(base);
            const uint64_t b0 = B_MN ? make_mn_desc(base + NA * A_BYTES, kBox) : make_b_desc(base + NA * A_BYTES);
            // 32 bytes of a K-major row, or 16 rows of 128 bytes of an MN-major box
            constexpr uint32_t IA = A_MN ? 16 * 128 / 16 : 2, IB = B_MN ? 16 * 128 / 16 : 2;
            const uint32_t idesc = KIND == kI8 ? idesc_i8(128 * CG, BN)
                                               : make_idesc_f16(128 * CG, BN, A_MN, B_MN) | (prm.bf16 ? (1u << 7) | (1u << 10) : 0u);
            for (int tile = first; tile < n_tiles && !failed; tile += stride, ++t) {
                const uint32_t buf = t & 1, d = tmem + buf * S::ACC;
                if (t > 1) {
                    if (!mbar_poll(d_empty + buf, ((t >> 1) - 1) & 1, abort_flag)) { failed = true; break; }
                    tc_fence_after();
                }
                for (int st = st0; st < st1; ++st) {
                    if (!mbar_poll(full + s, phase, abort_flag)) { failed = true; break; }
                    tc_fence_after();
                    const uint64_t da = a0 + s * (S::STAGE >> 4), db = b0 + s * (S::STAGE >> 4);
                    auto issue = [&](int n_mma) {      // (a constant, except in a short last stage)
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (k < n_mma) {
#pragma unroll
                                for (int i = 0; i < NA; ++i) {
                                    const uint64_t ak = da + i * (A_BYTES >> 4) + k * IA, bk = db + k * IB;
                                    if (KIND == kI8) mma_i8<CG>(d + i * BN, ak, bk, idesc, st > st0 || k > 0);
                                    else tc_mma_f16<CG>(d + i * BN, ak, bk, idesc, st > st0 || k > 0);
                                }
                            }
                    };
                    if (prm.n_last < 4 && (st == prm.n_stages - 1 || st == prm.seg_stages - 1)) issue(prm.n_last); else issue(4);
                    if (CG == 2) tc_commit_pair(empty + s); else tc_commit(empty + s);
                    if (st == st1 - 1) { if (CG == 2) tc_commit_pair(d_full + buf); else tc_commit(d_full + buf); }
                    if (++s == S::STAGES) { s = 0; phase ^= 1; }
                }
            }
        }
        failed = __any_sync(0xffffffffu, failed);
    } else {
        // ------------------------------------------------------------------ epilogue
        const int q = warp & 3;
        const uint32_t lane_base = (uint32_t)(32 * q) << 16;
        unsigned char *mine = staging + (warp - 2) * S::STAGING;
        float *piece_buf = reinterpret_cast<float *>(mine);
        uint32_t t = 0, stores = 0;
        const int dtype = prm.dtype;
        for (int tile = first; tile < n_tiles; tile += stride, ++t) {
            int tm, tn;
            place(prm, tile, tm, tn);
            const int half = tm >= prm.half_tiles;
            const int64_t m0 = (int64_t)(tm - half * prm.half_tiles) * 128 * CG + 128 * rank + 32 * q, n0 = (int64_t)tn * HN;
            const int rows = (int)max((int64_t)0, min((int64_t)32, prm.M - m0));
            // 8-bit operands: the scale of this lane's row, and of every 32nd column from this lane's on (of either matrix)
            constexpr int NS = KIND == kI8 ? (HN + 31) / 32 : 1;
            float sm[NA], sn[SIDE ? 2 : 1][NS];
            if constexpr (KIND == kI8) {
                if (parts == 1) {
#pragma unroll
                    for (int i = 0; i < NA; ++i) sm[i] = lane < rows ? __ldg(prm.scale_m[i] + m0 + lane) : 0.0f;
#pragma unroll
                    for (int i = 0; i < (SIDE ? 2 : 1); ++i)
#pragma unroll
                        for (int j = 0; j < NS; ++j)
                            sn[i][j] = n0 + 32 * j + lane < prm.N ? __ldg(prm.scale_n[i] + n0 + 32 * j + lane) : 0.0f;
                }
            }
            const uint32_t buf = t & 1;
            bool ok = mbar_poll(d_full + buf, (t >> 1) & 1, abort_flag);
            if (!__all_sync(0xffffffffu, ok)) { failed = true; break; }
            tc_fence_after();
            const uint32_t acc = tmem + lane_base + buf * S::ACC;
            if (parts > 1) {           // the stages have been read: what the part has goes into their place
                if constexpr (CG == 1) {
#pragma unroll 1
                    for (int c = 0; c < (int)S::ACC; c += 16) {
                        float v[16];
                        tmem_ld16_wait(acc + c, v);
#pragma unroll
                        for (int i = 0; i < 16; i += 4)
                            join[(c + i) / 4 * kJoinPitch + 32 * q + lane] = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                    }
                }
                continue;
            }
            // 32 columns of one matrix's sums; `j`: c / 32, a constant where it indexes registers
            auto sums = [&](int which, int c, int j, float (&v)[32]) {
                if constexpr (BN >= 32) tmem_ld32_wait(acc + (GATED ? which * UP : 0) + c, v);
                else {
                    float w[16];
                    tmem_ld16_wait(acc + (GATED ? which * UP : 0), w);
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = i < 16 ? w[i] : 0.0f;
                }
                if constexpr (KIND == kI8) {
                    float mine_n = 0.0f;
#pragma unroll
                    for (int x = 0; x < NS; ++x)
                        if (x == j) mine_n = sn[SIDE ? which : 0][x];
                    const float mine_m = sm[NA == 2 ? which : 0];
#pragma unroll
                    for (int i = 0; i < (BN >= 32 ? 32 : 16); ++i)
                        v[i] = __int2float_rn(__float_as_int(v[i])) * mine_m * __shfl_sync(0xffffffffu, mine_n, i);
                }
            };
            // output `o` (0: the product, or the block's; 1, 2: its projections)
            auto values = [&](int o, int c, int j, float (&v)[32]) {
                if constexpr (GATED) {
                    if (o > 0) { sums(o - 1, c, j, v); return; }
                    float u[32];
                    sums(0, c, j, v);
                    sums(1, c, j, u);
                    activate(prm.act, v, u);
                } else sums(0, c, j, v);
            };
            const int n_out = GATED && prm.out[1] ? 3 : 1;
            constexpr int PW = HN < 64 ? HN : 64;                      // columns of a piece
            constexpr int NP = HN / PW;
#pragma unroll 1
            for (int oi = 0; oi < n_out; ++oi) {
                const int o = n_out - 1 - oi;                          // (the block's output last)
                const int slot = GATED ? o : half;
                void *out = prm.out[slot];
                const int64_t ld = prm.ld[slot];
                const bool tma = prm.tma_out >> slot & 1;
#pragma unroll 1
                for (int p = 0; p < NP; ++p) {
                    const int64_t n = n0 + p * PW;
                    const bool wanted = rows > 0 && n < prm.N;
                    // (a tiled store writes whole 16-byte chunks: past the last column where that does not end at one)
                    const bool by_tma = PW == 64 && tma && (n + 64 <= prm.N || prm.N * (dtype == GVQ_F32 ? 4 : 2) % 16 == 0);
                    unsigned char *to = dtype != GVQ_F32 && by_tma ? mine + (stores & 1) * 4096 : mine;
#pragma unroll
                    for (int h = 0; h < (PW + 31) / 32; ++h) {
                        float v[32];
                        values(o, p * PW + 32 * h, p * (PW / 32) + h, v);
                        if (oi == n_out - 1 && p == NP - 1 && h == (PW + 31) / 32 - 1) {
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) { if (CG == 2) mbar_arrive_cluster(in_leader(d_empty + buf)); else mbar_arrive(d_empty + buf); }
                        }
                        const int cols = (int)min((int64_t)min(PW, 32), prm.N - n - 32 * h);
                        if (!wanted || cols <= 0) continue;
                        if (by_tma) {
                            // rows of 128 bytes, swizzled, stored by the copy engine: what the pieces cost in shared-memory
                            // bandwidth is taken from the MMAs, so they pass through it in the output's type and once
                            if (h == 0) {
                                if (lane == 0) { if (dtype != GVQ_F32) bulk_wait_group_read<1>(); else bulk_wait_group_read<0>(); }
                                __syncwarp();
                            }
                            if (dtype == GVQ_F32) stage_swizzled(to + 4096 * h, lane, v);
                            else stage_half16(to, lane, h, dtype, v);
                        } else if (prm.swapped) {       // rows of A run along the output's rows: a warp's lanes do too
                            if (lane < rows) {
#pragma unroll
                                for (int i = 0; i < 32; ++i)
                                    if (i < cols) store_one(out, dtype, m0 + lane + (n + 32 * h + i) * ld, v[i]);
                            }
                        } else {
                            if (lane == 0) bulk_wait_group_read<0>();      // the staging area may still be on its way out
                            __syncwarp();
                            if constexpr (S::STAGING >= 32 * kPiecePitch * 4) {
                                stage_piece(piece_buf, lane, v);
                                const int64_t at = m0 * ld + n + 32 * h;
                                if (dtype == GVQ_F32) store_piece(piece_buf, lane, static_cast<float *>(out) + at, ld, rows, cols);
                                else if (dtype == GVQ_BF16) store_piece(piece_buf, lane, static_cast<__nv_bfloat16 *>(out) + at, ld, rows, cols);
                                else store_piece(piece_buf, lane, static_cast<__half *>(out) + at, ld, rows, cols);
                            }
                        }
                    }
                    if (by_tma && wanted) {
                        fence_proxy_async();
                        __syncwarp();
                        if (lane == 0) {
                            tma_store_2d(prm.o + slot, (int)n, (int)m0, to);
                            if (dtype == GVQ_F32 && n + 32 < prm.N) tma_store_2d(prm.o + slot, (int)n + 32, (int)m0, to + 4096);
                            bulk_commit_group();
                        }
                        ++stores;
                    }
                }
            }
        }
        if (lane == 0) bulk_wait_group_all();
    }

    if constexpr (CG == 1) {
        if (parts > 1) {
            __syncwarp();
            cluster_sync();
            if (!failed) {
                int tm, tn;
                place(prm, first, tm, tn);
                if (parts == 2) join_parts<KIND, BN, NA, GATED, 2>(prm, join, part, tm, tn);
                else if (parts == 4) join_parts<KIND, BN, NA, GATED, 4>(prm, join, part, tm, tn);
                else join_parts<KIND, BN, NA, GATED, 8>(prm, join, part, tm, tn);
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
    if (warp == 1) tmem_dealloc<CG>(tmem, S::TMEM);
}

// ---------------------------------------------------------------------------------------------------- host side
inline int tiles_of(int64_t n, int per) { return (int)((n + per - 1) / per); }

// How a product M x N (rows of tokens x outputs) is cut up.
struct Cut {
    bool swapped;      // the rows of tokens are B
    int cg, bn;
};

template <int KIND, int CG, int BN, int NA, bool A_MN, bool B_MN, bool GATED>
cudaError_t launch(cudaStream_t st, int num_sms, const Params &prm)
{
    using S = Shape<CG, BN, NA>;
    const int cluster = CG * prm.parts;
    const int64_t tiles = (int64_t)prm.tiles_m * prm.tiles_n;
    return launch_chained<product_kernel<KIND, CG, BN, NA, A_MN, B_MN, GATED>>(
        prm, cluster * (int)(tiles < num_sms / cluster ? tiles : num_sms / cluster), NTHREADS, S::SMEM, cluster, st);
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

// Output `slot` [M][N], rows ld entries apart: by TMA where its rows start at 16-byte boundaries.
inline void set_output(EncodeTiledFn enc, Params &prm, int slot, void *out, int dtype, int64_t M, int64_t N, int64_t ld)
{
    prm.out[slot] = out;
    prm.ld[slot] = ld;
    const size_t size = dtype == GVQ_F32 ? 4 : 2;
    if (prm.swapped || !out || (reinterpret_cast<uintptr_t>(out) & 15u) != 0 || (M > 1 && ld * size % 16 != 0)) return;
    cuuint64_t dims[2] = {(cuuint64_t)N, (cuuint64_t)M};
    cuuint64_t strides[1] = {(cuuint64_t)((M > 1 ? ld : (N * size + 15) / 16 * 16 / size) * size)};
    cuuint32_t box[2] = {(cuuint32_t)(128 / size), 32}, estr[2] = {1, 1};
    const CUtensorMapDataType type = dtype == GVQ_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                     : dtype == GVQ_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    if (enc(&prm.o[slot], type, 2, out, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS)
        prm.tma_out |= 1 << slot;      // (strides of 2^40 bytes and more are not taken)
}

// Few rows of tokens: the weights take the 128-row side of the tile, and the tile is as wide as the few rows need.  Otherwise
// pairs of CTAs on 256 x 256 tiles where smaller ones would need a second wave.  `n_small`: columns of the output a 64-column
// tile has.
inline Cut cut(int num_sms, int64_t M, int64_t N, int n_small)
{
    const bool waves = (int64_t)tiles_of(M, 128) * tiles_of(N, n_small) > num_sms;
    Cut c;
    c.swapped = M <= 32 || (M <= 64 && waves);
    c.cg = !c.swapped && waves ? 2 : 1;
    c.bn = c.cg == 2 ? 256 : !c.swapped ? 64 : M <= 16 ? 16 : M <= 32 ? 32 : 64;
    return c;
}

// Fills in how the product is gone through.  out_n: columns of the output a tile has; K: of a segment of the contraction.
inline void divide(Params &prm, int num_sms, const Cut &c, int kind, int out_n, int64_t K, int segments, int halves)
{
    const int ks = kind == kI8 ? 128 : 64;
    prm.half_tiles = tiles_of(prm.M, 128 * c.cg);
    prm.tiles_m = prm.half_tiles * halves;
    if (halves == 1) prm.half_tiles = prm.tiles_m;
    prm.tiles_n = tiles_of(prm.N, out_n);
    prm.seg_stages = tiles_of(K, ks);
    prm.n_stages = prm.seg_stages * segments;
    prm.n_last = (int)((K - (int64_t)(prm.seg_stages - 1) * ks + ks / 4 - 1) / (ks / 4));
    prm.group = prm.tiles_m < 8 ? prm.tiles_m : 8;
    prm.swapped = c.swapped;
    // Parts of a contraction: as many as there are SMs for, of a few stages each.
    const int min_stages = c.bn <= 32 ? 2 : 8;
    prm.parts = 1;
    while (c.cg == 1 && prm.parts < 8 && (int64_t)prm.tiles_m * prm.tiles_n * 2 * prm.parts <= (prm.parts < 4 ? num_sms : num_sms * 2 / 3) &&
           prm.n_stages >= 2 * prm.parts * min_stages)
        prm.parts *= 2;
}

}  // namespace product
}  // namespace gvq
