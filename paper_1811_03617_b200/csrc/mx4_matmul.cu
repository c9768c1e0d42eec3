// Product of two matrices in microscaled 4-bit floating point,  D[m][n] = sum_k A[m][k] B[n][k],  on the
// block-scaled tcgen05 tensor path (gvq.h, "microscaled 4-bit").
//
// Both operands are quantized along the contraction, so both are K-major: a row of codes is contiguous.  The tensor
// core multiplies codes and applies the two blocks' scales itself, 64 entries of the contraction an instruction, and
// accumulates in fp32.
//
// Tiles are CG * 128 rows of A x BN rows of B, 256 entries of the contraction a stage (128 bytes of codes a row).
//   CG = 2, BN = 256   a pair of CTAs on two SMs: each holds its own 128 rows of A and half of B's rows; the even one issues
//                      MMAs that read both.  35 KB a stage and SM for 512 clocks of MMAs, where a CTA alone on 128 x 256 would
//                      load 51 KB -- more than L2 delivers to all SMs at that rate.
//   CG = 1             one CTA, 128 x 64 or narrower: few rows (of a token, a small batch: they become B, the tile as narrow
//                      as they are), or products too small to give every SM a large tile.  Where the tiles are fewer than
//                      the SMs, a cluster of up to eight CTAs shares a tile's contraction; each leaves its sums in its shared
//                      memory, where the stages were, and they add them up across the cluster, always in the same order.
//   warp 0      producer: per stage TMA loads of both operands' codes (128-byte swizzle, zero fill outside) and scale bytes
//               (two tiles of 512 bytes, contiguous, for each 128 rows; read as rows of 8-byte words)
//   warp 1      MMA: copies the stage's scale tiles into tensor memory (each 128 x 4 tile becomes 4 columns), then up
//               to four MMAs; one elected lane issues, the order of issue is the order of execution
//   warps 2-5   epilogue: accumulator -> registers -> staging -> output along its rows
// Accumulators alternate between two column ranges.  Every mbarrier wait is bounded.
//
// Measured on the GPU: 8192 x 16384 x 4096 to bf16 202 us (5.4 PFLOP/s, 82 % of four times the measured bf16 rate, under the
// power cap), 4096 x 4096 x 8192 50 us (5.4); what a large product waits for is the loads of its operands from L2 (without the
// MMAs 8192 x 8192 x 8192 takes 162 of its 182 us).  Few rows are bound by a stage's fixed cost in the two issuing lanes, 0.22 us:
// 16 x 4096 x 16384 16.3 us with a CTA a tile, 7.6 us (4.4 TB/s of codes from L2) with four.
#include "gvq_internal.h"
#include "mx4.cuh"
#include "row32.cuh"
#include "sm100_ptx.cuh"

namespace gvq {
namespace {

using namespace ptx;
using mx4::kTileBytes;

constexpr int KS = 256;               // entries of the contraction a stage
constexpr int NTHREADS = 192;
constexpr int kJoinPitch = 129;        // (a row's words of 16 bytes, eight lanes' of them, lie in different banks)
constexpr uint32_t A_BYTES = 128 * 128, SFA_BYTES = 2 * kTileBytes;

template <int CG, int BN> struct Shape {
    static constexpr int NRT = (BN + 127) / 128;                       // scale tiles of B side by side
    static constexpr uint32_t B_BYTES = BN / CG * 128, SFB_BYTES = NRT * 2 * kTileBytes;
    static constexpr uint32_t LOADED = A_BYTES + B_BYTES + SFA_BYTES + SFB_BYTES;
    static constexpr uint32_t STAGE = (LOADED + 1023) / 1024 * 1024;
    static constexpr int STAGES = CG == 2 ? 5 : 6;
    // tensor memory: two accumulators (256 columns each do not fit beside the scales: they overlap by 48 columns,
    // which the epilogue reads first), then two sets of scale columns
    static constexpr uint32_t ACC1 = BN == 256 ? 208 : BN;
    static constexpr uint32_t SF0 = ACC1 + BN, SF_SET = 8 + 8 * NRT;
    static constexpr uint32_t TMEM = SF0 + 2 * SF_SET <= 128 ? 128 : SF0 + 2 * SF_SET <= 256 ? 256 : 512;
    static constexpr uint32_t STAGING = 8192;                          // of an epilogue warp: two pieces of 4 KB
    static constexpr size_t SMEM = (size_t)STAGE * STAGES + 4 * STAGING + 256 + 1024;
    static_assert(SF0 + 2 * SF_SET <= TMEM, "tensor memory");
    static_assert(CG == 2 || (size_t)BN / 4 * kJoinPitch * 16 <= (size_t)STAGE * STAGES, "room to join parts");
};

struct MmParams {
    CUtensorMap a, b;                 // codes: bytes x rows
    CUtensorMap sa, sb;               // scale bytes: 8-byte words x tiles of 128 rows
    CUtensorMap o;                    // the output, boxes of 128 bytes x 32 rows (tma_out)
    int tma_out;
    int64_t M, N, K;                  // rows of A, rows of B, contraction
    int tiles_m, tiles_n, n_stages;   // n_stages: of one tile's contraction
    int parts;                        // CTAs (a cluster) that share a tile's contraction; with more than one, a tile a cluster
    void *out;
    int64_t out_m, out_n;             // strides of the output in entries, one of them 1
    int32_t *error_word;
    int wait_kcycles, test_drop;
};

// 128 x 4 scale bytes (32 rows of 16 bytes) -> 4 columns of tensor memory, the same in all four lane quarters (for a
// pair: in both CTAs, each from its own shared memory)
template <int CG>
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint64_t desc)
{
    if (CG == 2) asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
    else asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
__device__ __forceinline__ uint64_t scales_desc(uint32_t smem_addr)
{
    return (uint64_t)((smem_addr & 0x3FFFFu) >> 4) | ((uint64_t)(128 >> 4) << 16) | ((uint64_t)(128 >> 4) << 32) | ((uint64_t)1 << 46);
}
template <int CG>
__device__ __forceinline__ void mma_mxf4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                         uint32_t accumulate)
{
    if (CG == 2)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
                     "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
}
// E2M1 x E2M1, power-of-two scales; `half`: which pair of a scale column's four bytes (of A and of B)
__host__ __device__ constexpr uint32_t idesc_mxf4(int m, int n, int half)
{
    return ((uint32_t)(2 * half) << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | (1u << 23) |
           ((uint32_t)(m >> 4) << 24) | ((uint32_t)(2 * half) << 29);
}

// The CTAs of a cluster of P add up the tile's entries that there are, four columns of a row a thread at a time, the parts in
// order.  Lanes lie along what is contiguous in the output: the columns, or with B's rows on this side the rows.
template <typename T, int BN, int P>
__device__ __forceinline__ void join_parts(const MmParams &prm, const float4 *join, int part, int tm, int tn)
{
    const bool by_row = prm.out_n == 1;
    const int rows = (int)min((int64_t)128, prm.M - (int64_t)tm * 128), cols = (int)min((int64_t)BN, prm.N - (int64_t)tn * BN);
    const int quads = (cols + 3) / 4, inner = by_row ? quads : rows;
    uint32_t from[P];
#pragma unroll
    for (int p = 0; p < P; ++p) from[p] = cluster_address(smem_u32(join), p);
#pragma unroll 2
    for (int it = part * NTHREADS + threadIdx.x; it < rows * quads; it += P * NTHREADS) {
        const int o = it / inner, i = it - o * inner, c4 = by_row ? i : o, r = by_row ? o : i;
        float4 x[P];
#pragma unroll
        for (int p = 0; p < P; ++p) x[p] = load_cluster(from[p] + (c4 * kJoinPitch + r) * 16);
#pragma unroll
        for (int p = 1; p < P; ++p) { x[0].x += x[p].x; x[0].y += x[p].y; x[0].z += x[p].z; x[0].w += x[p].w; }
        const T y[4] = {from_f<T>(x[0].x), from_f<T>(x[0].y), from_f<T>(x[0].z), from_f<T>(x[0].w)};
        T *out = static_cast<T *>(prm.out) + ((int64_t)tm * 128 + r) * prm.out_m + ((int64_t)tn * BN + c4 * 4) * prm.out_n;
        if (by_row && prm.tma_out && c4 * 4 + 4 <= cols) {      // (rows at 16-byte boundaries)
            if (sizeof(T) == 2) { uint2 w; memcpy(&w, y, sizeof(w)); *reinterpret_cast<uint2 *>(out) = w; }
            else { uint4 w; memcpy(&w, y, sizeof(T) == 4 ? 16 : 8); *reinterpret_cast<uint4 *>(out) = w; }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (c4 * 4 + e < cols) out[e * prm.out_n] = y[e];
        }
    }
}

template <typename T, int CG, int BN>
__global__ void __launch_bounds__(NTHREADS, 1) mx4_matmul_kernel(const __grid_constant__ MmParams prm)
{
    using S = Shape<CG, BN>;
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    unsigned char *staging = smem + (size_t)S::STAGE * S::STAGES;
    float4 *join = reinterpret_cast<float4 *>(smem);       // [BN / 4][kJoinPitch]: four columns of a row
    uint64_t *bars = reinterpret_cast<uint64_t *>(staging + 4 * S::STAGING);
    uint64_t *full = bars, *empty = full + S::STAGES;      // [STAGES]
    uint64_t *d_full = empty + S::STAGES;                  // [2] accumulator complete
    uint64_t *d_early = d_full + 2;                        // [2] the columns it shares with the other one are read
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(d_early + 2);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = CG == 2 ? (int)cluster_rank() : 0;
    const int parts = CG == 1 ? prm.parts : 1, part = parts > 1 ? (int)cluster_rank() : 0;
    if (threadIdx.x == 0) {
        for (int i = 0; i < S::STAGES; ++i) { mbar_init(full + i, 1); mbar_init(empty + i, 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(d_full + i, 1); mbar_init(d_early + i, 4 * CG); }
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
    grid_dependency_wait();      // what the quantizing launches wrote is visible from here on
    bool failed = false;

    const int n_tiles = prm.tiles_m * prm.tiles_n;
    const int first = blockIdx.x / (CG * parts), stride = gridDim.x / (CG * parts);
    const int st0 = prm.n_stages * part / parts, st1 = prm.n_stages * (part + 1) / parts;    // this CTA's stages
    const int n_last = (int)((prm.K - (int64_t)(prm.n_stages - 1) * KS + 63) / 64);   // MMAs of a tile's last stage, 1 .. 4

    if (warp == 0) {
        // ------------------------------------------------------------------ producer
        if (elect_one()) {
            fence_proxy_async_global();      // what plain stores of the previous launch wrote is read by TMA
            uint32_t c = 0, s = 0, phase = 1;
            for (int tile = first; tile < n_tiles && !failed; tile += stride) {
                const int tn = tile / prm.tiles_m, tm = tile - tn * prm.tiles_m;
                const int m0 = tm * 128 * CG + 128 * rank, n0 = tn * BN + BN / CG * rank;
                const int m_tile = m0 >> 7, n_tile = (tn * BN) >> 7;
                for (int st = st0; st < st1; ++st, ++c) {
                    if (!mbar_poll(empty + s, phase, abort_flag)) { failed = true; break; }
                    const bool drop = prm.test_drop && blockIdx.x == 0 && c == 0;   // test hook: this stage never arrives
                    if (!drop) {
                        unsigned char *dst = smem + s * S::STAGE;
                        if (rank == 0) mbar_arrive_expect_tx(full + s, CG * S::LOADED);
                        const uint32_t bar = CG == 2 ? in_leader(full + s) : 0;
                        auto load = [&](unsigned char *to, const CUtensorMap *map, int x, int y) {
                            if (CG == 2) tma_load_2d_pair(to, map, x, y, bar); else tma_load_2d(to, map, x, y, full + s);
                        };
                        load(dst, &prm.a, st * 128, m0);
                        load(dst + A_BYTES, &prm.b, st * 128, n0);
                        // this CTA's rows of A; all of the tile's rows of B, which both CTAs of a pair need
                        load(dst + A_BYTES + S::B_BYTES, &prm.sa, st * 128, m_tile);
                        load(dst + A_BYTES + S::B_BYTES + SFA_BYTES, &prm.sb, st * 128, n_tile);
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
        // One lane goes through the whole loop: electing it and bringing the warp together again for every stage took 180 of
        // a stage's 470 clocks, and that bounded narrow products.
        if (rank == 0 && elect_one()) {
            uint32_t s = 0, phase = 0, set = 0, t = 0;
            const uint32_t base0 = smem_u32(smem);
            const uint64_t a0 = make_b_desc(base0), sc0 = scales_desc(base0 + A_BYTES + S::B_BYTES);
            for (int tile = first; tile < n_tiles && !failed; tile += stride, ++t) {
                const uint32_t buf = t & 1;
                const uint32_t d = tmem + buf * S::ACC1;
                // a narrow tile's rows of B may begin inside their scale tile: 32 rows a column
                const uint32_t sf_shift = BN < 128 ? ((uint32_t)(tile / prm.tiles_m) * BN & 127u) >> 5 : 0;
                if (t > 0) {
                    // the tile before this one has been read where the two accumulators overlap (and the one before
                    // that, in this accumulator, entirely: the epilogue takes the tiles in order)
                    if (!mbar_poll(d_early + (buf ^ 1), ((t - 1) >> 1) & 1, abort_flag)) { failed = true; break; }
                    tc_fence_after();
                }
                for (int st = st0; st < st1; ++st) {
                    if (!mbar_poll(full + s, phase, abort_flag)) { failed = true; break; }
                    tc_fence_after();
                    const bool last = st == st1 - 1;
                    const uint32_t sfa = tmem + S::SF0 + set, sfb = sfa + 8;
                    const uint64_t da = a0 + s * (S::STAGE >> 4), db = da + (A_BYTES >> 4), sc = sc0 + s * (S::STAGE >> 4);
                    auto issue = [&](int n_mma) {      // (a constant, except in a short last stage)
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            if (2 * k < n_mma) {
                                copy_scales<CG>(sfa + 4 * k, sc + k * (kTileBytes >> 4));
#pragma unroll
                                for (int r = 0; r < S::NRT; ++r)
                                    copy_scales<CG>(sfb + 4 * (k * S::NRT + r), sc + ((SFA_BYTES * (1 + r) + k * kTileBytes) >> 4));
                            }
                        }
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (k < n_mma)
                                mma_mxf4<CG>(d, da + k * 2, db + k * 2, idesc_mxf4(128 * CG, BN, k & 1), sfa + 4 * (k >> 1),
                                             sfb + 4 * S::NRT * (k >> 1) + sf_shift, st > st0 || k > 0);
                    };
                    if (st == prm.n_stages - 1 && n_last < 4) issue(n_last); else issue(4);
                    if (CG == 2) tc_commit_pair(empty + s); else tc_commit(empty + s);
                    if (last) { if (CG == 2) tc_commit_pair(d_full + buf); else tc_commit(d_full + buf); }
                    set ^= S::SF_SET;
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
        T *out = static_cast<T *>(prm.out);
        uint32_t t = 0, stores = 0;
        for (int tile = first; tile < n_tiles; tile += stride, ++t) {
            const int tn = tile / prm.tiles_m, tm = tile - tn * prm.tiles_m;
            const uint32_t buf = t & 1;
            bool ok = mbar_poll(d_full + buf, (t >> 1) & 1, abort_flag);
            if (!__all_sync(0xffffffffu, ok)) { failed = true; break; }
            tc_fence_after();
            const uint32_t acc = tmem + lane_base + buf * S::ACC1;
            if (parts > 1) {           // the stages have been read: what the part has goes into their place
                if constexpr (CG == 1) {
#pragma unroll
                    for (int c = 0; c < BN; c += 16) {
                        float v[16];
                        tmem_ld16_wait(acc + c, v);
#pragma unroll
                        for (int i = 0; i < 16; i += 4)
                            join[(c + i) / 4 * kJoinPitch + 32 * q + lane] = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                    }
                }
                continue;
            }
            const int64_t m0 = (int64_t)tm * 128 * CG + 128 * rank + 32 * q;
            const int rows = (int)max((int64_t)0, min((int64_t)32, prm.M - m0));
            // pieces of 64 columns; the first accumulator's last columns are the second one's first: that piece comes first
            constexpr int NP = BN > 64 ? BN / 64 : 1;
            constexpr bool SHARED = BN == 256;
#pragma unroll 1
            for (int p = 0; p < NP; ++p) {
                const int piece = buf == 0 && SHARED ? (p + NP - 1) % NP : p;
                float v[2][32];
                if (BN >= 32) {
                    tmem_ld32_wait(acc + piece * 64, v[0]);
                    if (BN >= 64) tmem_ld32_wait(acc + piece * 64 + 32, v[1]);
                } else {
                    float w[16];
                    tmem_ld16_wait(acc, w);
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[0][i] = i < 16 ? w[i] : 0.0f;
                }
                if (p == (SHARED ? 0 : NP - 1)) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) { if (CG == 2) mbar_arrive_cluster(in_leader(d_early + buf)); else mbar_arrive(d_early + buf); }
                }
                const int64_t n = (int64_t)tn * BN + piece * 64;
                if (rows <= 0 || n >= prm.N) continue;
                // (a tiled store writes whole 16-byte chunks: past the last column where that does not end at one)
                if (BN >= 64 && prm.tma_out && (n + 64 <= prm.N || prm.N * (int)sizeof(T) % 16 == 0)) {
                    // rows of 128 bytes, swizzled, stored by the copy engine: what the pieces cost in shared-memory bandwidth
                    // is taken from the MMAs, so they pass through it in the output's type and once
                    unsigned char *to = sizeof(T) == 2 ? mine + (stores & 1) * 4096 : mine;
                    if (lane == 0) { if (sizeof(T) == 2) bulk_wait_group_read<1>(); else bulk_wait_group_read<0>(); }
                    __syncwarp();
                    if constexpr (sizeof(T) == 2) {
                        stage_swizzled16<T>(to, lane, v[0], v[1]);
                    } else {
                        stage_swizzled(to, lane, v[0]);
                        stage_swizzled(to + 4096, lane, v[1]);
                    }
                    fence_proxy_async();
                    __syncwarp();
                    if (lane == 0) {
                        tma_store_2d(&prm.o, (int)n, (int)m0, to);
                        if (sizeof(T) == 4 && n + 32 < prm.N) tma_store_2d(&prm.o, (int)n + 32, (int)m0, to + 4096);
                        bulk_commit_group();
                    }
                    ++stores;
                } else {
                    if (BN >= 64 && lane == 0) bulk_wait_group_read<0>();      // the staging area may still be on its way out
                    __syncwarp();
#pragma unroll
                    for (int h = 0; h < (BN >= 64 ? 2 : 1); ++h) {
                        const int cols = (int)min((int64_t)min(BN, 32), prm.N - n - 32 * h);
                        if (cols <= 0) break;
                        if (prm.out_n == 1) {
                            stage_piece(piece_buf, lane, v[h]);
                            store_piece(piece_buf, lane, out + m0 * prm.out_m + n + 32 * h, prm.out_m, rows, cols);
                        } else if (lane < rows) {      // rows of A run along the output's rows: a warp's lanes do too
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                if (i < cols) out[m0 + lane + (n + 32 * h + i) * prm.out_n] = from_f<T>(v[h][i]);
                        }
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
                const int tn = first / prm.tiles_m, tm = first - tn * prm.tiles_m;
                if (parts == 2) join_parts<T, BN, 2>(prm, join, part, tm, tn);
                else if (parts == 4) join_parts<T, BN, 4>(prm, join, part, tm, tn);
                else join_parts<T, BN, 8>(prm, join, part, tm, tn);
            }
        }
    }
    if (failed) {
        *abort_flag = 1;
        if (lane == 0) atomicExch(prm.error_word, 100 + warp);
    }
    tc_fence_before();
    __syncwarp();
    // (the other CTAs of a cluster use this one's barriers and memory until here)
    if (CG == 2 || parts > 1) cluster_sync(); else __syncthreads();
    tc_fence_after();
    if (warp == 1) tmem_dealloc<CG>(tmem, S::TMEM);
}

template <typename T, int CG, int BN>
cudaError_t launch_as(cudaStream_t st, int num_sms, const MmParams &prm)
{
    using S = Shape<CG, BN>;
    const int cluster = CG * prm.parts;
    return launch_chained<mx4_matmul_kernel<T, CG, BN>>(prm, cluster * min(num_sms / cluster, prm.tiles_m * prm.tiles_n), NTHREADS, S::SMEM,
                                                        cluster, st);
}
template <int CG, int BN>
cudaError_t launch_typed(cudaStream_t st, int num_sms, int dtype, const MmParams &prm)
{
    if (dtype == GVQ_F32) return launch_as<float, CG, BN>(st, num_sms, prm);
    if (dtype == GVQ_BF16) return launch_as<__nv_bfloat16, CG, BN>(st, num_sms, prm);
    return launch_as<__half, CG, BN>(st, num_sms, prm);
}

bool encode(EncodeTiledFn enc, CUtensorMap *map, const uint8_t *codes, int64_t rows, int64_t cols, int box_rows)
{
    const cuuint64_t pitch = (cuuint64_t)(16 * mx4::blocks(cols));
    cuuint64_t dims[2] = {pitch, (cuuint64_t)rows};
    cuuint64_t strides[1] = {pitch};
    cuuint32_t box[2] = {128, (cuuint32_t)box_rows};
    cuuint32_t estr[2] = {1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t *>(codes), dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Scale bytes of `rows` rows: tiles of 128 rows, each kt * 512 contiguous bytes; a box is a stage's two tiles of `tiles` rows.
bool encode_scales(EncodeTiledFn enc, CUtensorMap *map, const uint8_t *scales, int64_t rows, int64_t kt, int tiles)
{
    cuuint64_t dims[2] = {(cuuint64_t)(kt * kTileBytes / 8), (cuuint64_t)mx4::tiles_of(rows, 128)};
    cuuint64_t strides[1] = {(cuuint64_t)(kt * kTileBytes)};
    cuuint32_t box[2] = {2 * kTileBytes / 8, (cuuint32_t)tiles};
    cuuint32_t estr[2] = {1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_INT64, 2, const_cast<uint8_t *>(scales), dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

cudaError_t launch_mx4_matmul(cudaStream_t st, int num_sms, EncodeTiledFn enc, const uint8_t *a, const uint8_t *sa, const uint8_t *b,
                              const uint8_t *sb, int64_t M, int64_t N, int64_t K, void *out, int dtype, int64_t ld,
                              int32_t *error_word, int wait_kcycles, int test_drop)
{
    MmParams prm;
    // Few rows of A: B takes the 128-row side of the tile, and the tile is as wide as the few rows need.  Up to 32 rows that
    // is never slower than 128 x 64 tiles by more than 0.3 us and up to twice as fast (16 x 8192 x 8192 9.8 us against 17.2:
    // the copies of mostly empty tiles of A are slow); 64 rows cost the epilogue 1.5 us of short stores, which pays where
    // 128 x 64 tiles would need a second wave (64 x 16384 x 8192 12.0 us against 15.0, 64 x 8192 x 8192 11.5 against 9.9).
    // Otherwise pairs of CTAs on 256 x 256 tiles where smaller ones would need a second wave (1280 x 1024 x 4096 9.1 us
    // against 13.1 with them), and smaller ones where they do not (1024 x 1024 x 4096 6.5 us against 9.5 in pairs).
    const bool waves = mx4::tiles_of(M, 128) * mx4::tiles_of(N, 64) > num_sms;
    const bool swap = M <= 32 || (M <= 64 && waves), pair = !swap && waves;
    const int BN = pair ? 256 : !swap ? 64 : M <= 16 ? 16 : M <= 32 ? 32 : 64;
    prm.M = swap ? N : M; prm.N = swap ? M : N; prm.K = K;
    prm.tiles_m = (int)mx4::tiles_of(prm.M, pair ? 256 : 128);
    prm.tiles_n = (int)mx4::tiles_of(prm.N, BN);
    prm.n_stages = (int)mx4::tiles_of(K, KS);
    // Parts of a contraction: as many as there are SMs for (eight CTAs of a cluster find room less easily than four), and at
    // least 2 stages each of a narrow tile (1 x 2048 x 2048 4.6 -> 3.7 us with 4, 16 x 4096 x 16384 17.1 -> 7.6), 8 of a tile
    // of 64 columns, whose sums cost 2 us to add up (64 x 2048 x 8192 9.9 -> 6.8 us with 4; 64 x 4096 x 2048 4.6 -> 5.9 with 2).
    const int min_stages = BN <= 32 ? 2 : 8;
    prm.parts = 1;
    while (!pair && prm.parts < 8 && (int64_t)prm.tiles_m * prm.tiles_n * 2 * prm.parts <= (prm.parts < 4 ? num_sms : num_sms * 2 / 3) &&
           prm.n_stages >= 2 * prm.parts * min_stages)
        prm.parts *= 2;
    prm.out = out;
    prm.out_m = swap ? 1 : ld; prm.out_n = swap ? ld : 1;
    prm.error_word = error_word;
    prm.wait_kcycles = wait_kcycles > 0 ? wait_kcycles : WAIT_KCYCLES_DEFAULT;
    prm.test_drop = test_drop;
    const int64_t kt = mx4::tiles_of(mx4::blocks(K), mx4::kTileBlocks);
    if (!encode(enc, &prm.a, swap ? b : a, prm.M, K, 128) || !encode(enc, &prm.b, swap ? a : b, prm.N, K, pair ? 128 : BN) ||
        !encode_scales(enc, &prm.sa, swap ? sb : sa, prm.M, kt, 1) || !encode_scales(enc, &prm.sb, swap ? sa : sb, prm.N, kt, pair ? 2 : 1))
        return cudaErrorInvalidValue;
    const size_t size = dtype == GVQ_F32 ? 4 : 2;
    prm.tma_out = !swap && (reinterpret_cast<uintptr_t>(out) & 15u) == 0 && (M == 1 || ld * size % 16 == 0);
    if (prm.tma_out) {
        cuuint64_t dims[2] = {(cuuint64_t)N, (cuuint64_t)M};
        cuuint64_t strides[1] = {(cuuint64_t)(ld * size)};
        cuuint32_t box[2] = {(cuuint32_t)(128 / size), 32}, estr[2] = {1, 1};
        const CUtensorMapDataType type = dtype == GVQ_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                         : dtype == GVQ_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
        if (enc(&prm.o, type, 2, out, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            prm.tma_out = 0;    // (strides of 2^40 bytes and more)
    }
    if (pair) return launch_typed<2, 256>(st, num_sms, dtype, prm);
    switch (BN) {
    case 16: return launch_typed<1, 16>(st, num_sms, dtype, prm);
    case 32: return launch_typed<1, 32>(st, num_sms, dtype, prm);
    default: return launch_typed<1, 64>(st, num_sms, dtype, prm);
    }
}

}  // namespace gvq
