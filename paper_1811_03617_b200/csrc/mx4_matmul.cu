// Product of two matrices in microscaled 4-bit floating point,  D[m][n] = sum_k A[m][k] B[n][k],  on the
// block-scaled tcgen05 tensor path (gvq.h, "microscaled 4-bit").
//
// Both operands are quantized along the contraction, so both are K-major: a row of codes is contiguous.  The tensor
// core multiplies codes and applies the two blocks' scales itself, 64 entries of the contraction an instruction, and
// accumulates in fp32.
//
// One CTA: tiles of 128 rows of A x BN rows of B, 256 entries of the contraction a stage (128 bytes of codes a row).
//   warp 0      producer: per stage one TMA load of A's codes, one of B's (128-byte swizzle, zero fill outside), and a
//               bulk copy of the stage's scale bytes for each 128 rows (two tiles of 512 bytes, contiguous)
//   warp 1      MMA: copies the stage's scale tiles into tensor memory (each 128 x 4 tile becomes 4 columns), then up
//               to four MMAs; one elected lane issues, the order of issue is the order of execution
//   warps 2-5   epilogue: accumulator -> registers -> output
// Accumulators alternate between two column ranges.  Every mbarrier wait is bounded.
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
constexpr uint32_t A_BYTES = 128 * 128, SFA_BYTES = 2 * kTileBytes;

template <int BN> struct Shape {
    static constexpr int NRT = (BN + 127) / 128;                       // scale tiles of B side by side
    static constexpr uint32_t B_BYTES = BN * 128, SFB_BYTES = NRT * 2 * kTileBytes;
    static constexpr uint32_t STAGE = A_BYTES + B_BYTES + ((SFA_BYTES + SFB_BYTES + 1023) / 1024) * 1024;
    static constexpr int STAGES = BN == 256 ? 4 : 8;
    // tensor memory: two accumulators (256 columns each do not fit beside the scales: they overlap by 48 columns,
    // which the epilogue reads first), then two sets of scale columns
    static constexpr uint32_t ACC1 = BN == 256 ? 208 : BN;
    static constexpr uint32_t SF0 = ACC1 + BN, SF_SET = 8 + 8 * NRT;
    static constexpr uint32_t TMEM = 512;
    static constexpr size_t SMEM = (size_t)STAGE * STAGES + 256 + 1024;
    static_assert(SF0 + 2 * SF_SET <= TMEM, "tensor memory");
};

struct MmParams {
    CUtensorMap a, b;                 // codes: bytes x rows
    const uint8_t *sa, *sb;
    int64_t M, N, K;                  // rows of A, rows of B, contraction
    int kt;                           // scale tiles along the contraction
    int tiles_m, tiles_n, n_stages;   // of one tile's contraction
    void *out;
    int64_t out_m, out_n;             // strides of the output in entries, one of them 1
    int32_t *error_word;
    int wait_kcycles, test_drop;
};

__device__ __forceinline__ void bulk_load(void *dst, const void *src, uint32_t bytes, uint64_t *bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(smem_u32(dst)), "l"(src), "r"(bytes), "r"(smem_u32(bar)) : "memory");
}
// 128 x 4 scale bytes (32 rows of 16 bytes) -> 4 columns of tensor memory, the same in all four lane quarters
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint64_t desc)
{
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
__device__ __forceinline__ uint64_t scales_desc(uint32_t smem_addr)
{
    return (uint64_t)((smem_addr & 0x3FFFFu) >> 4) | ((uint64_t)(128 >> 4) << 16) | ((uint64_t)(128 >> 4) << 32) | ((uint64_t)1 << 46);
}
__device__ __forceinline__ void mma_mxf4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                         uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
}
// E2M1 x E2M1, power-of-two scales, M = 128; `half`: which pair of a scale column's four bytes (of A and of B)
__host__ __device__ constexpr uint32_t idesc_mxf4(int n, int half)
{
    return ((uint32_t)(2 * half) << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | (1u << 23) |
           ((uint32_t)(128 >> 4) << 24) | ((uint32_t)(2 * half) << 29);
}

template <typename T, int BN>
__global__ void __launch_bounds__(NTHREADS, 1) mx4_matmul_kernel(const __grid_constant__ MmParams prm)
{
    using S = Shape<BN>;
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    uint64_t *bars = reinterpret_cast<uint64_t *>(smem + (size_t)S::STAGE * S::STAGES);
    uint64_t *full = bars, *empty = full + S::STAGES;      // [STAGES]
    uint64_t *d_full = empty + S::STAGES;                  // [2] accumulator complete
    uint64_t *d_early = d_full + 2;                        // [2] the columns it shares with the other one are read
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(d_early + 2);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < S::STAGES; ++i) { mbar_init(full + i, 1); mbar_init(empty + i, 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(d_full + i, 1); mbar_init(d_early + i, 4); }
        *abort_flag = 0;
        const_cast<int *>(abort_flag)[2] = prm.wait_kcycles;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(smem_u32(tmem_slot)), "r"(S::TMEM) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    bool failed = false;

    const int n_tiles = prm.tiles_m * prm.tiles_n;
    const int64_t kb_last = prm.K - (int64_t)(prm.n_stages - 1) * KS;   // entries of the last stage, 1 .. 256

    if (warp == 0) {
        // ------------------------------------------------------------------ producer
        if (lane == 0) {
            uint32_t c = 0;
            for (int tile = blockIdx.x; tile < n_tiles && !failed; tile += gridDim.x) {
                const int tn = tile / prm.tiles_m, tm = tile - tn * prm.tiles_m;
                // scale tiles of B that exist (the second 128 rows may lie past the end)
                const int nrt = S::NRT == 2 && (int64_t)tn * BN + 128 >= prm.N ? 1 : S::NRT;
                for (int st = 0; st < prm.n_stages; ++st, ++c) {
                    const uint32_t s = c % S::STAGES;
                    if (!mbar_wait(empty + s, ((c / S::STAGES) & 1) ^ 1, abort_flag)) { failed = true; break; }
                    if (prm.test_drop && blockIdx.x == 0 && c == 0) continue;   // test hook: this stage never arrives
                    const uint32_t sf = min(2, prm.kt - 2 * st) * kTileBytes;
                    unsigned char *dst = smem + (size_t)s * S::STAGE;
                    mbar_arrive_expect_tx(full + s, A_BYTES + S::B_BYTES + sf * (1 + nrt));
                    tma_load_2d(dst, &prm.a, st * 128, tm * 128, full + s);
                    tma_load_2d(dst + A_BYTES, &prm.b, st * 128, tn * BN, full + s);
                    unsigned char *sc = dst + A_BYTES + S::B_BYTES;
                    bulk_load(sc, prm.sa + ((int64_t)tm * prm.kt + 2 * st) * kTileBytes, sf, full + s);
                    for (int r = 0; r < nrt; ++r)
                        bulk_load(sc + SFA_BYTES * (1 + r), prm.sb + (((int64_t)tn * BN / 128 + r) * prm.kt + 2 * st) * kTileBytes,
                                  sf, full + s);
                }
            }
            if (failed) {   // give the copies already in flight a bounded chance to land before the CTA exits
                for (uint32_t i = c > S::STAGES ? c - S::STAGES : 0; i < c; ++i)
                    for (int it = 0; it < 100000 && !mbar_try_wait(full + i % S::STAGES, (i / S::STAGES) & 1); ++it) {}
            }
        }
        failed = __shfl_sync(0xffffffffu, failed, 0);
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer
        uint32_t c = 0, t = 0;
        for (int tile = blockIdx.x; tile < n_tiles && !failed; tile += gridDim.x, ++t) {
            const uint32_t buf = t & 1;
            const uint32_t d = tmem + buf * S::ACC1;
            if (t > 0) {
                // the tile before this one has been read where the two accumulators overlap (and the one before
                // that, in this accumulator, entirely: the epilogue takes the tiles in order)
                bool ok = mbar_wait(d_early + (buf ^ 1), ((t - 1) >> 1) & 1, abort_flag);
                if (!__all_sync(0xffffffffu, ok)) { failed = true; break; }
                tc_fence_after();
            }
            for (int st = 0; st < prm.n_stages; ++st, ++c) {
                const uint32_t s = c % S::STAGES;
                bool ok = mbar_wait(full + s, (c / S::STAGES) & 1, abort_flag);
                if (!__all_sync(0xffffffffu, ok)) { failed = true; break; }
                tc_fence_after();
                const int64_t left = st == prm.n_stages - 1 ? kb_last : KS;
                const int n_mma = (int)((left + 63) / 64), n_kt = (n_mma + 1) >> 1;
                const uint32_t base = smem_u32(smem + (size_t)s * S::STAGE);
                const uint32_t sfa = tmem + S::SF0 + (c & 1) * S::SF_SET, sfb = sfa + 8;
                if (elect_one()) {
                    const uint32_t sc = base + A_BYTES + S::B_BYTES;
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        if (k < n_kt) {
                            copy_scales(sfa + 4 * k, scales_desc(sc + k * kTileBytes));
#pragma unroll
                            for (int r = 0; r < S::NRT; ++r)
                                copy_scales(sfb + 4 * (k * S::NRT + r), scales_desc(sc + SFA_BYTES * (1 + r) + k * kTileBytes));
                        }
                    }
                    const uint64_t da = make_b_desc(base), db = make_b_desc(base + A_BYTES);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (k < n_mma)
                            mma_mxf4(d, da + k * 2, db + k * 2, idesc_mxf4(BN, k & 1), sfa + 4 * (k >> 1),
                                     sfb + 4 * S::NRT * (k >> 1), (st | k) != 0);
                    tc_commit(empty + s);
                    if (st == prm.n_stages - 1) tc_commit(d_full + buf);
                }
                __syncwarp();
            }
        }
    } else {
        // ------------------------------------------------------------------ epilogue
        const int q = warp & 3;
        const uint32_t lane_base = (uint32_t)(32 * q) << 16;
        T *out = static_cast<T *>(prm.out);
        uint32_t t = 0;
        for (int tile = blockIdx.x; tile < n_tiles; tile += gridDim.x, ++t) {
            const int tn = tile / prm.tiles_m, tm = tile - tn * prm.tiles_m;
            const uint32_t buf = t & 1;
            bool ok = mbar_wait(d_full + buf, (t >> 1) & 1, abort_flag);
            if (!__all_sync(0xffffffffu, ok)) { failed = true; break; }
            tc_fence_after();
            const uint32_t acc = tmem + lane_base + buf * S::ACC1;
            const int64_t m = (int64_t)tm * 128 + 32 * q + lane;
            constexpr int PIECE = BN < 32 ? BN : 32, NP = BN / PIECE;
            // the first accumulator's last columns are the second one's first: those pieces come first
            constexpr int SHARED = BN == 256 ? 2 : 0;
#pragma unroll 1
            for (int p = 0; p < NP; ++p) {
                const int piece = buf == 0 && SHARED ? (p < SHARED ? NP - SHARED + p : p - SHARED) : p;
                float v[32];
                if (PIECE == 32) {
                    tmem_ld32_wait(acc + piece * 32, v);
                } else {
                    float w[16];
                    tmem_ld16_wait(acc + piece * 16, w);
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = i < 16 ? w[i] : 0.0f;
                }
                if (p == (SHARED ? SHARED - 1 : NP - 1)) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(d_early + buf);
                }
                const int64_t n = (int64_t)tn * BN + piece * PIECE;
                const int cols = (int)min((int64_t)PIECE, prm.N - n);
                if (m < prm.M && cols > 0) {
                    if (prm.out_n == 1) {
                        store_row32(out + m * prm.out_m + n, v, cols);
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (i < cols) out[m + (n + i) * prm.out_n] = from_f<T>(v[i]);
                    }
                }
            }
        }
    }

    if (failed) {
        *abort_flag = 1;
        if (lane == 0) atomicExch(prm.error_word, 100 + warp);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::TMEM) : "memory");
}

template <typename T, int BN>
cudaError_t launch_as(cudaStream_t st, int num_sms, const MmParams &prm)
{
    auto kernel = mx4_matmul_kernel<T, BN>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Shape<BN>::SMEM);
    if (e != cudaSuccess) return e;
    const int grid = min(num_sms, prm.tiles_m * prm.tiles_n);
    kernel<<<grid, NTHREADS, Shape<BN>::SMEM, st>>>(prm);
    return cudaGetLastError();
}
template <int BN>
cudaError_t launch_typed(cudaStream_t st, int num_sms, int dtype, const MmParams &prm)
{
    if (dtype == GVQ_F32) return launch_as<float, BN>(st, num_sms, prm);
    if (dtype == GVQ_BF16) return launch_as<__nv_bfloat16, BN>(st, num_sms, prm);
    return launch_as<__half, BN>(st, num_sms, prm);
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

}  // namespace

cudaError_t launch_mx4_matmul(cudaStream_t st, int num_sms, EncodeTiledFn enc, const uint8_t *a, const uint8_t *sa, const uint8_t *b,
                              const uint8_t *sb, int64_t M, int64_t N, int64_t K, void *out, int dtype, int64_t ld,
                              int32_t *error_word, int wait_kcycles, int test_drop)
{
    MmParams prm;
    // Few rows of A: B takes the 128-row side of the tile, and the tile is as wide as the few rows need.
    const bool swap = M <= 64;
    const int BN = !swap ? 256 : M <= 16 ? 16 : M <= 32 ? 32 : 64;
    prm.sa = swap ? sb : sa; prm.sb = swap ? sa : sb;
    prm.M = swap ? N : M; prm.N = swap ? M : N; prm.K = K;
    prm.kt = (int)mx4::tiles_of(mx4::blocks(K), mx4::kTileBlocks);
    prm.tiles_m = (int)mx4::tiles_of(prm.M, 128);
    prm.tiles_n = (int)mx4::tiles_of(prm.N, BN);
    prm.n_stages = (int)mx4::tiles_of(K, KS);
    prm.out = out;
    prm.out_m = swap ? 1 : ld; prm.out_n = swap ? ld : 1;
    prm.error_word = error_word;
    prm.wait_kcycles = wait_kcycles > 0 ? wait_kcycles : WAIT_KCYCLES_DEFAULT;
    prm.test_drop = test_drop;
    if (!encode(enc, &prm.a, swap ? b : a, prm.M, K, 128) || !encode(enc, &prm.b, swap ? a : b, prm.N, K, BN))
        return cudaErrorInvalidValue;
    switch (BN) {
    case 16: return launch_typed<16>(st, num_sms, dtype, prm);
    case 32: return launch_typed<32>(st, num_sms, dtype, prm);
    case 64: return launch_typed<64>(st, num_sms, dtype, prm);
    default: return launch_typed<256>(st, num_sms, dtype, prm);
    }
}

}  // namespace gvq
