// The orthogonalised update of all matrices of a flat gradient (gvq.h, gvq_ortho_*): momentum, five Newton-Schulz steps
//
//     X <- u / |u|_F;   A = X X^T,   B = b A + c A^2,   X <- a X + B X        (on the shorter side)
//
// and the weights' update, each pass over all matrices in one launch.
//
// Nothing is transposed.  A matrix with rows <= cols ("wide") works with X X^T and B X, one with rows > cols ("tall")
// with X^T X and X B; the tensor core reads an operand K-major or MN-major, so X is one row-major array for all of:
//     wide   A = X X^T   both operands K-major       X' = B X   B K-major (symmetric), X MN-major
//     tall   A = X^T X   both operands MN-major      X' = X B   both K-major
// A and B are symmetric: only tiles that touch or lie above the diagonal are computed, and stored twice.
//
// Precision.  The products take half-precision operands (11 significant bits; bf16 would leave 8) and accumulate in
// fp32.  Powers of two keep the operands in range.  X in half precision alone would lose what matters most: rounding X
// adds noise to every direction alike, and the first steps amplify the small singular directions, noise included, by
// 3.4 each (an rms error of 5e-3 in the result for a low-rank gradient over noise, against 1e-3 for a Gaussian one).
// The a X term carries X forward, so X is kept as a sum of two halves (22 bits) for the first kExactSteps steps; the
// products take the high half.  After that the steps contract the noise of the large directions, and carrying it exactly
// would not help.  Measured on the CPU, relative to 64 bits: 0.4e-3 to 1.4e-3 for sides of 256 and more.
#include "ortho.h"
#include "row32.cuh"
#include "sm100_ptx.cuh"

namespace gvq {
namespace ortho {
namespace {

using namespace ptx;

// ---- element-wise passes ---------------------------------------------------------------------------

__device__ __forceinline__ float block_sum(float v, float *scratch)   // 256 threads; fixed order
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    float t = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) t += scratch[i];
    __syncthreads();
    return t;
}

// u from the gradient and the momentum that momentum_kernel has updated: the same roundings in both passes
__device__ __forceinline__ float direction(float g, float mo, float beta, int mode)
{
    return mode == 0 ? g : mode == 1 ? mo : __fmaf_rn(beta, mo, g);
}

struct StartParams {
    Device dev;
    ElementArgs a;
    int mode;      // 0: no momentum, 1: momentum, 2: nesterov
};

__global__ void __launch_bounds__(256) momentum_kernel(const StartParams prm)
{
    __shared__ float scratch[8];
    const Chunk ch = prm.dev.chunks[blockIdx.x];
    const Matrix &mx = prm.dev.mats[ch.matrix];
    const int64_t total = (int64_t)mx.rows * mx.cols, begin = (int64_t)ch.index * kChunk;
    const int n = (int)min((int64_t)kChunk, total - begin);
    const float *g = prm.a.g + mx.off + begin;        // 16-byte aligned: layers start at multiples of 4
    float *mo = prm.mode ? prm.a.momentum + mx.off + begin : nullptr;
    float sum = 0.0f;
#pragma unroll 4
    for (int i = threadIdx.x * 4; i < n; i += 1024) {
        float gv[4], mv[4] = {0.f, 0.f, 0.f, 0.f};
        const bool full = i + 4 <= n;
        if (full) {
            const float4 q = *reinterpret_cast<const float4 *>(g + i);
            gv[0] = q.x; gv[1] = q.y; gv[2] = q.z; gv[3] = q.w;
            if (prm.mode) {
                const float4 m = *reinterpret_cast<const float4 *>(mo + i);
                mv[0] = m.x; mv[1] = m.y; mv[2] = m.z; mv[3] = m.w;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                gv[e] = i + e < n ? g[i + e] : 0.0f;
                if (prm.mode && i + e < n) mv[e] = mo[i + e];
            }
        }
        if (prm.mode) {
#pragma unroll
            for (int e = 0; e < 4; ++e) mv[e] = __fmaf_rn(prm.a.beta, mv[e], gv[e]);
            if (full) {
                *reinterpret_cast<float4 *>(mo + i) = make_float4(mv[0], mv[1], mv[2], mv[3]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (i + e < n) mo[i + e] = mv[e];
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float u = direction(gv[e], mv[e], prm.a.beta, prm.mode);
            sum = __fmaf_rn(u, u, sum);
        }
    }
    sum = block_sum(sum, scratch);
    if (threadIdx.x == 0) prm.dev.partial[blockIdx.x] = sum;
}

// X = u / (|u| + eps), as a sum of two halves, in rows of ldx entries.
__global__ void __launch_bounds__(256) normalise_kernel(const StartParams prm)
{
    __shared__ double norm_s[8];
    const Chunk ch = prm.dev.chunks[blockIdx.x];
    const Matrix mx = prm.dev.mats[ch.matrix];
    double s = 0.0;
    for (int i = threadIdx.x; i < mx.n_chunks; i += 256) s += (double)prm.dev.partial[mx.chunk0 + i];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((threadIdx.x & 31) == 0) norm_s[threadIdx.x >> 5] = s;
    __syncthreads();
    s = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += norm_s[i];
    const float f = mx.sx / ((float)sqrt(s) + kEps);
    const int64_t total = (int64_t)mx.rows * mx.cols, begin = (int64_t)ch.index * kChunk;
    const int n = (int)min((int64_t)kChunk, total - begin);
    const float *g = prm.a.g + mx.off + begin;
    const float *mo = prm.mode ? prm.a.momentum + mx.off + begin : nullptr;
#pragma unroll 4
    for (int i = threadIdx.x * 4; i < n; i += 1024) {
        float gv[4], mv[4] = {0.f, 0.f, 0.f, 0.f};
        const bool full = i + 4 <= n;
        if (full) {
            const float4 q = __ldcs(reinterpret_cast<const float4 *>(g + i));
            gv[0] = q.x; gv[1] = q.y; gv[2] = q.z; gv[3] = q.w;
            if (prm.mode) {
                const float4 m = __ldcs(reinterpret_cast<const float4 *>(mo + i));
                mv[0] = m.x; mv[1] = m.y; mv[2] = m.z; mv[3] = m.w;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                gv[e] = i + e < n ? g[i + e] : 0.0f;
                if (prm.mode && i + e < n) mv[e] = mo[i + e];
            }
        }
        __half hi[4], lo[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float x = direction(gv[e], mv[e], prm.a.beta, prm.mode) * f;
            hi[e] = __float2half_rn(x);
            lo[e] = __float2half_rn(x - __half2float(hi[e]));
        }
        const int64_t at = begin + i;
        const int64_t row = at / mx.cols;
        int col = (int)(at - row * mx.cols);
        int64_t dst = row * mx.ldx + col;
        if (full && (mx.cols & 3) == 0) {
            uint2 q;
            memcpy(&q, hi, 8); *reinterpret_cast<uint2 *>(mx.x[0] + dst) = q;
            memcpy(&q, lo, 8); *reinterpret_cast<uint2 *>(mx.lo + dst) = q;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (i + e < n) { mx.x[0][dst] = hi[e]; mx.lo[dst] = lo[e]; }
                ++dst;
                if (++col == mx.cols) { col = 0; dst += mx.ldx - mx.cols; }
            }
        }
    }
}

// ---- the products ------------------------------------------------------------------------------------
// One persistent CTA per SM, tiles of 128 x 256, 64 steps of the contraction a stage.  Every operand comes in boxes of
// 64 x 64 entries (8 KB, 128-byte swizzle, zero fill outside), the same tensor map for either major:
//   K-major   box = 64 steps x 64 rows     MN-major   box = 64 entries across x 64 steps
// two boxes for A, four for B.
//   warp 0      producer      warp 1  MMA      warps 2-9  epilogue (lane quarter warp % 4, half the columns each)
constexpr int KS = 64, STAGES = 4, NTHREADS = 320, NEPI = 8;
constexpr uint32_t BOX = 64 * 128, A_BYTES = 2 * BOX, B_BYTES = 4 * BOX, STAGE = A_BYTES + B_BYTES;
constexpr size_t PRODUCT_SMEM = (size_t)STAGES * STAGE + 256 + 1024;

struct ProductParams {
    Device dev;
    OutputArgs out;
    int step;            // 0 .. kSteps - 1
    int32_t *error_word;
    int wait_kcycles, test_drop;
};

// Geometry of a tile, the same for every role.
struct Work {
    int M, N, K;         // extents of the whole product
    int a_map, b_map;
    bool a_mn, b_mn;
};
template <int PHASE>
__device__ __forceinline__ Work work_of(const Matrix &m, int step)
{
    const int x = step & 1;
    if (PHASE == kGram) return {m.r, m.r, m.c, x, x, m.tall != 0, m.tall != 0};
    if (PHASE == kPoly) return {m.r, m.r, m.r, kGramMap, kGramMap, false, false};
    return m.tall ? Work{m.rows, m.cols, m.r, x, kPolyMap, false, false} : Work{m.rows, m.cols, m.r, kPolyMap, x, false, true};
}

// The last step's result of 32 columns of a row.
template <typename T>
__device__ __forceinline__ void write_result(const OutputArgs &o, const Matrix &mx, int m, int col0, int n, float (&v)[32])
{
    T *dst = static_cast<T *>(o.ptr) + mx.off + (int64_t)m * mx.cols + col0;
    if (o.update) {
        float w[32];
        load_row32(dst, w, n);
        const float k = o.step * mx.scale;
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = __fmaf_rn(-k, v[i], o.decay * w[i]);
    }
    store_row32(dst, v, n);
}

template <int PHASE>
__global__ void __launch_bounds__(NTHREADS, 1) product_kernel(const __grid_constant__ ProductParams prm)
{
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    uint64_t *bars = reinterpret_cast<uint64_t *>(smem + (size_t)STAGES * STAGE);
    uint64_t *full = bars, *empty = full + STAGES, *d_full = empty + STAGES, *d_empty = d_full + 2;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(d_empty + 2);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < STAGES; ++i) { mbar_init(full + i, 1); mbar_init(empty + i, 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(d_full + i, 1); mbar_init(d_empty + i, NEPI); }
        *abort_flag = 0;
        const_cast<int *>(abort_flag)[2] = prm.wait_kcycles;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(smem_u32(tmem_slot)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    bool failed = false;
    const Tile *tiles = PHASE == kApply ? prm.dev.apply_tiles : prm.dev.sym_tiles;
    const int n_tiles = PHASE == kApply ? prm.dev.n_apply : prm.dev.n_sym;

    if (warp == 0) {
        if (lane == 0) {
            uint32_t c = 0;
            for (int t = blockIdx.x; t < n_tiles && !failed; t += gridDim.x) {
                const Tile tile = tiles[t];
                const Work w = work_of<PHASE>(prm.dev.mats[tile.matrix], prm.step);
                const CUtensorMap *ma = prm.dev.maps + (size_t)tile.matrix * kMaps + w.a_map;
                const CUtensorMap *mb = prm.dev.maps + (size_t)tile.matrix * kMaps + w.b_map;
                const int m0 = tile.tm * kTileM, n0 = tile.tn * kTileN;
                // boxes that hold anything of the product
                const int na = min(2, (w.M - m0 + 63) / 64), nb = min(4, (w.N - n0 + 63) / 64);
                const int n_stages = (w.K + KS - 1) / KS;
                for (int st = 0; st < n_stages; ++st, ++c) {
                    const uint32_t s = c % STAGES;
                    if (!mbar_wait(empty + s, ((c / STAGES) & 1) ^ 1, abort_flag)) { failed = true; break; }
                    if (prm.test_drop && blockIdx.x == 0 && c == 0) continue;   // test hook: this stage never arrives
                    unsigned char *dst = smem + (size_t)s * STAGE;
                    mbar_arrive_expect_tx(full + s, (na + nb) * BOX);
                    const int k = st * KS;
                    for (int i = 0; i < na; ++i)
                        tma_load_2d(dst + i * BOX, ma, w.a_mn ? m0 + 64 * i : k, w.a_mn ? k : m0 + 64 * i, full + s);
                    for (int i = 0; i < nb; ++i)
                        tma_load_2d(dst + A_BYTES + i * BOX, mb, w.b_mn ? n0 + 64 * i : k, w.b_mn ? k : n0 + 64 * i, full + s);
                }
            }
            if (failed) {   // give the copies already in flight a bounded chance to land before the CTA exits
                for (uint32_t i = c > STAGES ? c - STAGES : 0; i < c; ++i)
                    for (int it = 0; it < 100000 && !mbar_try_wait(full + i % STAGES, (i / STAGES) & 1); ++it) {}
            }
        }
        failed = __shfl_sync(0xffffffffu, failed, 0);
    } else if (warp == 1) {
        uint32_t c = 0, u = 0;
        for (int t = blockIdx.x; t < n_tiles && !failed; t += gridDim.x, ++u) {
            const Tile tile = tiles[t];
            const Work w = work_of<PHASE>(prm.dev.mats[tile.matrix], prm.step);
            const uint32_t buf = u & 1, d = tmem + buf * 256;
            const int n = min(kTileN, (w.N - tile.tn * kTileN + 15) / 16 * 16);
            const uint32_t idesc = make_idesc_f16(n, w.a_mn, w.b_mn);
            const int n_stages = (w.K + KS - 1) / KS;
            bool ok = mbar_wait(d_empty + buf, ((u >> 1) & 1) ^ 1, abort_flag);
            if (!__all_sync(0xffffffffu, ok)) { failed = true; break; }
            tc_fence_after();
            for (int st = 0; st < n_stages; ++st, ++c) {
                const uint32_t s = c % STAGES;
                ok = mbar_wait(full + s, (c / STAGES) & 1, abort_flag);
                if (!__all_sync(0xffffffffu, ok)) { failed = true; break; }
                tc_fence_after();
                const uint32_t base = smem_u32(smem + (size_t)s * STAGE);
                const uint64_t da = w.a_mn ? make_mn_desc(base, BOX) : make_b_desc(base);
                const uint64_t db = w.b_mn ? make_mn_desc(base + A_BYTES, BOX) : make_b_desc(base + A_BYTES);
                // 16 steps of the contraction: 32 bytes of a K-major row, 16 rows of 128 bytes of an MN-major box
                const uint32_t ia = w.a_mn ? 16 * 128 / 16 : 2, ib = w.b_mn ? 16 * 128 / 16 : 2;
                const int n_mma = min(4, (w.K - st * KS + 15) / 16);
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (k < n_mma) tc_mma_f16(d, da + k * ia, db + k * ib, idesc, (st | k) != 0);
                    tc_commit(empty + s);
                    if (st == n_stages - 1) tc_commit(d_full + buf);
                }
                __syncwarp();
            }
        }
    } else {
        const int q = warp & 3, half = (warp - 2) >> 2;
        const uint32_t lane_base = (uint32_t)(32 * q) << 16;
        uint32_t u = 0;
        for (int t = blockIdx.x; t < n_tiles; t += gridDim.x, ++u) {
            const Tile tile = tiles[t];
            const Matrix mx = prm.dev.mats[tile.matrix];
            const Work w = work_of<PHASE>(mx, prm.step);
            const uint32_t buf = u & 1;
            bool ok = mbar_wait(d_full + buf, (u >> 1) & 1, abort_flag);
            if (!__all_sync(0xffffffffu, ok)) { failed = true; break; }
            tc_fence_after();
            const int m = tile.tm * kTileM + 32 * q + lane;
            // a tile right of the diagonal's 256 x 256 block stands for its mirror image too
            const bool mirror = PHASE != kApply && tile.tn > tile.tm / 2;
#pragma unroll 1
            for (int p = 0; p < 4; ++p) {
                const int cl = half * 128 + p * 32, col0 = tile.tn * kTileN + cl;
                if (col0 >= w.N) break;
                float v[32];
                tmem_ld32_wait(tmem + lane_base + buf * 256 + cl, v);
                const int n = m < w.M ? min(32, w.N - col0) : 0;
                if (n <= 0) continue;
                if (PHASE == kApply) {
                    const int64_t at = (int64_t)m * mx.ldx + col0;
                    const int np = min(32, mx.ldx - col0);     // rows are padded: whole pieces of eight
                    float x[32];
                    load_row32(mx.x[prm.step & 1] + at, x, np);
                    if (prm.step < kExactSteps) {
                        float lo[32];
                        load_row32(mx.lo + at, lo, np);
#pragma unroll
                        for (int i = 0; i < 32; ++i) x[i] += lo[i];
                    }
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = __fmaf_rn(kA, x[i], v[i] * (1.0f / kGramScale));
                    if (prm.step < kSteps - 1) {
                        store_row32(mx.x[(prm.step + 1) & 1] + at, v, np);
                        if (prm.step + 1 < kExactSteps) {
#pragma unroll
                            for (int i = 0; i < 32; ++i) v[i] -= __half2float(__float2half_rn(v[i]));
                            store_row32(mx.lo + at, v, np);
                        }
                    } else {
                        const float f = 1.0f / mx.sx;
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] *= f;
                        if (prm.out.dtype == GVQ_F32) write_result<float>(prm.out, mx, m, col0, n, v);
                        else if (prm.out.dtype == GVQ_BF16) write_result<__nv_bfloat16>(prm.out, mx, m, col0, n, v);
                        else write_result<__half>(prm.out, mx, m, col0, n, v);
                    }
                } else {
                    const int64_t at = (int64_t)m * mx.ldr + col0;
                    if (PHASE == kGram) {
                        const float f = kGramScale / (mx.sx * mx.sx);
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] *= f;
                    } else {
                        float a[32];
                        load_row32(mx.gram + at, a, min(32, mx.ldr - col0));
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] = __fmaf_rn(kB, a[i], v[i] * (kC / kGramScale));
                    }
                    __half *dst = PHASE == kGram ? mx.gram : mx.poly;
                    store_row32(dst + at, v, min(32, mx.ldr - col0));
                    if (mirror) {
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (i < n) dst[(int64_t)(col0 + i) * mx.ldr + m] = __float2half_rn(v[i]);
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(d_empty + buf);
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
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

}  // namespace

cudaError_t launch_start(cudaStream_t st, const Device &dev, const ElementArgs &a)
{
    StartParams prm;
    prm.dev = dev;
    prm.a = a;
    prm.mode = !a.momentum ? 0 : a.nesterov ? 2 : 1;
    momentum_kernel<<<dev.n_chunks, 256, 0, st>>>(prm);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    normalise_kernel<<<dev.n_chunks, 256, 0, st>>>(prm);
    return cudaGetLastError();
}

cudaError_t launch_product(cudaStream_t st, int num_sms, const Device &dev, Phase phase, int step, const OutputArgs *out,
                           int32_t *error_word, int wait_kcycles, int test_drop)
{
    ProductParams prm;
    prm.dev = dev;
    prm.out = out ? *out : OutputArgs{};
    prm.step = step;
    prm.error_word = error_word;
    prm.wait_kcycles = wait_kcycles > 0 ? wait_kcycles : WAIT_KCYCLES_DEFAULT;
    prm.test_drop = test_drop;
    const int n = phase == kApply ? dev.n_apply : dev.n_sym;
    const int grid = n < num_sms ? n : num_sms;
    auto launch = [&](auto kernel) {
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)PRODUCT_SMEM);
        if (e != cudaSuccess) return e;
        kernel<<<grid, NTHREADS, PRODUCT_SMEM, st>>>(prm);
        return cudaGetLastError();
    };
    if (phase == kGram) return launch(product_kernel<kGram>);
    if (phase == kPoly) return launch(product_kernel<kPoly>);
    return launch(product_kernel<kApply>);
}

}  // namespace ortho
}  // namespace gvq
