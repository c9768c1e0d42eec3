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
// A, b I + c A and P are symmetric: only tiles that touch or lie right of the diagonal are computed and stored; an operand
// tile left of it is read as the transposed tile, in the other major.
//
// Precision.  The products take half-precision operands (11 significant bits; bf16 would leave 8) and accumulate in
// fp32.  Powers of two keep the operands in range.  X in half precision alone would lose what matters most: rounding X
// adds noise to every direction alike, and the first steps amplify the small singular directions, noise included, by
// 3.4 each (an rms error of 5e-3 in the result for a low-rank gradient over noise, against 1e-3 for a Gaussian one).
// The a X term carries X forward, so X is kept as a sum of two halves (22 bits) for the first kExactSteps steps; the
// products take the high half,  X' = (a I + b A + c A^2) X_hi + a X_lo.  After that the steps contract the noise of the large directions, and carrying it exactly
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
    ptx::launch_dependents();
    ptx::grid_dependency_wait();
    const Chunk ch = prm.dev.chunks[blockIdx.x];
    const Matrix &mx = prm.dev.mats[ch.matrix];
    const int64_t total = (int64_t)mx.rows * mx.cols, begin = (int64_t)ch.index * prm.dev.chunk;
    const int n = (int)min((int64_t)prm.dev.chunk, total - begin);
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
    ptx::launch_dependents();
    ptx::grid_dependency_wait();
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
    const int64_t total = (int64_t)mx.rows * mx.cols, begin = (int64_t)ch.index * prm.dev.chunk;
    const int n = (int)min((int64_t)prm.dev.chunk, total - begin);
    const float *g = prm.a.g + mx.off + begin;
    const float *mo = prm.mode ? prm.a.momentum + mx.off + begin : nullptr;
    auto row_of = [&](int64_t at) { return (int64_t)__umul64hi((uint64_t)at << 2, mx.by_cols); };
    if ((mx.cols & 3) == 0) {       // (so n and every row hold whole quads)
#pragma unroll 4
        for (int i = threadIdx.x * 4; i < n; i += 1024) {
            const float4 gq = __ldcs(reinterpret_cast<const float4 *>(g + i));
            const float4 mq = prm.mode ? __ldcs(reinterpret_cast<const float4 *>(mo + i)) : make_float4(0.f, 0.f, 0.f, 0.f);
            const float x[4] = {direction(gq.x, mq.x, prm.a.beta, prm.mode) * f, direction(gq.y, mq.y, prm.a.beta, prm.mode) * f,
                                direction(gq.z, mq.z, prm.a.beta, prm.mode) * f, direction(gq.w, mq.w, prm.a.beta, prm.mode) * f};
            uint2 hi, lo;
            hi.x = pack2<__half>(x[0], x[1]);
            hi.y = pack2<__half>(x[2], x[3]);
            const float2 a = unpack_half2(hi.x), b = unpack_half2(hi.y);
            lo.x = pack2<__half>(x[0] - a.x, x[1] - a.y);
            lo.y = pack2<__half>(x[2] - b.x, x[3] - b.y);
            const int64_t at = begin + i, row = row_of(at), dst = row * mx.ldx + (at - row * mx.cols);
            *reinterpret_cast<uint2 *>(mx.x[0] + dst) = hi;
            *reinterpret_cast<uint2 *>(mx.lo + dst) = lo;
        }
    } else {                        // an entry a lane: rows begin anywhere
#pragma unroll 4
        for (int i = threadIdx.x; i < n; i += 256) {
            const float x = direction(__ldcs(g + i), prm.mode ? __ldcs(mo + i) : 0.0f, prm.a.beta, prm.mode) * f;
            const __half hi = __float2half_rn(x);
            const int64_t at = begin + i, row = row_of(at), dst = row * mx.ldx + (at - row * mx.cols);
            mx.x[0][dst] = hi;
            mx.lo[dst] = __float2half_rn(x - __half2float(hi));
        }
    }
}

// ---- the products ------------------------------------------------------------------------------------
// Persistent CTAs (or pairs of CTAs), 64 steps of the contraction a stage.  Every operand comes in boxes of 64 x 64 entries
// (8 KB, 128-byte swizzle, zero fill outside), the same tensor map for either major:
//   K-major   box = 64 steps x 64 rows     MN-major   box = 64 entries across x 64 steps
//   warp 0      producer      warp 1  MMA      then the epilogue's warps (lane quarter warp % 4; a pair's CTA has eight, half
//               the columns each): 64 columns at a time, staged in half precision and stored by TMA
// Two tilings:
//   CG = 2  a pair of CTAs on two SMs, tile 256 x 256: each loads and holds its own 128 rows of A and half of B's rows, the
//           even one issues MMAs that read both.  32 KB a stage and SM for 512 clocks of MMAs; a CTA alone on 128 x 256
//           would load 48 KB, more than L2 delivers to all SMs at that rate.
//   CG = 1  one CTA, tile 128 x 64, for plans without enough large tiles to fill the GPU: four times the CTAs at work, a
//           quarter of the time a stage.
// A's contraction is the long side of the matrix and its tiles may be few: there the contraction is split between CTAs
// (Tile::parts).  The sums of all parts go to scratch in fp32, a warp's piece by piece; of the warps that hold the same
// piece of a tile the last to arrive adds the parts in their order and goes on with the epilogue, so the result does not
// depend on who that is.
constexpr int KS = 64;
constexpr uint32_t BOX = 64 * 128;
constexpr uint32_t kStaging = 8192;      // of an epilogue warp: two pieces of 32 rows x 128 bytes

template <int CG> struct Shape {
    static constexpr int BN = CG == 2 ? kPairN : kSoloN;                     // columns of a tile
    static constexpr int BLOCK = 128 * CG;                                   // of the diagonal of a symmetric result
    static constexpr int NB = CG == 2 ? 2 : BN / 64;                        // boxes of B a CTA loads
    static constexpr uint32_t A_BYTES = 2 * BOX, STAGE = A_BYTES + NB * BOX;
    static constexpr int STAGES = 5;
    static constexpr int NEPI = CG == 2 ? 8 : 4, THREADS = 64 + 32 * NEPI;   // epilogue warps
    static constexpr uint32_t TMEM = 2 * BN;                                 // two accumulators
    static constexpr size_t SMEM = (size_t)STAGES * STAGE + NEPI * kStaging + 256 + 1024;
};

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
    bool a_mn, b_mn;     // MN-major operands
    bool a_sym, b_sym;   // symmetric ones, stored on and right of the diagonal
};
template <int PHASE>
__device__ __forceinline__ Work work_of(const Matrix &m, int step)
{
    const int x = step & 1;
    if (PHASE == kGram) return {m.r, m.r, m.c, x, x, m.tall != 0, m.tall != 0, false, false};
    if (PHASE == kPoly) return {m.r, m.r, m.r, kGramMap, kFactorMap, false, false, true, true};
    return m.tall ? Work{m.rows, m.cols, m.r, x, kPolyMap, false, false, false, true}
                  : Work{m.rows, m.cols, m.r, kPolyMap, x, false, true, true, false};
}

// The last step's result: out = X, or w = decay w - step scale X, with the weights fetched a piece ahead.
//   wide     rows start at 16-byte boundaries: a lane has a row, 128 bytes of it at a time, for the arithmetic (as tensor
//            memory is read), and an eighth of four rows' 128 bytes for the stores
//   others   32 x 32 entries at a time: a lane has a column, or two neighbouring ones of a 16-bit type whose rows start at
//            4-byte boundaries, of every row or every other row
template <typename T> struct Weights {
    static constexpr int WIDE = 128 / (int)sizeof(T);     // columns of a wide piece
    uint32_t w[32];

    static __device__ __forceinline__ bool wide(const OutputArgs &o, const Matrix &mx)
    {
        return (mx.cols * (int64_t)sizeof(T)) % 16 == 0 && (reinterpret_cast<uintptr_t>(static_cast<T *>(o.ptr) + mx.off) & 15u) == 0;
    }
    static __device__ __forceinline__ bool paired(const OutputArgs &o, const Matrix &mx)
    {
        return sizeof(T) == 2 && (mx.cols & 1) == 0 && (reinterpret_cast<uintptr_t>(static_cast<T *>(o.ptr) + mx.off) & 3u) == 0;
    }
    // the piece at (m, n); rows, cols: what of the matrix begins there
    __device__ __forceinline__ void fetch(const OutputArgs &o, const Matrix &mx, int lane, int m, int n, int rows, int cols)
    {
        if (!o.update) return;
        const T *at = static_cast<const T *>(o.ptr) + mx.off + (int64_t)m * mx.cols + n;
        if (wide(o, mx)) {
            const T *d = at + (int64_t)lane * mx.cols;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (lane < rows && i * (16 / (int)sizeof(T)) < cols) {
                    const uint4 q = *reinterpret_cast<const uint4 *>(d + i * (16 / (int)sizeof(T)));
                    w[4 * i] = q.x; w[4 * i + 1] = q.y; w[4 * i + 2] = q.z; w[4 * i + 3] = q.w;
                }
            }
        } else if (paired(o, mx)) {
            const T *d = at + (int64_t)(lane >> 4) * mx.cols + (lane & 15) * 2;
            const bool in = (lane & 15) * 2 < cols;      // cols is even: a layer's columns are, and 32
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (in && 2 * i + (lane >> 4) < rows) w[i] = *reinterpret_cast<const uint32_t *>(d + (int64_t)2 * i * mx.cols);
        } else {
            const T *d = at + lane;
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                if (lane < cols && i < rows) {
                    if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(d[(int64_t)i * mx.cols]);
                    else w[i] = *reinterpret_cast<const uint16_t *>(d + (int64_t)i * mx.cols);
                }
            }
        }
    }
    static __device__ __forceinline__ float entry(uint32_t bits)      // of a 16-bit type: the low half
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(bits);
        const uint16_t u = (uint16_t)bits;
        T e;
        memcpy(&e, &u, 2);
        return to_f(e);
    }
    // 64 columns of this lane's row (a 32-bit type: the first or last 32 of them), staged and stored
    __device__ __forceinline__ void finish_wide(const OutputArgs &o, const Matrix &mx, unsigned char *buf, int lane, int m, int n, int rows,
                                                int cols, float (&a)[32], float (&b)[32])
    {
        const float f = 1.0f / (kGramScale * mx.sx), k = o.update ? -o.step * mx.scale * f : f;
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float(&x)[32] = h ? b : a;
                    const uint32_t two = w[16 * h + i / 2];
                    x[i] = o.update ? __fmaf_rn(k, x[i], o.decay * entry(two)) : x[i] * k;
                    x[i + 1] = o.update ? __fmaf_rn(k, x[i + 1], o.decay * entry(two >> 16)) : x[i + 1] * k;
                }
            }
            __syncwarp();
            stage_swizzled16<T>(buf, lane, a, b);
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) a[i] = o.update ? __fmaf_rn(k, a[i], o.decay * entry(w[i])) : a[i] * k;
            __syncwarp();
            stage_swizzled(buf, lane, a);
        }
        __syncwarp();
        const int c = (lane & 7) * (16 / (int)sizeof(T));
        T *d = static_cast<T *>(o.ptr) + mx.off + (int64_t)m * mx.cols + n + c;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = 4 * i + (lane >> 3);
            if (r < rows && c < cols)
                *reinterpret_cast<uint4 *>(d + (int64_t)r * mx.cols) =
                    *reinterpret_cast<const uint4 *>(buf + r * 128 + (((lane & 7) ^ (r & 7)) << 4));
        }
    }
    // a staged piece of 32 x 32
    __device__ __forceinline__ void finish(const OutputArgs &o, const Matrix &mx, const float *buf, int lane, int m, int n, int rows,
                                           int cols)
    {
        T *at = static_cast<T *>(o.ptr) + mx.off + (int64_t)m * mx.cols + n;
        const float f = 1.0f / (kGramScale * mx.sx), k = o.update ? -o.step * mx.scale * f : f;
        if (paired(o, mx)) {
            const int c = (lane & 15) * 2;
            T *d = at + (int64_t)(lane >> 4) * mx.cols + c;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int r = 2 * i + (lane >> 4);
                if (c < cols && r < rows) {
                    float2 x = *reinterpret_cast<const float2 *>(buf + r * kPiecePitch + c);
                    x.x = o.update ? __fmaf_rn(k, x.x, o.decay * entry(w[i])) : x.x * k;
                    x.y = o.update ? __fmaf_rn(k, x.y, o.decay * entry(w[i] >> 16)) : x.y * k;
                    if constexpr (sizeof(T) == 2) *reinterpret_cast<uint32_t *>(d + (int64_t)2 * i * mx.cols) = pack2<T>(x.x, x.y);
                }
            }
        } else if (lane < cols) {
            T *d = at + lane;
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                if (i < rows) {
                    float x = buf[i * kPiecePitch + lane];
                    x = o.update ? __fmaf_rn(k, x, o.decay * entry(w[i])) : x * k;
                    d[(int64_t)i * mx.cols] = from_f<T>(x);
                }
            }
        }
    }
};

__device__ __forceinline__ void prefetch_l2(const void *p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }
// 16 halves of a row (32 bytes, aligned)
__device__ __forceinline__ void load16(const __half *p, uint32_t (&w)[8])
{
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
}

// T: the type of the last step's result (PHASE kLast).
template <int PHASE, int CG, typename T = float>
__global__ void __launch_bounds__(Shape<CG>::THREADS, 1) product_kernel(const __grid_constant__ ProductParams prm)
{
    using S = Shape<CG>;
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    unsigned char *staging = smem + (size_t)S::STAGES * S::STAGE;
    uint64_t *bars = reinterpret_cast<uint64_t *>(staging + S::NEPI * kStaging);
    uint64_t *full = bars, *empty = full + S::STAGES, *d_full = empty + S::STAGES, *d_empty = d_full + 2;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(d_empty + 2);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = CG == 2 ? (int)cluster_rank() : 0;
    launch_dependents();
    if (threadIdx.x == 0) {
        for (int i = 0; i < S::STAGES; ++i) { mbar_init(full + i, 1); mbar_init(empty + i, 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(d_full + i, 1); mbar_init(d_empty + i, CG * S::NEPI); }
        *abort_flag = 0;
        const_cast<int *>(abort_flag)[2] = prm.wait_kcycles;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc<CG>(tmem_slot, S::TMEM);
    tc_fence_before();
    if (CG == 2) cluster_sync(); else __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    bool failed = false;
    // this CTA's (pair's) run of tiles; the plan's tables do not change, so they are read before the wait for the last launch
    constexpr bool APPLY = PHASE == kApply || PHASE == kLast;
    const Tile *tiles = prm.dev.run[PHASE].tiles;
    const int t_begin = prm.dev.run[PHASE].start[blockIdx.x / CG], t_end = prm.dev.run[PHASE].start[blockIdx.x / CG + 1];

    if (warp == 0) {
        if (lane == 0) {
            // a tile's geometry, looked up while the one before it is loaded
            struct Loads {
                const CUtensorMap *a, *b;
                int m0, n0, k0, k1, a_left, b_left;
                bool a_mn, b_mn;
            };
            auto loads_of = [&](int t) {
                const Tile tile = tiles[t];
                const Work w = work_of<PHASE>(prm.dev.mats[tile.matrix], prm.step);
                Loads l;
                l.a = prm.dev.maps + (size_t)tile.matrix * kMaps + w.a_map;
                l.b = prm.dev.maps + (size_t)tile.matrix * kMaps + w.b_map;
                // a pair's columns are split in halves of a multiple of 8 (the last tile's may be narrow)
                const int half_n = CG == 2 ? min(S::BN, (w.N - tile.tn * S::BN + 15) / 16 * 16) / 2 : 0;
                l.m0 = tile.tm * 128 * CG + 128 * rank;
                l.n0 = tile.tn * S::BN + half_n * rank;
                // steps of the contraction left of the diagonal's block of a symmetric operand's rows
                l.a_left = w.a_sym ? l.m0 / S::BLOCK * S::BLOCK : 0;
                l.b_left = w.b_sym ? tile.tn * S::BN / S::BLOCK * S::BLOCK : 0;
                l.a_mn = w.a_mn;
                l.b_mn = w.b_mn;
                l.k0 = tile.k0;
                l.k1 = tile.k1;
                return l;
            };
            Loads l = loads_of(t_begin);
            asm volatile("prefetch.tensormap [%0];" ::"l"(l.a));
            asm volatile("prefetch.tensormap [%0];" ::"l"(l.b));
            grid_dependency_wait();          // what the previous launch wrote is visible from here on
            fence_proxy_async_global();      // and read by TMA, plain stores included
            uint32_t c = 0;
            for (int t = t_begin; t < t_end && !failed; ++t) {
                const Loads next = loads_of(min(t + 1, t_end - 1));
                for (int st = l.k0; st < l.k1; ++st, ++c) {
                    const uint32_t s = c % S::STAGES;
                    if (!mbar_poll(empty + s, ((c / S::STAGES) & 1) ^ 1, abort_flag)) { failed = true; break; }
                    if (prm.test_drop && blockIdx.x == 0 && c == 0) continue;   // test hook: this stage never arrives
                    unsigned char *dst = smem + (size_t)s * S::STAGE;
                    if (rank == 0) mbar_arrive_expect_tx(full + s, CG * S::STAGE);
                    const int k = st * KS;
                    const uint32_t bar = CG == 2 ? in_leader(full + s) : 0;
                    auto load = [&](unsigned char *to, const CUtensorMap *map, bool mn, int at) {
                        if (CG == 2) tma_load_2d_pair(to, map, mn ? at : k, mn ? k : at, bar);
                        else tma_load_2d(to, map, mn ? at : k, mn ? k : at, full + s);
                    };
#pragma unroll
                    for (int i = 0; i < 2; ++i) load(dst + i * BOX, l.a, l.a_mn || k < l.a_left, l.m0 + 64 * i);
#pragma unroll
                    for (int i = 0; i < S::NB; ++i) load(dst + S::A_BYTES + i * BOX, l.b, l.b_mn || k < l.b_left, l.n0 + 64 * i);
                }
                l = next;
            }
            if (failed && rank == 0) {   // give the copies already in flight a bounded chance to land before the CTA exits
                for (uint32_t i = c > S::STAGES ? c - S::STAGES : 0; i < c; ++i)
                    for (int it = 0; it < 100000 && !mbar_try_wait(full + i % S::STAGES, (i / S::STAGES) & 1); ++it) {}
            }
        }
        failed = __shfl_sync(0xffffffffu, failed, 0);
    } else if (warp == 1) {
        uint32_t c = 0, u = 0;
        for (int t = t_begin; rank == 0 && t < t_end && !failed; ++t, ++u) {
            const Tile tile = tiles[t];
            const Work w = work_of<PHASE>(prm.dev.mats[tile.matrix], prm.step);
            const uint32_t buf = u & 1, d = tmem + buf * S::BN;
            const int n = min(S::BN, (w.N - tile.tn * S::BN + 15) / 16 * 16);
            const int a_left = w.a_sym ? tile.tm * 128 * CG / S::BLOCK * S::BLOCK : 0;
            const int b_left = w.b_sym ? tile.tn * S::BN / S::BLOCK * S::BLOCK : 0;
            bool ok = mbar_poll(d_empty + buf, ((u >> 1) & 1) ^ 1, abort_flag);
            if (!__all_sync(0xffffffffu, ok)) { failed = true; break; }
            tc_fence_after();
            for (int st = tile.k0; st < tile.k1; ++st, ++c) {
                const uint32_t s = c % S::STAGES;
                ok = mbar_poll(full + s, (c / S::STAGES) & 1, abort_flag);
                if (!__all_sync(0xffffffffu, ok)) { failed = true; break; }
                tc_fence_after();
                const uint32_t base = smem_u32(smem + (size_t)s * S::STAGE);
                const bool a_mn = w.a_mn || st * KS < a_left, b_mn = w.b_mn || st * KS < b_left;
                const uint32_t idesc = make_idesc_f16(128 * CG, n, a_mn, b_mn);
                const uint64_t da = a_mn ? make_mn_desc(base, BOX) : make_b_desc(base);
                const uint64_t db = b_mn ? make_mn_desc(base + S::A_BYTES, BOX) : make_b_desc(base + S::A_BYTES);
                // 16 steps of the contraction: 32 bytes of a K-major row, 16 rows of 128 bytes of an MN-major box
                const uint32_t ia = a_mn ? 16 * 128 / 16 : 2, ib = b_mn ? 16 * 128 / 16 : 2;
                const int n_mma = min(4, (w.K - st * KS + 15) / 16);
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (k < n_mma) tc_mma_f16<CG>(d, da + k * ia, db + k * ib, idesc, st > tile.k0 || k > 0);
                    if (CG == 2) tc_commit_pair(empty + s); else tc_commit(empty + s);
                    if (st == tile.k1 - 1) { if (CG == 2) tc_commit_pair(d_full + buf); else tc_commit(d_full + buf); }
                }
                __syncwarp();
            }
        }
    } else {
        const int q = warp & 3, half = (warp - 2) >> 2;
        const uint32_t lane_base = (uint32_t)(32 * q) << 16;
        unsigned char *mine = staging + (warp - 2) * kStaging;
        constexpr int COLS = S::BN / (S::NEPI / 4), PIECES = COLS / 64;      // of a warp
        const bool read_lo = PHASE == kApply && prm.step < kExactSteps;
        const bool write_lo = PHASE == kApply && prm.step + 1 < kExactSteps;
        // A tile as this warp sees it: its first row and column, its rows inside the product.
        struct Place {
            const Matrix *mx;
            int m0, c0, rows, N;
        };
        auto place = [&](int t) {
            const Tile tile = tiles[t];
            const Matrix *mx = prm.dev.mats + tile.matrix;
            const Work w = work_of<PHASE>(*mx, prm.step);
            const int m0 = tile.tm * 128 * CG + 128 * rank + 32 * q;
            return Place{mx, m0, tile.tn * S::BN + half * COLS, min(32, w.M - m0), w.N};
        };
        // What the epilogue reads besides the accumulator is asked for a piece ahead, across tiles, and a tile ahead into L2.
        uint32_t lo[4][8];
        auto fetch_lo = [&](const Place &at, int n0) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
#pragma unroll
                for (int e = 0; e < 8; ++e) lo[i][e] = 0;
                if (lane < at.rows && n0 + 16 * i < at.mx->ldx)
                    load16(at.mx->lo + (int64_t)(at.m0 + lane) * at.mx->ldx + n0 + 16 * i, lo[i]);
            }
        };
        Weights<T> weights;
        auto fetch_weights = [&](const Place &at, int n) {
            const int most = Weights<T>::wide(prm.out, *at.mx) ? Weights<T>::WIDE : 32;
            weights.fetch(prm.out, *at.mx, lane, at.m0, n, max(at.rows, 0), max(0, min(most, at.N - n)));
        };
        auto look_ahead = [&](const Place &at) {
            if (lane >= at.rows) return;
            if (PHASE == kApply && read_lo) {
                const __half *row = at.mx->lo + (int64_t)(at.m0 + lane) * at.mx->ldx;
#pragma unroll
                for (int c = 0; c < COLS; c += 64)
                    if (at.c0 + c < at.mx->ldx) prefetch_l2(row + at.c0 + c);
            }
            if (PHASE == kLast && prm.out.update) {
                const T *row = static_cast<const T *>(prm.out.ptr) + at.mx->off + (int64_t)(at.m0 + lane) * at.mx->cols;
#pragma unroll
                for (int c = 0; c < COLS; c += 128 / (int)sizeof(T))
                    if (at.c0 + c < at.N) prefetch_l2(row + at.c0 + c);
            }
        };
        Place here = place(t_begin);
        grid_dependency_wait();      // (before anything that another launch writes is read, or written)
        if (PHASE == kApply && read_lo) fetch_lo(here, here.c0);
        if (PHASE == kLast) fetch_weights(here, here.c0);
        uint32_t u = 0, stores = 0;
        for (int t = t_begin; t < t_end; ++t, ++u) {
            const Place next = place(min(t + 1, t_end - 1));
            const Matrix &mx = *here.mx;
            const int m0 = here.m0, c0 = here.c0, rows = here.rows;
            const CUtensorMap *maps = prm.dev.maps + (size_t)tiles[t].matrix * kMaps;
            const uint32_t ab = u & 1;
            if (APPLY && t + 1 < t_end) look_ahead(next);
            bool ok = mbar_poll(d_full + ab, (u >> 1) & 1, abort_flag);
            if (!__all_sync(0xffffffffu, ok)) { failed = true; break; }
            tc_fence_after();
            auto read_accumulator = [&](int p, float (&v)[2][32]) {
                tmem_ld32_wait(tmem + lane_base + ab * S::BN + half * COLS + p * 64, v[0]);
                tmem_ld32_wait(tmem + lane_base + ab * S::BN + half * COLS + p * 64 + 32, v[1]);
                if (p == PIECES - 1) {       // the accumulator is free
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) { if (CG == 2) mbar_arrive_cluster(in_leader(d_empty + ab)); else mbar_arrive(d_empty + ab); }
                }
            };
            // a part of a contraction: this warp's pieces go to scratch, and the last warp to bring its part goes on
            const int parts = PHASE == kGram ? tiles[t].parts : 1;
            constexpr int PER_CTA = 4 * S::BN / 64, PER_PART = CG * PER_CTA;      // pieces
            float4 *scratch = nullptr;
            if (PHASE == kGram && parts > 1) {
                const int first = tiles[t].slot + rank * PER_CTA + (q * (S::NEPI / 4) + half) * PIECES;
                scratch = reinterpret_cast<float4 *>(prm.dev.parts) + (int64_t)first * 512 + lane;
                float4 *own = scratch + (int64_t)tiles[t].part * PER_PART * 512;
#pragma unroll
                for (int p = 0; p < PIECES; ++p) {
                    float v[2][32];
                    read_accumulator(p, v);
                    if (rows <= 0 || c0 + p * 64 >= here.N) continue;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float *x = &v[i >> 3][4 * (i & 7)];
                        __stcg(own + p * 512 + 32 * i, make_float4(x[0], x[1], x[2], x[3]));
                    }
                }
                __threadfence();
                __syncwarp();
                int arrived = 0;
                if (lane == 0) arrived = atomicAdd(prm.dev.tickets + first, 1);
                if (__shfl_sync(0xffffffffu, arrived, 0) != parts - 1) { here = next; continue; }
                if (lane == 0) prm.dev.tickets[first] = 0;
                __threadfence();
            }
#pragma unroll
            for (int p = 0; p < PIECES; ++p) {
                const int n0 = c0 + p * 64;
                const bool live = rows > 0 && n0 < here.N;
                float v[2][32];
                if (PHASE == kGram && parts > 1) {
                    if (!live) continue;
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[0][i] = v[1][i] = 0.0f;
                    for (int part = 0; part < parts; ++part) {
                        const float4 *from = scratch + (int64_t)part * PER_PART * 512 + p * 512;
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const float4 x = __ldcg(from + 32 * i);
                            float *y = &v[i >> 3][4 * (i & 7)];
                            y[0] += x.x; y[1] += x.y; y[2] += x.z; y[3] += x.w;
                        }
                    }
                } else {
                    read_accumulator(p, v);
                }
                if (PHASE == kLast) {
                    const bool wide = Weights<T>::wide(prm.out, mx);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int n = n0 + 32 * h;
                        if (sizeof(T) == 2 && wide && h == 1) break;        // the first round took all 64 columns
                        if (live && n < here.N) {
                            if (wide) {
                                weights.finish_wide(prm.out, mx, mine, lane, m0, n, rows, min(Weights<T>::WIDE, here.N - n), v[h], v[h ^ 1]);
                            } else {
                                stage_piece(reinterpret_cast<float *>(mine), lane, v[h]);
                                weights.finish(prm.out, mx, reinterpret_cast<const float *>(mine), lane, m0, n, rows, min(32, here.N - n));
                            }
                        }
                        const int after = p * 64 + h * 32 + (wide ? Weights<T>::WIDE : 32);
                        if (after < COLS) fetch_weights(here, c0 + after);
                        else if (t + 1 < t_end) fetch_weights(next, next.c0);
                    }
                    continue;
                }
                if (PHASE == kApply) {       // X' = P X_hi + a X_lo
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int i = 0; i < 32; i += 2) {
                            v[h][i] *= 1.0f / kGramScale;
                            v[h][i + 1] *= 1.0f / kGramScale;
                            if (read_lo) {
                                const float2 l = unpack_half2(lo[2 * h + (i >> 4)][(i & 15) >> 1]);
                                v[h][i] = __fmaf_rn(kA, l.x, v[h][i]);
                                v[h][i + 1] = __fmaf_rn(kA, l.y, v[h][i + 1]);
                            }
                        }
                    if (read_lo) {
                        if (p + 1 < PIECES) fetch_lo(here, n0 + 64);
                        else if (t + 1 < t_end) fetch_lo(next, next.c0);
                    }
                }
                if (!live) continue;
                auto store = [&](unsigned char *from, int map) {      // the staged piece, by one lane
                    fence_proxy_async();
                    __syncwarp();
                    if (lane == 0) {
                        tma_store_2d(maps + map, n0, m0, from);
                        bulk_commit_group();
                    }
                };
                auto room = [&]() {      // one of the warp's two staging areas, once its last store has read it
                    if (lane == 0) bulk_wait_group_read<1>();
                    __syncwarp();
                    return mine + (stores++ & 1) * 4096;
                };
                if (PHASE == kApply) {
                    unsigned char *to = room();
                    stage_swizzled16<__half>(to, lane, v[0], v[1]);
                    store(to, kX0Out + ((prm.step + 1) & 1));
                    if (write_lo) {
#pragma unroll
                        for (int h = 0; h < 2; ++h)
#pragma unroll
                            for (int i = 0; i < 32; i += 2) {
                                const float2 f = unpack_half2(pack2<__half>(v[h][i], v[h][i + 1]));
                                v[h][i] -= f.x;
                                v[h][i + 1] -= f.y;
                            }
                        to = room();
                        stage_swizzled16<__half>(to, lane, v[0], v[1]);
                        store(to, kLoOut);
                    }
                    continue;
                }
                // A = X X^T and b I + c A, whose product with A the next launch takes; then P = a I + A (b I + c A)
                auto put = [&](int map) {
                    unsigned char *to = room();
                    stage_swizzled16<__half>(to, lane, v[0], v[1]);
                    store(to, map);
                };
                const float f = PHASE == kGram ? kGramScale / (mx.sx * mx.sx) : 1.0f / kGramScale;
                const float diagonal = (PHASE == kGram ? kB : kA) * kGramScale;
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[h][i] *= f;
                if (PHASE == kGram) put(kGramOut);
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        if (PHASE == kGram) v[h][i] *= kC;
                        if (n0 + 32 * h + i == m0 + lane) v[h][i] += diagonal;
                    }
                if (PHASE == kGram) put(kFactorOut); else put(kPolyOut);
            }
            here = next;
        }
        if (lane == 0) bulk_wait_group_all();
    }

    if (failed) {
        *abort_flag = 1;
        if (lane == 0) atomicExch(prm.error_word, 100 + warp);
    }
    tc_fence_before();
    if (CG == 2) cluster_sync(); else __syncthreads();     // a pair: the other CTA's barriers and memory are in use until here
    tc_fence_after();
    if (warp == 1) tmem_dealloc<CG>(tmem, S::TMEM);
}

template <int PHASE, typename T>
cudaError_t launch_tiling(cudaStream_t st, const ProductParams &prm, int runs)
{
    return prm.dev.pair ? launch_chained<product_kernel<PHASE, 2, T>>(prm, 2 * runs, Shape<2>::THREADS, Shape<2>::SMEM, 2, st)
                        : launch_chained<product_kernel<PHASE, 1, T>>(prm, runs, Shape<1>::THREADS, Shape<1>::SMEM, 1, st);
}

}  // namespace

cudaError_t launch_start(cudaStream_t st, const Device &dev, const ElementArgs &a)
{
    StartParams prm;
    prm.dev = dev;
    prm.a = a;
    prm.mode = !a.momentum ? 0 : a.nesterov ? 2 : 1;
    cudaError_t e = ptx::launch_chained<momentum_kernel>(prm, dev.n_chunks, 256, 0, 1, st);
    if (e != cudaSuccess) return e;
    return ptx::launch_chained<normalise_kernel>(prm, dev.n_chunks, 256, 0, 1, st);
}

cudaError_t launch_product(cudaStream_t st, const Device &dev, Phase phase, int step, const OutputArgs *out,
                           int32_t *error_word, int wait_kcycles, int test_drop)
{
    ProductParams prm;
    prm.dev = dev;
    prm.out = out ? *out : OutputArgs{};
    prm.step = step;
    prm.error_word = error_word;
    prm.wait_kcycles = wait_kcycles > 0 ? wait_kcycles : WAIT_KCYCLES_DEFAULT;
    prm.test_drop = test_drop;
    const int runs = dev.run[phase].runs;
    if (phase == kGram) return launch_tiling<kGram, float>(st, prm, runs);
    if (phase == kPoly) return launch_tiling<kPoly, float>(st, prm, runs);
    if (step < kSteps - 1) return launch_tiling<kApply, float>(st, prm, runs);
    if (out->dtype == GVQ_F32) return launch_tiling<kLast, float>(st, prm, runs);
    if (out->dtype == GVQ_BF16) return launch_tiling<kLast, __nv_bfloat16>(st, prm, runs);
    return launch_tiling<kLast, __half>(st, prm, runs);
}

}  // namespace ortho
}  // namespace gvq
