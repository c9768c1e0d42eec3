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
// A and P = a I + b A + c A^2 are symmetric: only tiles that touch or lie right of the diagonal are computed and stored; an operand
// tile left of it is read as the transposed tile, in the other major.  P is made of what is symmetric exactly, A A and A:
// as A (b I + c A), its second factor rounded, its two sides differed (errors of 3.3e-3 instead of 2.7e-3 at 1024 x 1024).
//
// Precision.  The products take half-precision operands (11 significant bits; bf16 would leave 8) and accumulate in
// fp32.  Powers of two keep the operands in range.  X in half precision alone would lose what matters most: rounding X
// adds noise to every direction alike, and the steps amplify the small singular directions, noise included, by
// 3.4 each (an rms error of 5e-3 in the result for a low-rank gradient over noise, against 1e-3 for a Gaussian one).
// The a X term carries X forward, so X is kept as a sum of two halves (22 bits) for the first kExactSteps steps; the
// products take the high half,  X' = (a I + b A + c A^2) X_hi + a X_lo.  With three such steps instead of four, gradients of
// low rank were off by 3.3e-3 to 3.6e-3, with four by 1.9e-3 to 2.9e-3; in the last one the large directions, whose noise a step
// contracts, would get more back than they lose (Gaussian 2.1e-3 -> 2.2e-3).  Where the short side is short, A and P have few
// entries of like size and their own roundings do not average out.  Up to kSplitSide A is kept as a sum of two halves too, up
// to kSplitApply P as well, and the products are sums of products of halves (their contractions are short).
// Relative rms errors against 64 bits, shapes from 8 x 12 to 2000 x 2000 and 512 x 4608:
//   sums of rank-one terms of random factors, any number, over noise of any size    0.3e-3 to 2.9e-3
//   equal or decaying singular values                                              0.5e-3 to 3.6e-3
//   random entries in a few rows or columns, zeros elsewhere                        up to 5e-3
//   entries that are all alike: constants, signs, (partial) identities               up to 9.2e-3
// The last two are what is left of half-precision operands: roundings that do not average out, of X itself among them.
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

// Momentum and the sums of squares, fixed order.  Bound by memory: 14.7 M entries 27 us with cold caches, 6.5 TB/s.
__global__ void __launch_bounds__(256) momentum_kernel(const StartParams prm)
{
    __shared__ float scratch[8];
    ptx::launch_dependents();
    ptx::grid_dependency_wait();
    // (zero already, unless a launch of the last call gave up)
    for (int i = blockIdx.x * 256 + threadIdx.x; i < prm.dev.n_tickets; i += gridDim.x * 256) prm.dev.tickets[i] = 0;
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

// X = u / (|u| + eps), as a sum of two halves, in rows of ldx entries.  Bound by memory: 14.7 M entries 27 us, 6.4 TB/s.
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
// Persistent CTAs (or pairs of CTAs), 64 steps of the contraction a stage (a CTA alone: 128).  Every operand comes in boxes of 64 x 64 entries
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
// (Tile::parts).  The sums of all parts go to scratch in fp32, piece by piece; of the warps that hold the same piece of a
// tile the last to arrive adds the parts in their order and goes on with the epilogue, so the result does not depend on
// who that is.
constexpr int KS = 64;
constexpr uint32_t BOX = 64 * 128;
constexpr int kTable = 32;               // tiles of a run whose geometry is looked up ahead
constexpr uint32_t kStaging = 8192;      // of an epilogue warp: two pieces of 32 rows x 128 bytes

template <int CG> struct Shape {
    static constexpr int BN = CG == 2 ? kPairN : kSoloN;                     // columns of a tile
    static constexpr int BLOCK = 128 * CG;                                   // of the diagonal of a symmetric result
    static constexpr int NB = CG == 2 ? 2 : BN / 64;                        // boxes of B a CTA loads
    static constexpr uint32_t A_BYTES = 2 * BOX, BYTES = A_BYTES + NB * BOX;    // of KS steps of the contraction
    // Of a CTA alone they come two at a time: its four small MMAs take 128 clocks, waiting for them and reporting them 160.
    static constexpr int PER_STAGE = CG == 2 ? 1 : 2, STAGES = CG == 2 ? 5 : 4;
    static constexpr uint32_t STAGE = PER_STAGE * BYTES;
    static constexpr int NEPI = CG == 2 ? 8 : 4, THREADS = 64 + 32 * NEPI;   // epilogue warps
    static constexpr uint32_t TMEM = 2 * BN;                                 // two accumulators
    static constexpr size_t SMEM = (size_t)STAGES * STAGE + NEPI * kStaging + kTable * 48 + 256 + 1024;
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
    if (PHASE == kPoly) return {m.r, m.r, m.r, kGramMap, kGramMap, false, false, true, true};
    return m.tall ? Work{m.rows, m.cols, m.r, x, kPolyMap, false, false, false, true}
                  : Work{m.rows, m.cols, m.r, kPolyMap, x, false, true, true, false};
}

// The last step's result, 32 x 32 entries at a time: out = X, or w = decay w - step scale X, with the weights fetched a piece
// ahead.
//   quads    rows hold whole quads of entries: a lane has four entries of every fourth row, eight lanes a row's 32
//   others   a lane has a column, or two neighbouring ones of a 16-bit type whose rows start at 4-byte boundaries, of every
//            row or every other row
template <typename T> struct Weights {
    uint32_t w[32];
    struct alignas(4 * sizeof(T)) Quad { T v[4]; };

    static __device__ __forceinline__ bool quads(const Matrix &mx) { return (mx.cols & 3) == 0; }    // (layers start at quads too)
    static __device__ __forceinline__ bool paired(const OutputArgs &o, const Matrix &mx)
    {
        return sizeof(T) == 2 && (mx.cols & 1) == 0 && (reinterpret_cast<uintptr_t>(static_cast<T *>(o.ptr) + mx.off) & 3u) == 0;
    }
    // the piece at (m, n); rows, cols: what of the matrix begins there
    __device__ __forceinline__ void fetch(const OutputArgs &o, const Matrix &mx, int lane, int m, int n, int rows, int cols)
    {
        if (!o.update) return;
        const T *at = static_cast<const T *>(o.ptr) + mx.off + (int64_t)m * mx.cols + n;
        if (quads(mx)) {
            const int c = 4 * (lane & 7);
            const T *d = at + (int64_t)(lane >> 3) * mx.cols + c;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (c < cols && 4 * i + (lane >> 3) < rows) {
                    if constexpr (sizeof(T) == 2) {
                        const uint2 x = *reinterpret_cast<const uint2 *>(d + (int64_t)4 * i * mx.cols);
                        w[2 * i] = x.x; w[2 * i + 1] = x.y;
                    } else {
                        const uint4 x = *reinterpret_cast<const uint4 *>(d + (int64_t)4 * i * mx.cols);
                        w[4 * i] = x.x; w[4 * i + 1] = x.y; w[4 * i + 2] = x.z; w[4 * i + 3] = x.w;
                    }
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
    // a piece as stage_swizzled leaves it
    __device__ __forceinline__ void finish_quads(const OutputArgs &o, const Matrix &mx, const unsigned char *buf, int lane, int m, int n,
                                                 int rows, int cols)
    {
        const float f = 1.0f / (kGramScale * mx.sx), k = o.update ? -o.step * mx.scale * f : f;
        const int c = 4 * (lane & 7);
        T *d = static_cast<T *>(o.ptr) + mx.off + (int64_t)m * mx.cols + n + (int64_t)(lane >> 3) * mx.cols + c;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = 4 * i + (lane >> 3);
            const float4 q = *reinterpret_cast<const float4 *>(buf + r * 128 + (((lane & 7) ^ (r & 7)) << 4));
            float x[4] = {q.x * k, q.y * k, q.z * k, q.w * k};
            if (o.update) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    x[e] = __fmaf_rn(o.decay, sizeof(T) == 4 ? entry(w[4 * i + e]) : entry(w[2 * i + (e >> 1)] >> (16 * (e & 1))), x[e]);
            }
            if (r < rows && c < cols)
                *reinterpret_cast<Quad *>(d + (int64_t)4 * i * mx.cols) = Quad{{from_f<T>(x[0]), from_f<T>(x[1]), from_f<T>(x[2]), from_f<T>(x[3])}};
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

// A tile of the run as the roles need it.  The first kTable ones are looked up before the loops: in them a look-up, two
// dependent loads that miss L1 behind the tiles' own traffic, took longer than a stage.
struct Seen {
    int32_t matrix, m0, n0, M, N, K, k0, k1;
    uint16_t part, parts;
    uint16_t a_map, b_map;
    int32_t slot;
    bool a_mn, b_mn, a_sym, b_sym;
};
static_assert(sizeof(Seen) == 48, "table");

// Stages that take a tile once through its contraction (of products of halves, several follow one another).
template <int PHASE> __device__ __forceinline__ int stages_of_a_product(const Seen &s)
{
    return PHASE == kGram ? s.k1 : min((int)s.k1, (s.K + KS - 1) / KS);
}

// T: the type of the last step's result (PHASE kLast).  LOW: the plan has matrices whose A has a low half (kGram, kPoly);
// without, the code for them is left out of a kernel whose launches are short.
template <int PHASE, int CG, typename T = float, bool LOW = false>
__global__ void __launch_bounds__(Shape<CG>::THREADS, 1) product_kernel(const __grid_constant__ ProductParams prm)
{
    using S = Shape<CG>;
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    unsigned char *staging = smem + (size_t)S::STAGES * S::STAGE;
    Seen *table = reinterpret_cast<Seen *>(staging + S::NEPI * kStaging);
    uint64_t *bars = reinterpret_cast<uint64_t *>(table + kTable);
    uint64_t *full = bars, *empty = full + S::STAGES, *d_full = empty + S::STAGES, *d_empty = d_full + 2;
    uint64_t *fetched = d_empty + 2;         // [NEPI] what a warp's epilogue reads has landed
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(fetched + S::NEPI);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = CG == 2 ? (int)cluster_rank() : 0;
    launch_dependents();
    if (threadIdx.x == 0) {
        for (int i = 0; i < S::STAGES; ++i) { mbar_init(full + i, 1); mbar_init(empty + i, 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(d_full + i, 1); mbar_init(d_empty + i, CG * S::NEPI); }
        for (int i = 0; i < S::NEPI; ++i) mbar_init(fetched + i, 1);
        *abort_flag = 0;
        const_cast<int *>(abort_flag)[2] = prm.wait_kcycles;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc<CG>(tmem_slot, S::TMEM);
    // this CTA's (pair's) run of tiles; the plan's tables do not change, so they are read before the wait for the last launch
    const Tile *tiles = prm.dev.run[PHASE].tiles;
    const int t_begin = prm.dev.run[PHASE].start[blockIdx.x / CG], t_end = prm.dev.run[PHASE].start[blockIdx.x / CG + 1];
    auto look_up = [&](int t) {
        const Tile tile = tiles[t];
        const Work w = work_of<PHASE>(prm.dev.mats[tile.matrix], prm.step);
        Seen s;
        s.matrix = tile.matrix; s.m0 = tile.tm * 128 * CG; s.n0 = tile.tn * S::BN;
        s.M = w.M; s.N = w.N; s.K = w.K; s.k0 = tile.k0; s.k1 = tile.k1;
        s.part = (uint16_t)tile.part; s.parts = (uint16_t)tile.parts; s.slot = tile.slot;
        s.a_map = (uint16_t)w.a_map; s.b_map = (uint16_t)w.b_map;
        s.a_mn = w.a_mn; s.b_mn = w.b_mn; s.a_sym = w.a_sym; s.b_sym = w.b_sym;
        return s;
    };
    if ((int)threadIdx.x < min(kTable, t_end - t_begin)) table[threadIdx.x] = look_up(t_begin + threadIdx.x);
    auto seen = [&](int t) { return t - t_begin < kTable ? table[t - t_begin] : look_up(t); };
    tc_fence_before();
    if (CG == 2) cluster_sync(); else __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    bool failed = false;

    if (warp == 0) {
        if (lane == 0) {
            Seen l = seen(t_begin);
            const CUtensorMap *maps = prm.dev.maps + (size_t)l.matrix * kMaps;
            asm volatile("prefetch.tensormap [%0];" ::"l"(maps + l.a_map));
            asm volatile("prefetch.tensormap [%0];" ::"l"(maps + l.b_map));
            grid_dependency_wait();          // what the previous launch wrote is visible from here on
            fence_proxy_async_global();      // and read by TMA, plain stores included
            uint32_t c = 0, s = 0, phase = 1;
            for (int t = t_begin; t < t_end && !failed; ++t) {
                const Seen next = seen(min(t + 1, t_end - 1));
                const CUtensorMap *maps = prm.dev.maps + (size_t)l.matrix * kMaps;
                // a pair's columns are split in halves of a multiple of 8 (the last tile's may be narrow)
                const int half_n = CG == 2 ? min(S::BN, (l.N - l.n0 + 15) / 16 * 16) / 2 : 0;
                const int m0 = l.m0 + 128 * rank, n0 = l.n0 + half_n * rank;
                // steps of the contraction left of the diagonal's block of a symmetric operand's rows
                const int a_left = l.a_sym ? l.m0 / S::BLOCK * S::BLOCK : 0, b_left = l.b_sym ? l.n0 / S::BLOCK * S::BLOCK : 0;
                const int per = stages_of_a_product<PHASE>(l);
                for (int first = 0, term = 0; first < l.k1 && !failed; first += per, ++term) {      // products of halves
                    const CUtensorMap *map_a = maps + l.a_map, *map_b = maps + l.b_map;
                    if (PHASE == kPoly && term > 0) { if (term == 1) map_b = maps + kGramLoMap; else map_a = maps + kGramLoMap; }
                    if (PHASE >= kApply && term > 0) { if (l.a_map == kPolyMap) map_a = maps + kPolyLoMap; else map_b = maps + kPolyLoMap; }
                    for (int st = first > 0 ? first : l.k0; st < first + per; st += S::PER_STAGE, ++c) {
                        if (!mbar_poll(empty + s, phase, abort_flag)) { failed = true; break; }
                        unsigned char *dst = smem + s * S::STAGE;
                        uint64_t *here = full + s;
                        if (++s == S::STAGES) { s = 0; phase ^= 1; }
                        if (prm.test_drop && blockIdx.x == 0 && c == 0) continue;   // test hook: this stage never arrives
                        const int blocks = min(S::PER_STAGE, first + per - st);
                        if (rank == 0) mbar_arrive_expect_tx(here, CG * S::BYTES * blocks);
                        const uint32_t bar = CG == 2 ? in_leader(here) : 0;
#pragma unroll
                        for (int j = 0; j < S::PER_STAGE; ++j) {
                            if (j >= blocks) break;
                            const int k = (st + j - first) * KS;
                            auto load = [&](unsigned char *to, const CUtensorMap *map, bool mn, int at) {
                                if (CG == 2) tma_load_2d_pair(to, map, mn ? at : k, mn ? k : at, bar);
                                else tma_load_2d(to, map, mn ? at : k, mn ? k : at, here);
                            };
#pragma unroll
                            for (int i = 0; i < 2; ++i) load(dst + j * S::BYTES + i * BOX, map_a, l.a_mn || k < a_left, m0 + 64 * i);
#pragma unroll
                            for (int i = 0; i < S::NB; ++i)
                                load(dst + j * S::BYTES + S::A_BYTES + i * BOX, map_b, l.b_mn || k < b_left, n0 + 64 * i);
                        }
                    }
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
        // one lane goes through the whole loop: electing it and bringing the warp together again costs 180 clocks a stage
        if (rank == 0 && elect_one()) {
            uint32_t s = 0, phase = 0, u = 0;
            const uint32_t base0 = smem_u32(smem);
            for (int t = t_begin; t < t_end && !failed; ++t, ++u) {
                const Seen w = seen(t);
                const uint32_t buf = u & 1, d = tmem + buf * S::BN;
                const int n = min(S::BN, (w.N - w.n0 + 15) / 16 * 16);
                const int a_left = w.a_sym ? w.m0 / S::BLOCK * S::BLOCK : 0, b_left = w.b_sym ? w.n0 / S::BLOCK * S::BLOCK : 0;
                if (!mbar_poll(d_empty + buf, ((u >> 1) & 1) ^ 1, abort_flag)) { failed = true; break; }
                tc_fence_after();
                const int per = stages_of_a_product<PHASE>(w);
                for (int first = 0; first < w.k1 && !failed; first += per) {
                    for (int st = first > 0 ? first : w.k0; st < first + per; st += S::PER_STAGE) {
                        if (!mbar_poll(full + s, phase, abort_flag)) { failed = true; break; }
                        tc_fence_after();
#pragma unroll
                        for (int j = 0; j < S::PER_STAGE; ++j) {
                            const int k0 = (st + j - first) * KS;
                            if (j > 0 && st + j >= first + per) break;
                            const uint32_t base = base0 + s * S::STAGE + j * S::BYTES;
                            const bool a_mn = w.a_mn || k0 < a_left, b_mn = w.b_mn || k0 < b_left;
                            const uint32_t idesc = make_idesc_f16(128 * CG, n, a_mn, b_mn);
                            const uint64_t da = a_mn ? make_mn_desc(base, BOX) : make_b_desc(base);
                            const uint64_t db = b_mn ? make_mn_desc(base + S::A_BYTES, BOX) : make_b_desc(base + S::A_BYTES);
                            // 16 steps of the contraction: 32 bytes of a K-major row, 16 rows of 128 bytes of an MN-major box
                            const uint32_t ia = a_mn ? 16 * 128 / 16 : 2, ib = b_mn ? 16 * 128 / 16 : 2;
                            const int n_mma = min(4, (w.K - k0 + 15) / 16);
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                if (k < n_mma) tc_mma_f16<CG>(d, da + k * ia, db + k * ib, idesc, st + j > w.k0 || k > 0);
                        }
                        if (CG == 2) tc_commit_pair(empty + s); else tc_commit(empty + s);
                        if (first + per >= w.k1 && st + S::PER_STAGE >= w.k1) { if (CG == 2) tc_commit_pair(d_full + buf); else tc_commit(d_full + buf); }
                        if (++s == S::STAGES) { s = 0; phase ^= 1; }
                    }
                }
            }
        }
        failed = __any_sync(0xffffffffu, failed);
    } else {
        const int q = warp & 3, half = (warp - 2) >> 2;
        const uint32_t lane_base = (uint32_t)(32 * q) << 16;
        unsigned char *mine = staging + (warp - 2) * kStaging;
        constexpr int COLS = S::BN / (S::NEPI / 4), PIECES = COLS / 64;      // of a warp
        constexpr bool FETCH = PHASE == kPoly || PHASE == kApply;
        const bool write_lo = PHASE == kApply && prm.step + 1 < kExactSteps;      // (every step of this phase reads them)
        // What the epilogue reads besides the accumulator is on its way before the tile's MMAs are done: A or X's low halves come
        // into the staging areas by TMA, where the results take their place; the weights a piece ahead.
        auto fetch = [&](const Seen &at) {
            if (lane == 0) {
                mbar_arrive_expect_tx(fetched + warp - 2, PIECES * 4096);
#pragma unroll
                for (int p = 0; p < PIECES; ++p)
                    tma_load_2d(mine + p * 4096, prm.dev.maps + (size_t)at.matrix * kMaps + (PHASE == kPoly ? kGramOut : kLoOut),
                                at.n0 + half * COLS + 64 * p, at.m0 + 128 * rank + 32 * q, fetched + warp - 2);
            }
        };
        // A's low halves, a lane's row of a piece, by plain loads a piece ahead (short sides only; rows of ldr entries, a multiple of 32)
        uint4 lows[8];
        auto fetch_lows = [&](const Seen &at, int n) {
            const Matrix &m = prm.dev.mats[at.matrix];
            const int row = at.m0 + 128 * rank + 32 * q + lane;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                lows[j] = make_uint4(0, 0, 0, 0);
                if (m.split > 0 && row < at.M && n + 8 * j < m.ldr) lows[j] = *reinterpret_cast<const uint4 *>(m.gram_lo + (int64_t)row * m.ldr + n + 8 * j);
            }
        };
        Weights<T> weights;
        auto fetch_weights = [&](const Seen &at, int n) {
            const int m0 = at.m0 + 128 * rank + 32 * q;
            weights.fetch(prm.out, prm.dev.mats[at.matrix], lane, m0, n, max(0, min(32, at.M - m0)), max(0, min(32, at.N - n)));
        };
        Seen here = seen(t_begin);
        grid_dependency_wait();      // (before anything that another launch writes is read, or written)
        if (FETCH) {
            if (PHASE == kApply) fence_proxy_async_global();      // (X's first low halves were written by plain stores)
            fetch(here);
        }
        if (PHASE == kPoly && LOW) fetch_lows(here, here.n0 + half * COLS);
        if (PHASE == kLast) fetch_weights(here, here.n0 + half * COLS);
        uint32_t u = 0, stores = 0;
        for (int t = t_begin; t < t_end; ++t, ++u) {
            const Seen next = seen(min(t + 1, t_end - 1));
            const Matrix &mx = prm.dev.mats[here.matrix];
            const int m0 = here.m0 + 128 * rank + 32 * q, c0 = here.n0 + half * COLS;      // first row and column of this warp's pieces
            const int rows = min(32, here.M - m0);
            const CUtensorMap *maps = prm.dev.maps + (size_t)here.matrix * kMaps;
            const uint32_t ab = u & 1;
            const float sx = mx.sx;           // (read here, while the MMAs run)
            const bool low = LOW && mx.split > 0;
            bool ok = mbar_poll(d_full + ab, (u >> 1) & 1, abort_flag);
            if (!__all_sync(0xffffffffu, ok)) { failed = true; break; }
            tc_fence_after();
            uint32_t new_lo[PIECES][32];
            auto read_accumulator = [&](int p, bool last, float (&v)[2][32]) {
                tmem_ld32_wait(tmem + lane_base + ab * S::BN + half * COLS + p * 64, v[0]);
                tmem_ld32_wait(tmem + lane_base + ab * S::BN + half * COLS + p * 64 + 32, v[1]);
                if (last) {                  // the accumulator is free
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) { if (CG == 2) mbar_arrive_cluster(in_leader(d_empty + ab)); else mbar_arrive(d_empty + ab); }
                }
            };
            const int parts = PHASE == kGram ? here.parts : 1;
#pragma unroll
            for (int p_ = 0; p_ < PIECES; ++p_) {
                // (parts take their pieces in different orders, so that the last to bring one is not the last for all)
                const int p = PHASE == kGram && PIECES == 2 ? p_ ^ (here.part & 1) : p_;
                const int n0 = c0 + p * 64;
                const bool live = rows > 0 && n0 < here.N;
                float v[2][32];
                read_accumulator(p, p_ == PIECES - 1, v);
                if (PHASE == kGram && parts > 1) {
                    if (!live) continue;
                    // a part of a contraction: the piece goes to scratch, and whoever brings its last part adds them up
                    constexpr int PER_CTA = 4 * S::BN / 64, PER_PART = CG * PER_CTA;      // pieces
                    const int piece = here.slot + rank * PER_CTA + (q * (S::NEPI / 4) + half) * PIECES + p;
                    float4 *scratch = reinterpret_cast<float4 *>(prm.dev.parts) + (int64_t)piece * 512 + lane;
                    float4 *own = scratch + (int64_t)here.part * PER_PART * 512;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float *x = &v[i >> 3][4 * (i & 7)];
                        __stcg(own + 32 * i, make_float4(x[0], x[1], x[2], x[3]));
                    }
                    __threadfence();
                    __syncwarp();
                    int arrived = 0;
                    if (lane == 0) arrived = atomicAdd(prm.dev.tickets + piece, 1);
                    if (__shfl_sync(0xffffffffu, arrived, 0) != parts - 1) continue;
                    if (lane == 0) prm.dev.tickets[piece] = 0;
                    __threadfence();
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[0][i] = v[1][i] = 0.0f;
                    for (int part = 0; part < parts; ++part) {
                        const float4 *from = scratch + (int64_t)part * PER_PART * 512;
                        float4 x[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) x[i] = __ldcg(from + 32 * i);
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            float *y = &v[i >> 3][4 * (i & 7)];
                            y[0] += x[i].x; y[1] += x[i].y; y[2] += x[i].z; y[3] += x[i].w;
                        }
                    }
                }
                if (PHASE == kLast) {
                    const bool quads = Weights<T>::quads(mx);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int n = n0 + 32 * h, cols = min(32, here.N - n);
                        if (live && cols > 0) {
                            if (quads) {
                                __syncwarp();
                                stage_swizzled(mine, lane, v[h]);
                                __syncwarp();
                                weights.finish_quads(prm.out, mx, mine, lane, m0, n, rows, cols);
                            } else {
                                stage_piece(reinterpret_cast<float *>(mine), lane, v[h]);
                                weights.finish(prm.out, mx, reinterpret_cast<const float *>(mine), lane, m0, n, rows, cols);
                            }
                        }
                        const int after = p * 64 + h * 32 + 32;
                        if (after < COLS) fetch_weights(here, c0 + after);
                        else if (t + 1 < t_end) fetch_weights(next, next.n0 + half * COLS);
                    }
                    continue;
                }
                auto store = [&](unsigned char *from, int map, int n) {      // a staged piece, by one lane
                    fence_proxy_async();
                    __syncwarp();
                    if (lane == 0) {
                        tma_store_2d(maps + map, n, m0, from);
                        bulk_commit_group();
                    }
                };
                auto room = [&]() {      // one of the warp's two staging areas, once its last store has read it
                    if (lane == 0) bulk_wait_group_read<1>();
                    __syncwarp();
                    return mine + (stores++ & 1) * 4096;
                };
                if (FETCH && p == 0) {
                    ok = mbar_poll(fetched + warp - 2, u & 1, abort_flag);
                    if (!__all_sync(0xffffffffu, ok)) { failed = true; break; }
                }
                auto fetch_next = [&]() {      // once the tile's stores have read their areas
                    if (t + 1 == t_end) return;
                    if (lane == 0) bulk_wait_group_read<0>();
                    __syncwarp();
                    fetch(next);
                };
                // the low halves of what a lane holds of a piece, as it is staged
                auto stage_low = [&](unsigned char *to) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        uint32_t w[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float a = v[j >> 2][8 * (j & 3) + 2 * e], b = v[j >> 2][8 * (j & 3) + 2 * e + 1];
                            const float2 r = unpack_half2(pack2<__half>(a, b));
                            w[e] = pack2<__half>(a - r.x, b - r.y);
                        }
                        *reinterpret_cast<uint4 *>(to + lane * 128 + ((j ^ (lane & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                };
                if (PHASE == kApply) {       // X' = P X_hi + a X_lo
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint4 l = *reinterpret_cast<const uint4 *>(mine + p * 4096 + lane * 128 + (((4 * h + j) ^ (lane & 7)) << 4));
                            const uint32_t w[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const int i = 8 * j + 2 * e;
                                const float2 x = unpack_half2(w[e]);
                                v[h][i] = __fmaf_rn(kA, x.x, v[h][i] * (1.0f / kGramScale));
                                v[h][i + 1] = __fmaf_rn(kA, x.y, v[h][i + 1] * (1.0f / kGramScale));
                            }
                        }
                    if (live) {
                        // (in place: a lane has read its row of the piece)
                        unsigned char *to = mine + p * 4096;
                        stage_swizzled16<__half>(to, lane, v[0], v[1]);
                        store(to, kX0Out + ((prm.step + 1) & 1), n0);
                    }
                    if (write_lo) {
#pragma unroll
                        for (int h = 0; h < 2; ++h)
#pragma unroll
                            for (int i = 0; i < 32; i += 2) {
                                const float2 x = unpack_half2(pack2<__half>(v[h][i], v[h][i + 1]));
                                new_lo[p][16 * h + i / 2] = pack2<__half>(v[h][i] - x.x, v[h][i + 1] - x.y);
                            }
                    }
                    if (p < PIECES - 1) continue;
                    // the pieces' new low halves, each once X's store has read its area
                    if (write_lo) {
#pragma unroll
                        for (int r = 0; r < PIECES; ++r) {
                            if (rows <= 0 || c0 + 64 * r >= here.N) break;
                            // (the store after the one of this area may still be reading)
                            if (lane == 0) { if (PIECES == 2 && c0 + 64 < here.N) bulk_wait_group_read<1>(); else bulk_wait_group_read<0>(); }
                            __syncwarp();
#pragma unroll
                            for (int j = 0; j < 8; ++j)
                                *reinterpret_cast<uint4 *>(mine + r * 4096 + lane * 128 + ((j ^ (lane & 7)) << 4)) =
                                    make_uint4(new_lo[r][4 * j], new_lo[r][4 * j + 1], new_lo[r][4 * j + 2], new_lo[r][4 * j + 3]);
                            store(mine + r * 4096, kLoOut, c0 + 64 * r);
                        }
                    }
                    fetch_next();
                    continue;
                }
                if (PHASE == kPoly) {        // P = a I + b A + c A^2
                    if (live) {
                        unsigned char *to = mine + p * 4096;
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const uint4 hi = *reinterpret_cast<const uint4 *>(to + lane * 128 + ((j ^ (lane & 7)) << 4));
                            const uint32_t w[4] = {hi.x, hi.y, hi.z, hi.w};
                            const uint32_t l[4] = {lows[j].x, lows[j].y, lows[j].z, lows[j].w};
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                const float2 x = unpack_half2(w[e >> 1]);
                                float a = e & 1 ? x.y : x.x;
                                if (LOW) {
                                    const float2 y = unpack_half2(l[e >> 1]);
                                    a += e & 1 ? y.y : y.x;
                                }
                                float &r = v[j >> 2][8 * (j & 3) + e];
                                r = __fmaf_rn(kB, a, r * (kC / kGramScale));
                                if (n0 + 8 * j + e == m0 + lane) r += kA * kGramScale;
                            }
                        }
                        if (LOW && p + 1 < PIECES) fetch_lows(here, n0 + 64);
                        stage_swizzled16<__half>(to, lane, v[0], v[1]);       // (in place: a lane has read its row of the piece)
                        store(to, kPolyOut, n0);
                        // P's low halves: only of short sides that the first piece holds, so that the other area is free
                        static_assert(kSplitApply <= 64, "a piece");
                        if (LOW && mx.split > 1) {
                            stage_low(mine + 4096);
                            store(mine + 4096, kPolyLoOut, n0);
                        }
                    }
                    if (p == PIECES - 1) {
                        if (LOW && t + 1 < t_end) fetch_lows(next, next.n0 + half * COLS);
                        fetch_next();
                    }
                    continue;
                }
                if (PHASE == kGram && live) {       // A = X X^T
                    const float f = kGramScale / (sx * sx);
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[h][i] *= f;
                    unsigned char *to = room();
                    stage_swizzled16<__half>(to, lane, v[0], v[1]);
                    store(to, kGramOut, n0);
                    if (LOW && low) {
                        to = room();
                        stage_low(to);
                        store(to, kGramLoOut, n0);
                    }
                }
            }
            if (failed) break;
            here = next;
        }
        if (lane == 0) bulk_wait_group_all();
        if (FETCH && failed)         // what is still under way gets a bounded chance to land before the CTA exits
            for (int it = 0; it < 100000 && !mbar_try_wait(fetched + warp - 2, u & 1); ++it) {}
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

template <int PHASE, typename T = float, bool LOW = false>
cudaError_t launch_tiling(cudaStream_t st, const ProductParams &prm, int runs)
{
    return prm.dev.pair ? launch_chained<product_kernel<PHASE, 2, T, LOW>>(prm, 2 * runs, Shape<2>::THREADS, Shape<2>::SMEM, 2, st)
                        : launch_chained<product_kernel<PHASE, 1, T, LOW>>(prm, runs, Shape<1>::THREADS, Shape<1>::SMEM, 1, st);
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
    static_assert(kExactSteps == kSteps - 1, "every product with an X that is not the last result reads its low half");
    ProductParams prm;
    prm.dev = dev;
    prm.out = out ? *out : OutputArgs{};
    prm.step = step;
    prm.error_word = error_word;
    prm.wait_kcycles = wait_kcycles > 0 ? wait_kcycles : WAIT_KCYCLES_DEFAULT;
    prm.test_drop = test_drop;
    const int runs = dev.run[phase].runs;
    if (phase == kGram) return dev.split > 0 ? launch_tiling<kGram, float, true>(st, prm, runs) : launch_tiling<kGram>(st, prm, runs);
    if (phase == kPoly) return dev.split > 0 ? launch_tiling<kPoly, float, true>(st, prm, runs) : launch_tiling<kPoly>(st, prm, runs);
    if (step < kSteps - 1) return launch_tiling<kApply>(st, prm, runs);
    if (out->dtype == GVQ_F32) return launch_tiling<kLast, float>(st, prm, runs);
    if (out->dtype == GVQ_BF16) return launch_tiling<kLast, __nv_bfloat16>(st, prm, runs);
    return launch_tiling<kLast, __half>(st, prm, runs);
}

}  // namespace ortho
}  // namespace gvq
