// The orthogonalised update of matrices that fit one SM, or the few of a cluster, a whole update in one launch.
//
// A cluster of `parts` CTAs has a matrix, each a span of its long side.  All but A's sum stays in a CTA: the parts' sums meet in
// shared memory (of the cluster, read by all, each in an order of its own that does not change), and every CTA makes P for itself.
//
// For a small matrix the products take a microsecond and the fifteen launches of ortho.cu 3.3 us each.  Here X stays in
// shared memory from the gradient to the weights: as a sum of two halves (ortho.cu has the reasons), transposed, the long
// side as rows: 64 entries of the short side are a row of 128 bytes (with the 128-byte swizzle), a second array holds
// the next 64.  Then X^T is the K-major operand of X^T P and the MN-major ones of A = X X^T, nothing moves between the products
// but the accumulators, and a thread that reads one of their rows writes it back as a row:
//     A      D[R x R]   = sum over the long side             -> A as a sum of two halves, shared memory; in fp32 in registers
//     A^2    D[R x R]   = A_hi A_hi + A_hi A_lo + A_lo A_hi  -> P = a I + b A + c D as a sum of two halves in A's place
//     X^T P  D[128 x R] for every 128 of the long side       -> X = X_hi P + a X_lo in place
// A and P rounded to one half would leave errors of 2e-3 to 4e-3 of the result where the short side is short (their entries
// are then few and of like size, and the steps amplify what the singular values are off by); with A's low half, and P's up
// to kSplitApply, it is what ortho.cu's header lists, at most 2.6e-3 for gradients of random factors.  Where the long side has 64
// entries or fewer too, what X loses does not average out either; its low half takes part in every product, and about 1e-4 is left.
// R is the short side's room, 64 or 128.  The unused rows and columns of X are zeros and stay zeros; an MMA's 128 rows
// may run on into the next array, and those rows of the accumulator are not read.
//
// What bounds it is the chain of its steps (MMAs, a wait, accumulator to shared memory, a fence, fifteen times, 2.5 us a
// step at 64 x 64), beyond that the conversions of X, an entry a lane, and between CTAs the join of A (1 us a step with four
// and a short side of 64).
#include <algorithm>

#include "ortho.h"
#include "row32.cuh"
#include "sm100_ptx.cuh"

namespace gvq {
namespace ortho {
namespace {

using namespace ptx;

constexpr int NTHREADS = 512, NPART = NTHREADS / 128;     // warps that share a quarter of the accumulator's rows

struct SmallParams {
    const Matrix *mats;
    ElementArgs in;
    OutputArgs out;
    int mode;                // of the momentum, as in ortho.cu
    int parts, span;         // CTAs of a matrix; entries of the long side each has, a multiple of 64
    int32_t *error_word;
    int wait_kcycles, test_drop;
};

// Byte of entry (i of the long side, j of the short side) in an array of `half`-byte columns of 64 entries.
__device__ __forceinline__ uint32_t place(int i, int j, uint32_t half)
{
    return (uint32_t)(j >> 6) * half + i * 128 + ((((j & 63) >> 3) ^ (i & 7)) << 4) + (j & 7) * 2;
}

template <int R, typename T>
__global__ void __launch_bounds__(NTHREADS, 1) ortho_small_kernel(const SmallParams prm)
{
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    __shared__ float sums[NTHREADS / 32];
    __shared__ uint64_t bar;
    __shared__ uint32_t tmem_slot;
    __shared__ int flags[4];                 // abort flag, -, limit of the waits
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    __shared__ float shared_sum;             // of the squares, for the cluster
    __shared__ float shared_ok;
    const Matrix &mx = prm.mats[blockIdx.x / prm.parts];
    // this CTA's span of the long side (it may be empty: zeros, which add nothing)
    const int part_of = blockIdx.x % prm.parts, first = min(part_of * prm.span, mx.c), mine = min(prm.span, mx.c - first);
    const int my_rows = mx.tall ? mine : mx.rows, my_cols = mx.tall ? mx.cols : mine;
    const int64_t off = mx.off + (mx.tall ? (int64_t)first * mx.cols : first);
    const int rows = max(64, (mine + 63) & ~63), tiles = (rows + 127) / 128;
    constexpr uint32_t SQUARE_HALF = R * 128, SQUARE = R / 64 * SQUARE_HALF;
    const uint32_t half = rows * 128, array = R / 64 * half;
    unsigned char *sq = smem, *sq_lo = sq + SQUARE, *hi = sq_lo + SQUARE, *lo = hi + array;     // sq: A, then P
    const bool full = rows == 64;            // X's low half in every product
    const bool split_p = full || mx.r <= kSplitApply;

    launch_dependents();
    if (threadIdx.x == 0) {
        mbar_init(&bar, 1);
        flags[0] = 0;
        flags[2] = prm.wait_kcycles;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) tmem_alloc<1>(&tmem_slot, 512);
    for (uint32_t i = threadIdx.x; i < 2 * array / 16; i += NTHREADS) reinterpret_cast<uint4 *>(hi)[i] = make_uint4(0, 0, 0, 0);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    grid_dependency_wait();

    // u = g + beta * momentum, its bits in the two arrays until the norm is known
    const int total = my_rows * my_cols;
    const float *g = prm.in.g + off;
    float *mo = prm.mode ? prm.in.momentum + off : nullptr;
    float sum = 0.0f;
    const uint64_t by_cols = my_cols == mx.cols ? mx.by_cols : ((uint64_t)1 << 62) / (uint64_t)max(1, my_cols) + 1;
    int from = 0;                            // where entry e of this CTA's is in memory, once at(e) has been asked for
    auto at = [&](int e) {
        const int row = (int)__umul64hi((uint64_t)e << 2, by_cols), col = e - row * my_cols;
        from = row * mx.cols + col;
        return mx.tall ? place(row, col, half) : place(col, row, half);
    };
    auto direct = [&](float u, float &m) {
        if (prm.mode) {
            m = __fmaf_rn(prm.in.beta, m, u);
            u = prm.mode == 1 ? m : __fmaf_rn(prm.in.beta, m, u);
        }
        sum = __fmaf_rn(u, u, sum);
        return __float_as_uint(u);
    };
    // Four entries of a row at a time where rows hold whole quads.  A tall matrix' row is one here too.  Of a wide one a warp
    // takes 8 rows x 32 columns (128 bytes of each), a lane two rows x 4 columns; the two rows' entries of a column make a word
    // here, and the lanes take their four columns in orders that keep a warp's words in different banks.
    const bool quads = (mx.cols & 3) == 0;
    const int tall_quads = quads && mx.tall ? total / 4 : 0;
    const int strips = (my_rows + 7) / 8, wide_tiles = quads && !mx.tall ? strips * ((my_cols + 31) / 32) : 0;
    const int lane_row = 2 * (lane >> 3), lane_col = 4 * (lane & 7), turn = (lane & 7) >> 1;
    auto turned = [&](uint32_t (&w)[4]) {      // w[c] = w[(c + turn) % 4]
        if (turn & 1) { const uint32_t x = w[0]; w[0] = w[1]; w[1] = w[2]; w[2] = w[3]; w[3] = x; }
        if (turn & 2) { uint32_t x = w[0]; w[0] = w[2]; w[2] = x; x = w[1]; w[1] = w[3]; w[3] = x; }
    };
    // Loads are unconditional (entry 0 stands in for what is outside, the gradient for a momentum that is not there), so that a
    // batch's are issued together, before its first store.
    const float *mo_or_g = prm.mode ? mo : g;
    auto load4 = [](const float *from, int e, bool in) { return *reinterpret_cast<const float4 *>(from + (in ? e : 0)); };
    constexpr int BATCH = 6, TILES = 3;
    for (int e0 = threadIdx.x; e0 < tall_quads; e0 += BATCH * NTHREADS) {
        float4 x[BATCH], m[BATCH];
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int e = e0 + i * NTHREADS;
            x[i] = load4(g, 4 * e, e < tall_quads);
            m[i] = load4(mo_or_g, 4 * e, e < tall_quads);
        }
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int e = e0 + i * NTHREADS;
            if (e >= tall_quads) break;
            const uint32_t b[4] = {direct(x[i].x, m[i].x), direct(x[i].y, m[i].y), direct(x[i].z, m[i].z), direct(x[i].w, m[i].w)};
            if (prm.mode) reinterpret_cast<float4 *>(mo)[e] = m[i];
            const uint32_t p = at(4 * e);
            *reinterpret_cast<uint2 *>(hi + p) = make_uint2(__byte_perm(b[0], b[1], 0x7632), __byte_perm(b[2], b[3], 0x7632));
            *reinterpret_cast<uint2 *>(lo + p) = make_uint2(__byte_perm(b[0], b[1], 0x5410), __byte_perm(b[2], b[3], 0x5410));
        }
    }
    auto tile_at = [&](int w, int &row, int &col) {
        row = 8 * (w % strips) + lane_row;
        col = 32 * (w / strips) + lane_col;
        return w < wide_tiles && row < my_rows && col < my_cols;
    };
    for (int w0 = warp; w0 < wide_tiles; w0 += TILES * (NTHREADS / 32)) {
        float4 x[TILES][2], m[TILES][2];
#pragma unroll
        for (int i = 0; i < TILES; ++i) {
            int row, col;
            const bool in = tile_at(w0 + i * (NTHREADS / 32), row, col);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int e = (row + h) * mx.cols + col;
                x[i][h] = load4(g, e, in && row + h < my_rows);
                m[i][h] = load4(mo_or_g, e, in && row + h < my_rows);
            }
        }
#pragma unroll
        for (int i = 0; i < TILES; ++i) {
            int row, col;
            if (!tile_at(w0 + i * (NTHREADS / 32), row, col)) continue;
            uint32_t b[2][4];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (row + h >= my_rows) x[i][h] = make_float4(0.f, 0.f, 0.f, 0.f), m[i][h] = x[i][h];
                b[h][0] = direct(x[i][h].x, m[i][h].x); b[h][1] = direct(x[i][h].y, m[i][h].y);
                b[h][2] = direct(x[i][h].z, m[i][h].z); b[h][3] = direct(x[i][h].w, m[i][h].w);
                if (prm.mode && row + h < my_rows) *reinterpret_cast<float4 *>(mo + (row + h) * mx.cols + col) = m[i][h];
            }
            turned(b[0]);
            turned(b[1]);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint32_t p = place(col + ((c + turn) & 3), row, half);
                *reinterpret_cast<uint32_t *>(hi + p) = __byte_perm(b[0][c], b[1][c], 0x7632);
                *reinterpret_cast<uint32_t *>(lo + p) = __byte_perm(b[0][c], b[1][c], 0x5410);
            }
        }
    }
#pragma unroll 8
    for (int e = threadIdx.x; !quads && e < total; e += NTHREADS) {
        const uint32_t p = at(e);
        float m = prm.mode ? mo[from] : 0.0f;
        const uint32_t b = direct(g[from], m);
        if (prm.mode) mo[from] = m;
        *reinterpret_cast<uint16_t *>(hi + p) = (uint16_t)(b >> 16);
        *reinterpret_cast<uint16_t *>(lo + p) = (uint16_t)b;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) sums[warp] = sum;
    __syncthreads();
    sum = 0.0f;
#pragma unroll
    for (int i = 0; i < NTHREADS / 32; ++i) sum += sums[i];
    if (prm.parts > 1) {
        if (threadIdx.x == 0) shared_sum = sum;
        __syncwarp();
        cluster_sync();
        sum = 0.0f;
        for (int p = 0; p < prm.parts; ++p) sum += load_cluster1(cluster_address(smem_u32(&shared_sum), p));
    }
    const float f = mx.sx / (sqrtf(sum) + kEps);
    // X = u / |u|: places do not matter here (zeros stay zeros)
    for (uint32_t i = threadIdx.x; i < array / 16; i += NTHREADS) {
        uint4 h4 = reinterpret_cast<const uint4 *>(hi)[i], l4 = reinterpret_cast<const uint4 *>(lo)[i];
        uint32_t h[4] = {h4.x, h4.y, h4.z, h4.w}, l[4] = {l4.x, l4.y, l4.z, l4.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float a = __uint_as_float(__byte_perm(l[k], h[k], 0x5410)) * f, b = __uint_as_float(__byte_perm(l[k], h[k], 0x7632)) * f;
            h[k] = pack2<__half>(a, b);
            const float2 r = unpack_half2(h[k]);
            l[k] = pack2<__half>(a - r.x, b - r.y);
        }
        reinterpret_cast<uint4 *>(hi)[i] = make_uint4(h[0], h[1], h[2], h[3]);
        reinterpret_cast<uint4 *>(lo)[i] = make_uint4(l[0], l[1], l[2], l[3]);
    }

    const int q = warp & 3, part = warp >> 2, m = 32 * q + lane;       // this thread's row of an accumulator
    const uint32_t lane_base = (uint32_t)(32 * q) << 16;
    const bool live = 32 * q < R;                                       // in a square result (uniform in a warp)
    uint32_t phase = 0;
    bool ok = true;
    // shared memory written so far is seen by the MMAs; the accumulators have been read
    auto hand_over = [&]() {
        fence_proxy_async();
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
    };
    auto wait = [&]() {
        if (warp == 0) ok = ok && mbar_poll(&bar, phase & 1, flags);     // (one warp polls, the others wait at the barrier)
        ++phase;
        ok = __syncthreads_and(ok);
        tc_fence_after();
    };
    // 16 entries of row m of the square operand from column n on
    auto put16 = [&](int n, const float *v) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            uint32_t h[4], l[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float a = v[8 * i + 2 * e], b = v[8 * i + 2 * e + 1];
                h[e] = pack2<__half>(a, b);
                const float2 r = unpack_half2(h[e]);
                l[e] = pack2<__half>(a - r.x, b - r.y);
            }
            const uint32_t p = place(m, n + 8 * i, SQUARE_HALF);
            *reinterpret_cast<uint4 *>(sq + p) = make_uint4(h[0], h[1], h[2], h[3]);
            *reinterpret_cast<uint4 *>(sq_lo + p) = make_uint4(l[0], l[1], l[2], l[3]);
        }
    };
    const uint32_t a_sq = smem_u32(sq), a_sq_lo = smem_u32(sq_lo), a_hi = smem_u32(hi), a_lo = smem_u32(lo);
    // step k of 16 of the short side's contraction in a K-major operand
    auto along = [](uint32_t base, uint32_t half, int k) { return make_b_desc(base + (k >> 2) * half) + 2 * (k & 3); };
    constexpr int SQUARE_PIECES = R / 16 / NPART;      // of 16 columns, of a warp

    for (int step = 0; step < kSteps; ++step) {
        // ---- A
        float gram[SQUARE_PIECES][16];      // this thread's entries of it
        hand_over();
        if (warp == 0) {
            constexpr uint32_t idesc = make_idesc_f16(128, R, true, true);
            if (elect_one()) {
                // 16 rows of X^T a step.  With R = 64 the second 64 rows of the result repeat the first (chunk distance 0).
                const uint64_t a = make_mn_desc(a_hi, R == 128 ? half : 0), b = make_mn_desc(a_hi, half);
                for (int k = 0; k < rows / 16; ++k) tc_mma_f16<1>(tmem, a + k * (16 * 128 / 16), b + k * (16 * 128 / 16), idesc, k != 0);
                if (full) {
                    const uint64_t al = make_mn_desc(a_lo, R == 128 ? half : 0), bl = make_mn_desc(a_lo, half);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        tc_mma_f16<1>(tmem, a + k * (16 * 128 / 16), bl + k * (16 * 128 / 16), idesc, 1);
                        tc_mma_f16<1>(tmem, al + k * (16 * 128 / 16), b + k * (16 * 128 / 16), idesc, 1);
                    }
                }
                // (test hook: without this the wait below runs out and the kernel gives up)
                if (!(prm.test_drop && blockIdx.x == 0 && step == 0)) tc_commit(&bar);
            }
            __syncwarp();
        }
        wait();
        if (prm.parts == 1 && !ok) break;
        if (live)
#pragma unroll
            for (int p = 0; p < SQUARE_PIECES; ++p) tmem_ld16_wait(tmem + lane_base + 16 * (part * SQUARE_PIECES + p), gram[p]);
        if (prm.parts > 1) {
            // The parts' sums, in the place of the square operand (nothing reads it now): words of four columns, rows next to
            // each other.  If one CTA has given up, all do.
            float4 *join = reinterpret_cast<float4 *>(sq);
            if (live)
#pragma unroll
                for (int p = 0; p < SQUARE_PIECES; ++p)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        join[(4 * (part * SQUARE_PIECES + p) + i) * R + m] =
                            make_float4(gram[p][4 * i], gram[p][4 * i + 1], gram[p][4 * i + 2], gram[p][4 * i + 3]);
            if (threadIdx.x == 0) shared_ok = ok ? 1.0f : 0.0f;
            __syncwarp();
            cluster_sync();
            // (each starts from its own, so that they do not all read the same one at a time)
            const uint32_t join_at = smem_u32(join) + m * 16, ok_at = smem_u32(&shared_ok);
            constexpr int AHEAD = 3;
            for (int i0 = 1; i0 < prm.parts; i0 += AHEAD) {
                uint32_t there[AHEAD];
                float fine[AHEAD];
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) {
                    const int c = part_of + min(i0 + i, prm.parts - 1), peer = c < prm.parts ? c : c - prm.parts;
                    there[i] = cluster_address(join_at, peer);
                    fine[i] = load_cluster1(cluster_address(ok_at, peer));
                }
#pragma unroll
                for (int p = 0; p < SQUARE_PIECES; ++p) {
                    float4 x[AHEAD][4];
#pragma unroll
                    for (int i = 0; i < AHEAD; ++i)
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            x[i][k] = live && i0 + i < prm.parts ? load_cluster(there[i] + (4 * (part * SQUARE_PIECES + p) + k) * R * 16)
                                                                 : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                    for (int i = 0; i < AHEAD; ++i)
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            gram[p][4 * k] += x[i][k].x; gram[p][4 * k + 1] += x[i][k].y;
                            gram[p][4 * k + 2] += x[i][k].z; gram[p][4 * k + 3] += x[i][k].w;
                        }
                }
                ok = ok && fine[0] != 0.0f && fine[1] != 0.0f && fine[2] != 0.0f;
            }
            __syncwarp();
            cluster_sync();
            if (!ok) break;
        }
        if (live) {
            const float s = kGramScale / (mx.sx * mx.sx);
#pragma unroll
            for (int p = 0; p < SQUARE_PIECES; ++p) {
                const int n = 16 * (part * SQUARE_PIECES + p);
#pragma unroll
                for (int i = 0; i < 16; ++i) gram[p][i] *= s;
                put16(n, gram[p]);
            }
        }
        // ---- P
        hand_over();
        constexpr uint32_t idesc = make_idesc_f16(128, R, false, false);
        if (warp == 0) {
            if (elect_one()) {
#pragma unroll
                for (int k = 0; k < R / 16; ++k) {
                    const uint64_t h = along(a_sq, SQUARE_HALF, k), l = along(a_sq_lo, SQUARE_HALF, k);
                    tc_mma_f16<1>(tmem, h, h, idesc, k != 0);
                    tc_mma_f16<1>(tmem, h, l, idesc, 1);
                    tc_mma_f16<1>(tmem, l, h, idesc, 1);
                }
                tc_commit(&bar);
            }
            __syncwarp();
        }
        wait();
        if (!ok) {
            if (prm.parts > 1) continue;     // (the others hear of it where the parts meet)
            break;
        }
        if (live) {
#pragma unroll
            for (int p = 0; p < SQUARE_PIECES; ++p) {
                const int n = 16 * (part * SQUARE_PIECES + p);
                float v[16];
                tmem_ld16_wait(tmem + lane_base + n, v);
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    v[i] = __fmaf_rn(kB, gram[p][i], v[i] * (kC / kGramScale)) + (n + i == m ? kA * kGramScale : 0.0f);
                put16(n, v);
            }
        }
        // ---- X^T P, the accumulators of all tiles side by side
        hand_over();
        if (warp == 0) {
            if (elect_one()) {
                for (int t = 0; t < tiles; ++t)
#pragma unroll
                    for (int k = 0; k < R / 16; ++k) {
                        const uint64_t x = along(a_hi + t * (128 * 128), half, k);
                        tc_mma_f16<1>(tmem + R * t, x, along(a_sq, SQUARE_HALF, k), idesc, k != 0);
                        if (split_p) tc_mma_f16<1>(tmem + R * t, x, along(a_sq_lo, SQUARE_HALF, k), idesc, 1);
                    }
                if (full)
#pragma unroll
                    for (int k = 0; k < R / 16; ++k) tc_mma_f16<1>(tmem, along(a_lo, half, k), along(a_sq, SQUARE_HALF, k), idesc, 1);
                tc_commit(&bar);
            }
            __syncwarp();
        }
        wait();
        if (!ok) {
            if (prm.parts > 1) continue;     // (the others hear of it where the parts meet)
            break;
        }
#pragma unroll 1
        for (int p = part; p < tiles * (R / 32); p += NPART) {       // 32 columns at a time
            const int t = p / (R / 32), n = 32 * (p - t * (R / 32)), i = 128 * t + m;
            float v[32];
            tmem_ld32_wait(tmem + lane_base + R * t + n, v);
            if (i >= rows) continue;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint32_t o = place(i, n + 8 * c, half);
                uint4 *l = reinterpret_cast<uint4 *>(lo + o);
                const uint4 old = *l;
                const uint32_t w[4] = {old.x, old.y, old.z, old.w};
                uint32_t nh[4], nl[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float2 x = make_float2(v[8 * c + 2 * e] * (1.0f / kGramScale), v[8 * c + 2 * e + 1] * (1.0f / kGramScale));
                    if (step < kExactSteps && !full) {
                        const float2 a = unpack_half2(w[e]);
                        x.x = __fmaf_rn(kA, a.x, x.x);
                        x.y = __fmaf_rn(kA, a.y, x.y);
                    }
                    nh[e] = pack2<__half>(x.x, x.y);
                    const float2 r = unpack_half2(nh[e]);
                    nl[e] = pack2<__half>(x.x - r.x, x.y - r.y);
                }
                *reinterpret_cast<uint4 *>(hi + o) = make_uint4(nh[0], nh[1], nh[2], nh[3]);
                *l = make_uint4(nl[0], nl[1], nl[2], nl[3]);
            }
        }
    }
    __syncthreads();

    if (ok) {
        // the result, from both halves
        T *out = static_cast<T *>(prm.out.ptr) + off;
        const float k = (prm.out.update ? -prm.out.step * mx.scale : 1.0f) / mx.sx;
        auto entry = [&](uint32_t p) {
            return __half2float(*reinterpret_cast<const __half *>(hi + p)) + __half2float(*reinterpret_cast<const __half *>(lo + p));
        };
        auto back = [&](uint32_t (&w)[4]) {        // undoes turned()
            if (turn & 1) { const uint32_t x = w[3]; w[3] = w[2]; w[2] = w[1]; w[1] = w[0]; w[0] = x; }
            if (turn & 2) { uint32_t x = w[0]; w[0] = w[2]; w[2] = x; x = w[1]; w[1] = w[3]; w[3] = x; }
        };
        struct alignas(4 * sizeof(T)) Quad { T v[4]; };
        auto finish = [&](Quad &o, int i, float x) { o.v[i] = from_f<T>(prm.out.update ? __fmaf_rn(k, x, prm.out.decay * to_f(o.v[i])) : k * x); };
        for (int e0 = threadIdx.x; e0 < tall_quads; e0 += BATCH * NTHREADS) {
            Quad o[BATCH];
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                const int e = e0 + i * NTHREADS;
                if (prm.out.update) o[i] = reinterpret_cast<const Quad *>(out)[e < tall_quads ? e : 0];
            }
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                const int e = e0 + i * NTHREADS;
                if (e >= tall_quads) break;
                const uint32_t p = at(4 * e);
                const uint2 h = *reinterpret_cast<const uint2 *>(hi + p), l = *reinterpret_cast<const uint2 *>(lo + p);
                const float2 h0 = unpack_half2(h.x), h1 = unpack_half2(h.y), l0 = unpack_half2(l.x), l1 = unpack_half2(l.y);
                finish(o[i], 0, h0.x + l0.x);
                finish(o[i], 1, h0.y + l0.y);
                finish(o[i], 2, h1.x + l1.x);
                finish(o[i], 3, h1.y + l1.y);
                reinterpret_cast<Quad *>(out)[e] = o[i];
            }
        }
        for (int w0 = warp; w0 < wide_tiles; w0 += TILES * (NTHREADS / 32)) {
            Quad o[TILES][2];
#pragma unroll
            for (int i = 0; i < TILES; ++i) {
                int row, col;
                const bool in = tile_at(w0 + i * (NTHREADS / 32), row, col);
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    if (prm.out.update) o[i][h] = *reinterpret_cast<const Quad *>(out + (in && row + h < my_rows ? (row + h) * mx.cols + col : 0));
            }
#pragma unroll
            for (int i = 0; i < TILES; ++i) {
                int row, col;
                if (!tile_at(w0 + i * (NTHREADS / 32), row, col)) continue;
                uint32_t x[2][4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const uint32_t p = place(col + ((c + turn) & 3), row, half);
                    const float2 h = unpack_half2(*reinterpret_cast<const uint32_t *>(hi + p)), l = unpack_half2(*reinterpret_cast<const uint32_t *>(lo + p));
                    x[0][c] = __float_as_uint(h.x + l.x);
                    x[1][c] = __float_as_uint(h.y + l.y);
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    back(x[h]);
#pragma unroll
                    for (int c = 0; c < 4; ++c) finish(o[i][h], c, __uint_as_float(x[h][c]));
                }
                *reinterpret_cast<Quad *>(out + row * mx.cols + col) = o[i][0];
                if (row + 1 < my_rows) *reinterpret_cast<Quad *>(out + (row + 1) * mx.cols + col) = o[i][1];
            }
        }
#pragma unroll 8
        for (int e = threadIdx.x; !quads && e < total; e += NTHREADS) {
            const float x = entry(at(e));
            out[from] = from_f<T>(prm.out.update ? __fmaf_rn(k, x, prm.out.decay * to_f(out[from])) : k * x);
        }
    } else if (threadIdx.x == 0) {
        atomicExch(prm.error_word, 100);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 0) tmem_dealloc<1>(tmem, 512);
}

template <int R> size_t small_smem(int blocks) { return (size_t)(R / 64) * 128 * (2 * R + 2 * 64 * blocks) + 1024; }

template <int R, typename T>
cudaError_t launch_as(cudaStream_t st, const SmallParams &prm, int n)
{
    // (the launch helper raises a kernel's limit once: every launch asks for all there is)
    return launch_chained<ortho_small_kernel<R, T>>(prm, n * prm.parts, NTHREADS, kSmallSmem, prm.parts, st);
}
template <int R>
cudaError_t launch_typed(cudaStream_t st, const SmallParams &prm, int n)
{
    if (prm.out.dtype == GVQ_F32) return launch_as<R, float>(st, prm, n);
    if (prm.out.dtype == GVQ_BF16) return launch_as<R, __nv_bfloat16>(st, prm, n);
    return launch_as<R, __half>(st, prm, n);
}

}  // namespace

// Whatever fits is faster here, in us a step of bf16 weights against a launch a product (ortho.cu): 64 x 64 19 against 62,
// 100 x 300 55 / 77, 64 x 1500 50 / 88, 20 x 3333 66 / 98, 128 x 512 65 / 86, 128 x 1000 87 / 95, 32 matrices of up to 64 x 576
// 44 / 93; but not eight parts of a short side of more than 64, whose sums are four times as long (90 x 2400 128 / 98).  As few
// parts as fit, or up to four of short sides of up to 64 while a part has more than five blocks of the long side (the
// orthogonalisation alone): 64 x 576 40 us with one, 38 with two, 37 with four, 47 with eight; 64 x 1500 46 with four, 50 with
// eight; 100 x 300 49 with one, 58 with two.
SmallPlan small_plan(int n, int r, int c, int num_sms)
{
    SmallPlan p{r <= 64 ? 64 : 128, 1, 0};
    const int blocks = (c + 63) / 64, most = p.room == 64 ? 8 : 4;
    auto span = [&](int parts) { return (blocks + parts - 1) / parts; };
    auto fits = [&](int parts) { return (p.room == 64 ? small_smem<64>(span(parts)) : small_smem<128>(span(parts))) <= kSmallSmem; };
    while (p.parts < most && !fits(p.parts)) p.parts *= 2;
    if (n == 0 || r > 128 || !fits(p.parts) || (p.parts > 1 && n * p.parts > num_sms)) return SmallPlan{};
    while (p.room == 64 && p.parts < 4 && n * 2 * p.parts <= num_sms && span(p.parts) > 5) p.parts *= 2;
    p.span = 64 * span(p.parts);
    return p;
}

cudaError_t launch_small(cudaStream_t st, const Matrix *mats, int n, const SmallPlan &plan, const ElementArgs &in, const OutputArgs &out,
                         int32_t *error_word, int wait_kcycles, int test_drop)
{
    SmallParams prm;
    prm.mats = mats;
    prm.parts = plan.parts;
    prm.span = plan.span;
    prm.in = in;
    prm.out = out;
    prm.mode = !in.momentum ? 0 : in.nesterov ? 2 : 1;
    prm.error_word = error_word;
    prm.wait_kcycles = wait_kcycles > 0 ? wait_kcycles : WAIT_KCYCLES_DEFAULT;
    prm.test_drop = test_drop;
    return plan.room == 64 ? launch_typed<64>(st, prm, n) : launch_typed<128>(st, prm, n);
}

}  // namespace ortho
}  // namespace gvq
