// Backward pass of the gated block (gvq.h, "the gated block"):
//   dg = dh u act'(g),  du = dh act(g)             gated_slopes_kernel; in half precision gated_tops_kernel before it
//   dx = dg Wg + du Wu                             one product whose contraction has two segments
//   dWg = dg^T x,  dWu = du^T x                    one product of two halves that have x in common
// in one launch for the slopes (two in half precision) and one or two for the products,
// and the copies of operands whose rows do not start at 16-byte boundaries, which TMA cannot address.
#include <float.h>

#include "load8.cuh"
#include "product.cuh"

namespace gvq {
namespace {

using namespace product;

// The copies, eight entries a thread at a time; rows of a copy are padded to eight entries by zeros.
__device__ __forceinline__ void copy_rows(const RowCopies &k)
{
    for (int i = 0; i < k.n; ++i)
        for_chunks(k.rows[i], k.chunks[i], [&](int64_t r, int c) {
            const int64_t at = (int64_t)c * 8;
            const int n = (int)min((int64_t)8, k.cols[i] - at);
            *reinterpret_cast<uint4 *>(k.to[i] + r * k.chunks[i] * 8 + at) = load8<false>(k.from[i] + r * k.ld[i] + at, n).q[0];
        });
}
__global__ void __launch_bounds__(256) align_rows_kernel(const __grid_constant__ RowCopies copies)
{
    launch_dependents();
    grid_dependency_wait();
    copy_rows(copies);
}

struct SlopeParams {
    const void *dh, *g, *u;
    int64_t ld_dh, ld_g, ld_u;
    void *d[4];                // dg, du and what rounding them left (or null); rows ld_out entries apart, starting at 16-byte boundaries
    int64_t rows, cols, ld_out;
    int chunks;                // groups of eight columns of a row
    RowCopies copies;          // done on the way: the products after this launch read them
    uint16_t *tops;            // half precision: of each CTA of gated_tops_kernel, see there
    int n_tops;
    float *unscale;            // half precision: what makes the products of dg and du as they are held those of dg and du
};

template <typename T, bool VEC>
__device__ __forceinline__ void load_eight(const void *p, int64_t at, int n, float (&v)[8])
{
    const Raw8<uint16_t> q = load8<VEC>(static_cast<const uint16_t *>(p) + at, n);
    T e[8];
    memcpy(e, &q, 16);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = to_f(e[i]);
}

// Eight entries of dg and of du from column `chunk * 8` of row r on.
template <typename T, int ACT, bool VEC>
__device__ __forceinline__ void slopes_at(const SlopeParams &prm, int64_t r, int chunk, float (&d)[2][8])
{
    const int64_t c = (int64_t)chunk * 8;
    const int n = (int)min((int64_t)8, prm.cols - c);
    float dh[8], g[8], u[8];
    load_eight<T, VEC>(prm.dh, r * prm.ld_dh + c, n, dh);
    load_eight<T, VEC>(prm.g, r * prm.ld_g + c, n, g);
    load_eight<T, VEC>(prm.u, r * prm.ld_u + c, n, u);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float2 a = activation_and_slope<ACT>(g[i]);
        d[0][i] = dh[i] * u[i] * a.y;
        d[1][i] = dh[i] * a.x;
    }
}
__device__ __forceinline__ uint32_t block_max(uint32_t v)      // 256 threads
{
    __shared__ uint32_t of_warp[8];
    v = __reduce_max_sync(0xffffffffu, v);
    if ((threadIdx.x & 31) == 0) of_warp[threadIdx.x >> 5] = v;
    __syncthreads();
    v = of_warp[threadIdx.x & 7];
    return __reduce_max_sync(0xffffffffu, v);
}

// Half precision has 5 bits of exponent: dg and du of tokens with small gradients would be among its subnormal numbers (1e-6 in steps of
// 6e-8), and those past 65504 infinite, although fp32 sums and the weights' gradients in fp32 hold them.  So they are held times a power of
// two, the largest finite entry of both between 2^15 and 2^16, and the products' epilogues undo it (exactly): entries down to 2^-29 of the
// largest keep their 11 bits.  The largest has to be known before the first is rounded, so inputs are read once more (all gradients in
// fp16, us, with and without: 100 x 100 x 100 12, 9.7; 777 x 1029 x 515 25, 19; 2048 x 2048 x 1024 40, 31; 8192 x 8192 x 512 434, 338).  Two or
// three chunks of a thread on their way at a time are no faster (777 x 1029 x 515 26 and 28).
// A bfloat16 has fp32's exponents and needs none of this.
// A CTA leaves its entries' largest exponent, as fp32 has it; one more where times a power of two up to 2^16 it would round past 65504.
constexpr int kMostTops = 1024;
template <typename T, int ACT, bool VEC>
__global__ void __launch_bounds__(256) gated_tops_kernel(const __grid_constant__ SlopeParams prm)
{
    launch_dependents();
    grid_dependency_wait();
    uint32_t top = 0;
    for_chunks(prm.rows, prm.chunks, [&](int64_t r, int chunk) {
        float d[2][8];
        slopes_at<T, ACT, VEC>(prm, r, chunk, d);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint32_t m = __float_as_uint(d[i / 8][i % 8]) & 0x7FFFFFFFu;
            top = max(top, m < 0x7F800000u ? m : 0u);
        }
    });
    __syncwarp();
    top = block_max(top);
    if (threadIdx.x == 0) prm.tops[blockIdx.x] = (uint16_t)((top >> 23) + ((top & 0x7FFFFFu) > 0x7FE000u));
}
// The power of two, and its reciprocal for the products.
__device__ __forceinline__ float half_scale(const SlopeParams &prm)
{
    uint32_t top = 0;
    for (int i = threadIdx.x; i < prm.n_tops; i += 256) top = max(top, (uint32_t)__ldcg(prm.tops + i));
    __syncwarp();
    const int e = min(126, 15 + 127 - (int)block_max(top));      // (both are normal numbers)
    if (blockIdx.x == 0 && threadIdx.x == 0) *prm.unscale = __uint_as_float((uint32_t)(127 - e) << 23);
    return __uint_as_float((uint32_t)(127 + e) << 23);
}

// Eight entries a thread, each read and written once: 8192 x 8192 in 106 us, where the bytes take 103 at the copy rate.
constexpr int kResident = 6;      // CTAs of an SM: the grid is as many as there is room for at once (16 an SM: 109 us)
template <typename T, int ACT, bool VEC>
__global__ void __launch_bounds__(256, kResident) gated_slopes_kernel(const __grid_constant__ SlopeParams prm)
{
    launch_dependents();
    grid_dependency_wait();
    float scale = 1.0f;
    if constexpr (std::is_same_v<T, __half>) scale = half_scale(prm);
    for_chunks(prm.rows, prm.chunks, [&](int64_t r, int chunk) {
        float d[2][8];
        slopes_at<T, ACT, VEC>(prm, r, chunk, d);
        const int64_t at = r * prm.ld_out + (int64_t)chunk * 8;      // (rows are padded to eight entries)
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            uint32_t w[4];
            if constexpr (std::is_same_v<T, __half>) {
#pragma unroll
                for (int i = 0; i < 8; ++i) d[which][i] *= scale;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = pack2<T>(d[which][2 * i], d[which][2 * i + 1]);
            *reinterpret_cast<uint4 *>(static_cast<T *>(prm.d[which]) + at) = make_uint4(w[0], w[1], w[2], w[3]);
            if (prm.d[2]) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    T e[2];
                    memcpy(e, &w[i], 4);
                    auto rest = [](float x, float of) { return fabsf(x - of) <= FLT_MAX ? x - of : 0.0f; };      // (none of an infinity or a NaN)
                    w[i] = pack2<T>(rest(d[which][2 * i], to_f(e[0])), rest(d[which][2 * i + 1], to_f(e[1])));
                }
                *reinterpret_cast<uint4 *>(static_cast<T *>(prm.d[2 + which]) + at) = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
    });
    copy_rows(prm.copies);
}

Params start(const Launch &l, const GatedGrads &g, int out_dtype)
{
    Params prm = {};
    prm.dtype = out_dtype;
    prm.bf16 = g.dtype == GVQ_BF16;
    prm.unscale = g.unscale;
    prm.error_word = l.error_word;
    prm.wait_kcycles = l.wait_kcycles > 0 ? l.wait_kcycles : WAIT_KCYCLES_DEFAULT;
    prm.test_drop = l.test_drop;
    return prm;
}

int grid_of(int num_sms, int64_t items, int per_sm)
{
    const int64_t blocks = (items + 255) / 256, most = (int64_t)num_sms * per_sm;
    return (int)(blocks < most ? blocks : most);
}

int64_t items_of(const RowCopies &c)      // of the largest
{
    int64_t items = 0;
    for (int k = 0; k < c.n; ++k) items = items > c.rows[k] * c.chunks[k] ? items : c.rows[k] * c.chunks[k];
    return items;
}

template <typename T, int ACT, bool VEC>
cudaError_t launch_slopes_of(const Launch &l, SlopeParams &prm)
{
    const int64_t slopes = prm.rows * prm.chunks, copies = items_of(prm.copies);
    if constexpr (std::is_same_v<T, __half>) {
        const int grid = grid_of(l.num_sms, slopes, kResident);
        prm.n_tops = grid < kMostTops ? grid : kMostTops;
        const cudaError_t e = launch_chained<gated_tops_kernel<T, ACT, VEC>>(prm, prm.n_tops, 256, 0, 1, l.stream);
        if (e != cudaSuccess) return e;
    }
    const int grid = grid_of(l.num_sms, slopes > copies ? slopes : copies, kResident);
    return launch_chained<gated_slopes_kernel<T, ACT, VEC>>(prm, grid, 256, 0, 1, l.stream);
}
template <typename T, bool VEC>
cudaError_t launch_slopes_as(const Launch &l, SlopeParams &prm, int act)
{
    switch (act) {
    case GVQ_SILU: return launch_slopes_of<T, GVQ_SILU, VEC>(l, prm);
    case GVQ_GELU: return launch_slopes_of<T, GVQ_GELU, VEC>(l, prm);
    case GVQ_GELU_TANH: return launch_slopes_of<T, GVQ_GELU_TANH, VEC>(l, prm);
    case GVQ_RELU: return launch_slopes_of<T, GVQ_RELU, VEC>(l, prm);
    default: return launch_slopes_of<T, GVQ_SIGMOID, VEC>(l, prm);
    }
}

}  // namespace

cudaError_t launch_align_rows(const Launch &l, const RowCopies &copies)
{
    return launch_chained<align_rows_kernel>(copies, grid_of(l.num_sms, items_of(copies), kResident), 256, 0, 1, l.stream);
}

static_assert(kGatedRoom >= kMostTops * sizeof(uint16_t) + sizeof(float) && kGatedRoom % 256 == 0, "the workspace's room");

cudaError_t launch_gated_slopes(const Launch &l, const void *dh, int64_t ld_dh, const void *g, int64_t ld_g, const void *u, int64_t ld_u,
                                int act, const GatedGrads &of, void *room, const RowCopies &copies)
{
    auto aligned = [](const void *p, int64_t ld) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld % 8 == 0; };
    SlopeParams prm = {dh, g, u, ld_dh, ld_g, ld_u, {of.d[0], of.d[1], of.d[2], of.d[3]}, of.M, of.F, of.ld_d, (int)((of.F + 7) / 8), copies,
                       static_cast<uint16_t *>(room), 0, of.unscale};
    const bool vec = aligned(dh, ld_dh) && aligned(g, ld_g) && aligned(u, ld_u);      // all rows start at 16-byte boundaries
    if (of.dtype == GVQ_BF16) return vec ? launch_slopes_as<__nv_bfloat16, true>(l, prm, act) : launch_slopes_as<__nv_bfloat16, false>(l, prm, act);
    return vec ? launch_slopes_as<__half, true>(l, prm, act) : launch_slopes_as<__half, false>(l, prm, act);
}

namespace {

// Halves that dg and du have: one, or two where what rounding left of them is multiplied too.
int precise(const GatedGrads &g) { return g.d[2] ? 2 : 1; }
// dx = dg Wg + du Wu: a contraction of two segments (four).  The weights are MN-major here: boxes of 64 of a row's entries by 64 rows.
bool dx_problem(Params &prm, const Launch &l, const Cut &c, const GatedGrads &g)
{
    prm = start(l, g, g.dtype);
    prm.M = c.few ? g.K : g.M;
    prm.N = c.few ? g.M : g.K;
    const int segments = 2 * precise(g);
    divide(prm, c, k16, false, g.F, segments, 1);
    CUtensorMap *map_w = c.few ? prm.a : prm.b, *map_d = c.few ? prm.b : prm.a;
    const int box_d = c.few ? c.bn : 128;
    set_output(prm, 0, g.dx, g.dtype, g.ld_dx);
    bool ok = true;
    for (int i = 0; i < segments; ++i) {
        ok = ok && encode(l.encode, map_d + i, k16, g.d[i], g.M, g.F, g.ld_d, box_d);
        if (i < 2) ok = ok && encode(l.encode, map_w + i, k16, g.w[i], g.F, g.K, g.ld_w[i], 64);
        else map_w[i] = map_w[i - 2];
    }
    return ok;
}
// dWg = dg^T x, dWu = du^T x, or the one of them that is wanted: two halves of a product, both operands MN-major.
int halves_of(const GatedGrads &g) { return g.dw[0] && g.dw[1] ? 2 : 1; }
bool dw_problem(Params &prm, const Launch &l, const Cut &c, const GatedGrads &g)
{
    const int halves = halves_of(g), segments = precise(g);
    prm = start(l, g, g.dw_dtype);
    prm.M = g.F;
    prm.N = g.K;
    prm.a_mn = 1;
    divide(prm, c, k16, false, g.M, segments, halves);
    bool ok = encode(l.encode, &prm.b[0], k16, g.x, g.M, g.K, g.ldx, 64);
    prm.b[1] = prm.b[0];
    for (int i = 0; i < halves; ++i) {
        const int which = g.dw[0] ? i : 1;
        for (int seg = 0; seg < segments; ++seg)
            ok = ok && encode(l.encode, &prm.a[i * segments + seg], k16, g.d[2 * seg + which], g.M, g.F, g.ld_d, 64);
        set_output(prm, i, g.dw[which], g.dw_dtype, g.ld_dw[which]);
    }
    return ok;
}
Cut cut_dx(const Launch &l, const GatedGrads &g) { return cut(l.num_sms, g.M, g.K, false, 2 * precise(g) * stages_of(g.F, k16), 64); }
Cut cut_dw(const Launch &l, const GatedGrads &g) { return cut_tiles(l.num_sms, g.F, g.K, false, precise(g) * stages_of(g.M, k16), halves_of(g)); }

cudaError_t launch_dx(const Launch &l, const Cut &c, const GatedGrads &g)
{
    Params prm;
    if (!dx_problem(prm, l, c, g)) return cudaErrorInvalidValue;
    const cudaStream_t st = l.stream;
    if (c.few) {
        switch (c.bn) {
        case 16: return launch<k16, 1, 16, true, true, false, false>(st, l.num_sms, prm);
        case 32: return launch<k16, 1, 32, true, true, false, false>(st, l.num_sms, prm);
        default: return launch<k16, 1, 64, true, true, false, false>(st, l.num_sms, prm);
        }
    }
    switch (c.bn) {
    case 256: return launch<k16, 2, 256, false, false, true, false>(st, l.num_sms, prm);
    case 128: return launch<k16, 2, 128, false, false, true, false>(st, l.num_sms, prm);
    default: return launch<k16, 1, 64, false, false, true, false>(st, l.num_sms, prm);
    }
}
cudaError_t launch_dw(const Launch &l, const Cut &c, const GatedGrads &g)
{
    Params prm;
    if (!dw_problem(prm, l, c, g)) return cudaErrorInvalidValue;
    switch (c.bn) {
    case 256: return launch<k16, 2, 256, false, true, true, false>(l.stream, l.num_sms, prm);
    case 128: return launch<k16, 2, 128, false, true, true, false>(l.stream, l.num_sms, prm);
    default: return launch<k16, 1, 64, false, true, true, false>(l.stream, l.num_sms, prm);
    }
}

}  // namespace

// Neither product needs the other: where one of them, or its last round of tiles, would leave SMs idle, they share a launch, each on
// SMs of its own.
cudaError_t launch_gated_products(const Launch &l, const GatedGrads &g)
{
    const bool dw = g.dw[0] || g.dw[1];
    Cut cx = {}, cw = {};
    if (g.dx) cx = cut_dx(l, g);
    if (dw) cw = cut_dw(l, g);
    if (g.dx && dw && !cx.few) {
        const Extent e[2] = {{g.M, g.K, 2 * precise(g) * stages_of(g.F, k16), 1}, {g.F, g.K, precise(g) * stages_of(g.M, k16), halves_of(g)}};
        const PairCut c = cut_pair(l.num_sms, e);
        // (the second of two launches starts while the first ends)
        if (c.time && c.time < 0.98 * (cx.time + cw.time - 1.5)) {
            Pair pair;
            if (!dx_problem(pair.p[0], l, c.c[0], g) || !dw_problem(pair.p[1], l, c.c[1], g)) return cudaErrorInvalidValue;
            pair.blocks = c.blocks[0];
            switch (c.c[0].bn) {
            case 256: return launch_pair<k16, 2, 256, true>(l.stream, pair, c.blocks);
            case 128: return launch_pair<k16, 2, 128, true>(l.stream, pair, c.blocks);
            default: return launch_pair<k16, 1, 64, true>(l.stream, pair, c.blocks);
            }
        }
    }
    if (g.dx) {
        const cudaError_t e = launch_dx(l, cx, g);
        if (e != cudaSuccess || !dw) return e;
    }
    return launch_dw(l, cw, g);
}

}  // namespace gvq
