// C entry points of the microscaled 4-bit format: argument checks and dispatch.
#include "api_util.h"
#include "gvq_internal.h"
#include "mx4.cuh"

using namespace gvq;

namespace {

bool sizes_ok(int64_t rows, int64_t cols)
{
    // (the first two bounds keep the products below from wrapping)
    return rows >= 1 && cols >= 1 && rows < ((int64_t)1 << 38) && cols < ((int64_t)1 << 38) &&
           mx4::tiles_of(rows, 128) < INT32_MAX / mx4::tiles_of(cols, 128);
}
bool dtype_ok(int dtype) { return dtype == GVQ_F32 || dtype == GVQ_BF16 || dtype == GVQ_F16; }
bool entry_aligned(const void *p, int dtype) { return (reinterpret_cast<uintptr_t>(p) & (dtype == GVQ_F32 ? 3u : 1u)) == 0; }

// N device pointers of an optional output or of a required input
template <typename T>
gvq_status gather(T *const *src, int N, NodePtrs<T> &dst)
{
    for (int n = 0; n < GVQ_MAX_NODES; ++n) dst.p[n] = nullptr;
    for (int n = 0; n < N; ++n) {
        if (!src[n]) return GVQ_ERR_NULL;
        if (!aligned16(src[n])) return GVQ_ERR_ALIGN;
        dst.p[n] = src[n];
    }
    return GVQ_OK;
}

}  // namespace

extern "C" {

int64_t gvq_mx4_codes_bytes(int64_t rows, int64_t cols)
{
    return sizes_ok(rows, cols) ? rows * 16 * mx4::blocks(cols) : -1;
}

int64_t gvq_mx4_scales_bytes(int64_t rows, int64_t cols)
{
    return sizes_ok(rows, cols) ? mx4::tiles_of(rows, 128) * mx4::tiles_of(cols, 128) * mx4::kTileBytes : -1;
}

gvq_status gvq_mx4_quantize(gvq_ctx *ctx, const void *x, int dtype, int64_t rows, int64_t cols, int64_t ld, int rounding,
                            uint64_t seed, uint32_t node, uint8_t *codes, uint8_t *scales, uint8_t *codes_t,
                            uint8_t *scales_t)
{
    if (!ctx || !x || (!codes && !codes_t) || !codes != !scales || !codes_t != !scales_t) return GVQ_ERR_NULL;
    if (!sizes_ok(rows, cols) || !dtype_ok(dtype) || ld < cols) return GVQ_ERR_SHAPE;
    if (rounding != GVQ_ROUND_NEAREST && rounding != GVQ_ROUND_STOCHASTIC) return GVQ_ERR_SHAPE;
    if (!entry_aligned(x, dtype) || !aligned16(codes) || !aligned16(scales) || !aligned16(codes_t) || !aligned16(scales_t))
        return GVQ_ERR_ALIGN;
    DeviceGuard guard(ctx->device);
    GVQ_CUDA(ctx, launch_mx4_quantize(ctx->stream, x, dtype, rows, cols, ld, rounding == GVQ_ROUND_STOCHASTIC, seed, node,
                                      codes, scales, codes_t, scales_t));
    return GVQ_OK;
}

gvq_status gvq_mx4_dequantize(gvq_ctx *ctx, const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols,
                              float *out, int64_t ld)
{
    if (!ctx || !codes || !scales || !out) return GVQ_ERR_NULL;
    if (!sizes_ok(rows, cols) || ld < cols) return GVQ_ERR_SHAPE;
    if (!aligned16(codes) || !aligned16(scales) || !entry_aligned(out, GVQ_F32)) return GVQ_ERR_ALIGN;
    NodePtrs<const uint8_t> c{}, s{};
    c.p[0] = codes;
    s.p[0] = scales;
    DeviceGuard guard(ctx->device);
    GVQ_CUDA(ctx, launch_mx4_dequantize(ctx->stream, ctx->num_sms, c, s, 1, rows, cols, out, ld, nullptr, 0));
    return GVQ_OK;
}

gvq_status gvq_mx4_matmul(gvq_ctx *ctx, const uint8_t *a_codes, const uint8_t *a_scales, const uint8_t *b_codes,
                          const uint8_t *b_scales, int64_t M, int64_t N, int64_t K, void *out, int dtype, int64_t ld)
{
    if (!ctx || !a_codes || !a_scales || !b_codes || !b_scales || !out) return GVQ_ERR_NULL;
    if (!sizes_ok(M, K) || !sizes_ok(N, K) || !sizes_ok(M, N) || !dtype_ok(dtype) || ld < N) return GVQ_ERR_SHAPE;
    // a tensor map's extents and coordinates are 32-bit
    if (M > INT32_MAX || N > INT32_MAX || 16 * mx4::blocks(K) > INT32_MAX) return GVQ_ERR_SHAPE;
    if (!aligned16(a_codes) || !aligned16(a_scales) || !aligned16(b_codes) || !aligned16(b_scales) || !entry_aligned(out, dtype))
        return GVQ_ERR_ALIGN;
    if (!ctx->encode_fn) return GVQ_ERR_UNSUPPORTED;
    DeviceGuard guard(ctx->device);
    GVQ_CUDA(ctx, launch_mx4_matmul(ctx->stream, ctx->num_sms, (EncodeTiledFn)ctx->encode_fn, a_codes, a_scales, b_codes,
                                    b_scales, M, N, K, out, dtype, ld, ctx->error_word, ctx->wait_kcycles, ctx->drop_last_load));
    return GVQ_OK;
}

gvq_status gvq_mx4_quantize_aggregate(gvq_ctx *ctx, const float *const *g_nodes, int N, uint32_t node0, int rounding,
                                      uint64_t seed, float *g_sum, uint8_t *const *codes_nodes_opt,
                                      uint8_t *const *scales_nodes_opt)
{
    if (!ctx || (!g_sum && !codes_nodes_opt) || !codes_nodes_opt != !scales_nodes_opt) return GVQ_ERR_NULL;
    if (rounding != GVQ_ROUND_NEAREST && rounding != GVQ_ROUND_STOCHASTIC) return GVQ_ERR_SHAPE;
    NodePtrs<const float> g;
    gvq_status st = gather_nodes(g_nodes, N, g);
    if (st != GVQ_OK) return st;
    if (!aligned16(g_sum)) return GVQ_ERR_ALIGN;
    for (int n = 0; n < N; ++n)
        if (g.p[n] == g_sum) return GVQ_ERR_SHAPE;
    NodePtrs<uint8_t> c, s;
    if (codes_nodes_opt) {
        if ((st = gather(codes_nodes_opt, N, c)) != GVQ_OK || (st = gather(scales_nodes_opt, N, s)) != GVQ_OK) return st;
    }
    DeviceGuard guard(ctx->device);
    GVQ_CUDA(ctx, launch_mx4_quantize_aggregate(ctx->stream, ctx->num_sms, ctx->d, ctx->S, ctx->decompress_tiles, ctx->lt, g, N, node0,
                                                rounding == GVQ_ROUND_STOCHASTIC, seed, g_sum, codes_nodes_opt ? &c : nullptr,
                                                codes_nodes_opt ? &s : nullptr));
    return GVQ_OK;
}

gvq_status gvq_mx4_dequantize_aggregate(gvq_ctx *ctx, const uint8_t *const *codes_nodes,
                                        const uint8_t *const *scales_nodes, const float *const *g_nodes_for_tails, int N,
                                        float *g_sum)
{
    if (!ctx || !codes_nodes || !scales_nodes || !g_sum) return GVQ_ERR_NULL;
    NodePtrs<const uint8_t> c, s;
    gvq_status st;
    if ((st = gather_nodes(codes_nodes, N, c)) != GVQ_OK || (st = gather_nodes(scales_nodes, N, s)) != GVQ_OK) return st;
    NodePtrs<const float> g;
    if (ctx->has_tails && (st = gather_nodes(g_nodes_for_tails, N, g)) != GVQ_OK) return st;
    if (!aligned16(g_sum)) return GVQ_ERR_ALIGN;
    DeviceGuard guard(ctx->device);
    GVQ_CUDA(ctx, launch_mx4_dequantize(ctx->stream, ctx->num_sms, c, s, N, ctx->S, ctx->d, g_sum, 0, &ctx->lt, ctx->n_layers));
    if (ctx->has_tails) GVQ_CUDA(ctx, launch_tail_sum(ctx->stream, ctx->lt, ctx->d, g, N, g_sum));
    return GVQ_OK;
}

}  // extern "C"
