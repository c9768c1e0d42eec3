// C entry points of the 8-bit integer format and of the gated block: argument checks and dispatch.
#include "api_util.h"
#include "gvq_internal.h"

using namespace gvq;

namespace {

constexpr int64_t kMost = INT32_MAX - 1024;       // a tensor map's extents and coordinates are 32-bit
constexpr int64_t kMostTerms = 131072;            // 127^2 of them and more fit 32 bits

bool sizes_ok(int64_t rows, int64_t cols)
{
    return rows >= 1 && cols >= 1 && rows <= kMost && cols <= kMost && (rows + 127) / 128 < INT32_MAX / ((cols + 127) / 128);
}
bool dtype_ok(int dtype) { return dtype == GVQ_F32 || dtype == GVQ_BF16 || dtype == GVQ_F16; }
bool half_ok(int dtype) { return dtype == GVQ_BF16 || dtype == GVQ_F16; }
bool act_ok(int act) { return act >= GVQ_SILU && act <= GVQ_SIGMOID; }
bool entry_aligned(const void *p, int dtype) { return (reinterpret_cast<uintptr_t>(p) & (dtype == GVQ_F32 ? 3u : 1u)) == 0; }
bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

Launch launch_of(const gvq_ctx *ctx)
{
    return {ctx->stream, ctx->num_sms, (EncodeTiledFn)ctx->encode_fn, ctx->error_word, ctx->wait_kcycles, ctx->drop_last_load};
}

// The gated block's workspace: dg and du of a backward pass and what holding them in half precision takes, then copies of operands whose rows TMA cannot address.
int64_t padded(int64_t n, int per) { return (n + per - 1) / per * per; }
// Matrices of a backward pass: dg and du, and where they are held in two halves what rounding them left.  Rounded, they add as much to a
// gradient's error as rounding a 16-bit gradient does: sqrt 2 of that in all where both average, but few outputs may carry a gradient's norm
// where products are short (of 99 thousand blocks' gradients with M, F and K spread over 65..8192, 33..8192 and 33..4096, the worst
// 3.3 times, 5 % more than 1.5 times; with the low halves up to 2^26 multiply-adds 1.7 times and 0.4 %).  There the low halves cost least
// (us, dx and both weights' gradients, with and without: 100 x 100 x 100 10.6, 9.0; 150 x 400 x 200 9.1, 7.2; 386 x 380 x 464 13.9, 12.4; the
// call from Python takes 10); with more multiply-adds they double the tensor pipe's time.  Where a caller does not say, the size does.
constexpr int64_t kShort = 1 << 26;
constexpr int kSlopes = GVQ_SLOPES_ROUNDED | GVQ_SLOPES_PRECISE;
bool slopes_ok(int mode) { return (mode & kSlopes) != kSlopes; }
int slopes_of(int64_t M, int64_t F, int64_t K, int mode)
{
    return mode & GVQ_SLOPES_PRECISE ? 4 : mode & GVQ_SLOPES_ROUNDED ? 2 : M * F <= kShort / K ? 4 : 2;
}
int64_t bytes_of(int64_t rows, int64_t cols) { return padded(rows * padded(cols, 8) * 2, 256); }
bool rows_aligned(const void *p, int64_t rows, int64_t ld) { return aligned16(p) && (rows == 1 || ld % 8 == 0); }
// A row that is alone may have any leading dimension: one that a tensor map takes.
int64_t ld_of(int64_t rows, int64_t cols, int64_t ld) { return rows == 1 ? padded(cols, 8) : ld; }

struct Operand { const void *p; int64_t rows, cols, ld; };
// Operands whose rows do not start at 16-byte boundaries get copies at `at`, which the caller has made.
RowCopies align_operands(Operand *ops, int n, char *at)
{
    RowCopies c = {};
    for (int i = 0; i < n; ++i) {
        Operand &o = ops[i];
        if (!o.p) continue;
        if (!rows_aligned(o.p, o.rows, o.ld)) {
            const int k = c.n++;
            c.from[k] = static_cast<const uint16_t *>(o.p);
            c.to[k] = reinterpret_cast<uint16_t *>(at);
            c.ld[k] = o.ld;
            c.rows[k] = o.rows;
            c.cols[k] = o.cols;
            c.chunks[k] = (int)(padded(o.cols, 8) / 8);
            o.p = at;
            o.ld = padded(o.cols, 8);
            at += bytes_of(o.rows, o.cols);
        }
        o.ld = ld_of(o.rows, o.cols, o.ld);
    }
    return c;
}
bool all_aligned(const Operand *ops, int n)
{
    for (int i = 0; i < n; ++i)
        if (ops[i].p && !rows_aligned(ops[i].p, ops[i].rows, ops[i].ld)) return false;
    return true;
}

}  // namespace

extern "C" {

int64_t gvq_i8_codes_bytes(int64_t rows, int64_t cols) { return sizes_ok(rows, cols) ? rows * padded(cols, 16) : -1; }

int64_t gvq_i8_scratch_bytes(int64_t rows, int64_t cols) { return sizes_ok(rows, cols) ? i8_scratch_bytes(rows, cols) : -1; }

gvq_status gvq_i8_quantize(gvq_ctx *ctx, const void *x, int dtype, int64_t rows, int64_t cols, int64_t ld, int rounding,
                           uint64_t seed, uint32_t node, int8_t *codes, float *scales, int8_t *codes_t, float *scales_t,
                           void *scratch, size_t scratch_bytes)
{
    if (!ctx || !x || (!codes && !codes_t) || !codes != !scales || !codes_t != !scales_t) return GVQ_ERR_NULL;
    if (!sizes_ok(rows, cols) || !dtype_ok(dtype) || ld < cols) return GVQ_ERR_SHAPE;
    if (rounding != GVQ_ROUND_NEAREST && rounding != GVQ_ROUND_STOCHASTIC) return GVQ_ERR_SHAPE;
    if (!entry_aligned(x, dtype) || !aligned16(codes) || !aligned4(scales) || !aligned16(codes_t) || !aligned4(scales_t) || !aligned4(scratch))
        return GVQ_ERR_ALIGN;
    const size_t need = codes_t ? (size_t)i8_scratch_bytes(rows, cols) : 0;
    if (need && (!scratch || scratch_bytes < need)) return GVQ_ERR_WORKSPACE;
    DeviceGuard guard(ctx->device);
    GVQ_CUDA(ctx, launch_i8_quantize(ctx->stream, x, dtype, rows, cols, ld, rounding == GVQ_ROUND_STOCHASTIC, seed, node, codes, scales,
                                     codes_t, scales_t, scratch));
    return GVQ_OK;
}

gvq_status gvq_i8_dequantize(gvq_ctx *ctx, const int8_t *codes, const float *scales, int64_t rows, int64_t cols, float *out, int64_t ld)
{
    if (!ctx || !codes || !scales || !out) return GVQ_ERR_NULL;
    if (!sizes_ok(rows, cols) || ld < cols) return GVQ_ERR_SHAPE;
    if (!aligned16(codes) || !aligned4(scales) || !entry_aligned(out, GVQ_F32)) return GVQ_ERR_ALIGN;
    DeviceGuard guard(ctx->device);
    GVQ_CUDA(ctx, launch_i8_dequantize(ctx->stream, ctx->num_sms, codes, scales, rows, cols, out, ld));
    return GVQ_OK;
}

gvq_status gvq_i8_matmul(gvq_ctx *ctx, const int8_t *a_codes, const float *a_scales, const int8_t *b_codes, const float *b_scales,
                         int64_t M, int64_t N, int64_t K, void *out, int dtype, int64_t ld)
{
    if (!ctx || !a_codes || !a_scales || !b_codes || !b_scales || !out) return GVQ_ERR_NULL;
    if (!sizes_ok(M, K) || !sizes_ok(N, K) || !sizes_ok(M, N) || K > kMostTerms || !dtype_ok(dtype) || ld < N) return GVQ_ERR_SHAPE;
    if (!aligned16(a_codes) || !aligned4(a_scales) || !aligned16(b_codes) || !aligned4(b_scales) || !entry_aligned(out, dtype))
        return GVQ_ERR_ALIGN;
    if (!ctx->encode_fn) return GVQ_ERR_UNSUPPORTED;
    DeviceGuard guard(ctx->device);
    GVQ_CUDA(ctx, launch_i8_matmul(launch_of(ctx), a_codes, a_scales, b_codes, b_scales, M, N, K, out, dtype, ld));
    return GVQ_OK;
}

gvq_status gvq_i8_gated(gvq_ctx *ctx, const int8_t *a_codes, const float *a_scales, const int8_t *gate_codes, const float *gate_scales,
                        const int8_t *up_codes, const float *up_scales, int64_t M, int64_t F, int64_t K, int activation, void *out, int dtype,
                        int64_t ld)
{
    if (!ctx || !a_codes || !a_scales || !gate_codes || !gate_scales || !up_codes || !up_scales || !out) return GVQ_ERR_NULL;
    if (!sizes_ok(M, K) || !sizes_ok(F, K) || !sizes_ok(M, F) || K > kMostTerms || !dtype_ok(dtype) || ld < F || !act_ok(activation))
        return GVQ_ERR_SHAPE;
    if (!aligned16(a_codes) || !aligned4(a_scales) || !aligned16(gate_codes) || !aligned4(gate_scales) || !aligned16(up_codes) ||
        !aligned4(up_scales) || !entry_aligned(out, dtype))
        return GVQ_ERR_ALIGN;
    if (!ctx->encode_fn) return GVQ_ERR_UNSUPPORTED;
    DeviceGuard guard(ctx->device);
    GVQ_CUDA(ctx, launch_i8_gated(launch_of(ctx), a_codes, a_scales, gate_codes, gate_scales, up_codes, up_scales, M, F, K, activation, out,
                                  dtype, ld));
    return GVQ_OK;
}

int64_t gvq_gated_workspace_bytes(int64_t M, int64_t F, int64_t K, int backward, int aligned)
{
    if (!sizes_ok(M, F) || !sizes_ok(M, K) || !sizes_ok(F, K) || !slopes_ok(backward)) return -1;
    return (backward ? slopes_of(M, F, K, backward) * bytes_of(M, F) + kGatedRoom : 0) + (aligned ? 0 : bytes_of(M, K) + 2 * bytes_of(F, K));
}

gvq_status gvq_gated_forward(gvq_ctx *ctx, const void *x, int64_t ldx, const void *w_gate, int64_t ld_gate, const void *w_up, int64_t ld_up,
                             int dtype, int64_t M, int64_t F, int64_t K, int activation, void *h, int64_t ldh, void *gate_opt,
                             int64_t ld_gate_out, void *up_opt, int64_t ld_up_out, void *workspace, size_t workspace_bytes)
{
    if (!ctx || !x || !w_gate || !w_up || !h || !gate_opt != !up_opt) return GVQ_ERR_NULL;
    if (!sizes_ok(M, F) || !sizes_ok(M, K) || !sizes_ok(F, K) || !half_ok(dtype) || !act_ok(activation) || ldx < K || ld_gate < K ||
        ld_up < K || ldh < F || (gate_opt && (ld_gate_out < F || ld_up_out < F)))
        return GVQ_ERR_SHAPE;
    for (const void *p : {x, w_gate, w_up, (const void *)h, (const void *)gate_opt, (const void *)up_opt, (const void *)workspace})
        if (!entry_aligned(p, dtype)) return GVQ_ERR_ALIGN;
    Operand ops[3] = {{x, M, K, ldx}, {w_gate, F, K, ld_gate}, {w_up, F, K, ld_up}};
    if (!all_aligned(ops, 3)) {
        if (!workspace || workspace_bytes < (size_t)gvq_gated_workspace_bytes(M, F, K, 0, 0)) return GVQ_ERR_WORKSPACE;
        if (!aligned16(workspace)) return GVQ_ERR_ALIGN;
    }
    if (!ctx->encode_fn) return GVQ_ERR_UNSUPPORTED;
    DeviceGuard guard(ctx->device);
    const Launch l = launch_of(ctx);
    const RowCopies copies = align_operands(ops, 3, static_cast<char *>(workspace));
    if (copies.n) GVQ_CUDA(ctx, launch_align_rows(l, copies));
    GVQ_CUDA(ctx, launch_gated(l, ops[0].p, ops[0].ld, ops[1].p, ops[1].ld, ops[2].p, ops[2].ld, dtype, M, F, K, activation, h, ldh, gate_opt,
                               ld_gate_out, up_opt, ld_up_out));
    return GVQ_OK;
}

gvq_status gvq_gated_backward(gvq_ctx *ctx, const void *dh, int64_t ld_dh, const void *gate, int64_t ld_gate_in, const void *up,
                              int64_t ld_up_in, const void *x, int64_t ldx, const void *w_gate, int64_t ld_gate, const void *w_up,
                              int64_t ld_up, int dtype, int64_t M, int64_t F, int64_t K, int activation, void *dx_opt, int64_t ld_dx,
                              void *dw_gate_opt, int64_t ld_dw_gate, void *dw_up_opt, int64_t ld_dw_up, int dw_dtype, void *workspace,
                              size_t workspace_bytes)
{
    const bool dw = dw_gate_opt || dw_up_opt;
    const int slopes = activation & kSlopes;
    activation &= ~kSlopes;
    if (!ctx || !dh || !gate || !up || (!dx_opt && !dw) || (dx_opt && (!w_gate || !w_up)) || (dw && !x)) return GVQ_ERR_NULL;
    if (!sizes_ok(M, F) || !sizes_ok(M, K) || !sizes_ok(F, K) || !half_ok(dtype) || (dw && !dtype_ok(dw_dtype)) || !act_ok(activation) || !slopes_ok(slopes) ||
        ld_dh < F || ld_gate_in < F || ld_up_in < F || (dw && ldx < K) || (dx_opt && (ld_gate < K || ld_up < K || ld_dx < K)) ||
        (dw_gate_opt && ld_dw_gate < K) || (dw_up_opt && ld_dw_up < K))
        return GVQ_ERR_SHAPE;
    for (const void *p : {dh, gate, up, dw ? x : nullptr, dx_opt ? w_gate : nullptr, dx_opt ? w_up : nullptr, (const void *)dx_opt})
        if (!entry_aligned(p, dtype)) return GVQ_ERR_ALIGN;
    if (!entry_aligned(dw_gate_opt, dw_dtype) || !entry_aligned(dw_up_opt, dw_dtype) || !aligned16(workspace)) return GVQ_ERR_ALIGN;
    Operand ops[3] = {{dw ? x : nullptr, M, K, ldx}, {dx_opt ? w_gate : nullptr, F, K, ld_gate}, {dx_opt ? w_up : nullptr, F, K, ld_up}};
    if (!workspace || workspace_bytes < (size_t)gvq_gated_workspace_bytes(M, F, K, 1 | slopes, all_aligned(ops, 3))) return GVQ_ERR_WORKSPACE;
    if (!ctx->encode_fn) return GVQ_ERR_UNSUPPORTED;
    DeviceGuard guard(ctx->device);
    const Launch l = launch_of(ctx);
    char *at = static_cast<char *>(workspace);
    const int n = slopes_of(M, F, K, slopes);
    char *room = at + n * bytes_of(M, F);
    const RowCopies copies = align_operands(ops, 3, room + kGatedRoom);
    GatedGrads g = {{}, {ops[1].p, ops[2].p}, ops[0].p, padded(F, 8), {ops[1].ld, ops[2].ld}, ops[0].ld, dtype, dw_dtype, M, F, K,
                    dx_opt, {dw_gate_opt, dw_up_opt}, ld_dx, {ld_dw_gate, ld_dw_up},
                    dtype == GVQ_F16 ? reinterpret_cast<float *>(room + kGatedRoom) - 1 : nullptr};
    for (int i = 0; i < n; ++i) g.d[i] = at + i * bytes_of(M, F);
    GVQ_CUDA(ctx, launch_gated_slopes(l, dh, ld_dh, gate, ld_gate_in, up, ld_up_in, activation, g, room, copies));
    GVQ_CUDA(ctx, launch_gated_products(l, g));
    return GVQ_OK;
}

}  // extern "C"
