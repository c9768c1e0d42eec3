// Products of 8-bit integer matrices with a scale a row (gvq.h, "8-bit integers"), plain and gated.
#include "product.cuh"

namespace gvq {
namespace {

using namespace product;

bool encode_codes(EncodeTiledFn enc, CUtensorMap *map, const int8_t *codes, int64_t rows, int64_t cols, int box_rows)
{
    return encode(enc, map, kI8, codes, rows, cols, (cols + 15) / 16 * 16, box_rows);
}

Params start(const Launch &l, int dtype)
{
    Params prm = {};
    prm.dtype = dtype;
    prm.error_word = l.error_word;
    prm.wait_kcycles = l.wait_kcycles > 0 ? l.wait_kcycles : WAIT_KCYCLES_DEFAULT;
    prm.test_drop = l.test_drop;
    return prm;
}

}  // namespace

cudaError_t launch_i8_matmul(const Launch &l, const int8_t *a, const float *sa, const int8_t *b, const float *sb, int64_t M, int64_t N,
                             int64_t K, void *out, int dtype, int64_t ld)
{
    Params prm = start(l, dtype);
    const Cut c = cut(l.num_sms, M, N, 64);
    prm.M = c.swapped ? N : M;
    prm.N = c.swapped ? M : N;
    divide(prm, l.num_sms, c, kI8, c.bn, K, 1, 1);
    prm.scale_m[0] = c.swapped ? sb : sa;
    prm.scale_n[0] = c.swapped ? sa : sb;
    if (!encode_codes(l.encode, &prm.a[0], c.swapped ? b : a, prm.M, K, 128) ||
        !encode_codes(l.encode, &prm.b[0], c.swapped ? a : b, prm.N, K, c.bn / c.cg))
        return cudaErrorInvalidValue;
    set_output(l.encode, prm, 0, out, dtype, M, N, ld);
    if (c.cg == 2) return launch<kI8, 2, 256, 1, false, false, false>(l.stream, l.num_sms, prm);
    switch (c.bn) {
    case 16: return launch<kI8, 1, 16, 1, false, false, false>(l.stream, l.num_sms, prm);
    case 32: return launch<kI8, 1, 32, 1, false, false, false>(l.stream, l.num_sms, prm);
    default: return launch<kI8, 1, 64, 1, false, false, false>(l.stream, l.num_sms, prm);
    }
}

cudaError_t launch_i8_gated(const Launch &l, const int8_t *a, const float *sa, const int8_t *gate, const float *s_gate, const int8_t *up,
                            const float *s_up, int64_t M, int64_t F, int64_t K, int act, void *out, int dtype, int64_t ld)
{
    Params prm = start(l, dtype);
    prm.act = act;
    const Cut c = cut(l.num_sms, M, F, 32);
    prm.M = c.swapped ? F : M;
    prm.N = c.swapped ? M : F;
    divide(prm, l.num_sms, c, kI8, c.swapped ? c.bn : c.bn / 2, K, 1, 1);
    const int8_t *w[2] = {gate, up};
    const float *sw[2] = {s_gate, s_up};
    CUtensorMap *map_w = c.swapped ? prm.a : prm.b;
    for (int i = 0; i < 2; ++i) {
        (c.swapped ? prm.scale_m : prm.scale_n)[i] = sw[i];
        if (!encode_codes(l.encode, map_w + i, w[i], F, K, c.swapped || c.cg == 2 ? 128 : 32)) return cudaErrorInvalidValue;
    }
    (c.swapped ? prm.scale_n : prm.scale_m)[0] = sa;
    if (!encode_codes(l.encode, c.swapped ? prm.b : prm.a, a, M, K, c.swapped ? c.bn : 128)) return cudaErrorInvalidValue;
    set_output(l.encode, prm, 0, out, dtype, M, F, ld);
    if (c.cg == 2) return launch<kI8, 2, 256, 1, false, false, true>(l.stream, l.num_sms, prm);
    if (!c.swapped) return launch<kI8, 1, 64, 1, false, false, true>(l.stream, l.num_sms, prm);
    switch (c.bn) {
    case 16: return launch<kI8, 1, 16, 2, false, false, true>(l.stream, l.num_sms, prm);
    case 32: return launch<kI8, 1, 32, 2, false, false, true>(l.stream, l.num_sms, prm);
    default: return launch<kI8, 1, 64, 2, false, false, true>(l.stream, l.num_sms, prm);
    }
}

}  // namespace gvq
