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
    const Cut c = cut(l.num_sms, M, N, false, stages_of(K, kI8));
    prm.M = c.few ? N : M;
    prm.N = c.few ? M : N;
    divide(prm, c, kI8, false, K, 1, 1);
    prm.scale_m[0] = c.few ? sb : sa;
    prm.scale_n[0] = c.few ? sa : sb;
    if (!encode_codes(l.encode, &prm.a[0], c.few ? b : a, prm.M, K, prm.rows_a) ||
        !encode_codes(l.encode, &prm.b[0], c.few ? a : b, prm.N, K, c.bn / c.cg))
        return cudaErrorInvalidValue;
    set_output(prm, 0, out, dtype, ld);
    const cudaStream_t st = l.stream;
    if (c.few) {
        switch (c.bn) {
        case 16: return launch<kI8, 1, 16, true, false, false, false>(st, l.num_sms, prm);
        case 32: return launch<kI8, 1, 32, true, false, false, false>(st, l.num_sms, prm);
        default: return launch<kI8, 1, 64, true, false, false, false>(st, l.num_sms, prm);
        }
    }
    switch (c.bn) {
    case 256: return launch<kI8, 2, 256, false, false, false, false>(st, l.num_sms, prm);
    case 128: return launch<kI8, 2, 128, false, false, false, false>(st, l.num_sms, prm);
    default: return launch<kI8, 1, 64, false, false, false, false>(st, l.num_sms, prm);
    }
}

cudaError_t launch_i8_gated(const Launch &l, const int8_t *a, const float *sa, const int8_t *gate, const float *s_gate, const int8_t *up,
                            const float *s_up, int64_t M, int64_t F, int64_t K, int act, void *out, int dtype, int64_t ld)
{
    Params prm = start(l, dtype);
    prm.act = act;
    const Cut c = cut(l.num_sms, M, F, true, stages_of(K, kI8));
    prm.M = c.few ? F : M;
    prm.N = c.few ? M : F;
    divide(prm, c, kI8, true, K, 1, 1);
    const int8_t *w[2] = {gate, up};
    const float *sw[2] = {s_gate, s_up};
    CUtensorMap *map_w = c.few ? prm.a : prm.b;
    for (int i = 0; i < 2; ++i) {
        (c.few ? prm.scale_m : prm.scale_n)[i] = sw[i];
        if (!encode_codes(l.encode, map_w + i, w[i], F, K, c.few ? prm.rows_a : c.bn / 2)) return cudaErrorInvalidValue;
    }
    (c.few ? prm.scale_n : prm.scale_m)[0] = sa;
    if (!encode_codes(l.encode, c.few ? prm.b : prm.a, a, M, K, c.few ? c.bn : 128)) return cudaErrorInvalidValue;
    set_output(prm, 0, out, dtype, ld);
    const cudaStream_t st = l.stream;
    if (c.few) {
        switch (c.bn) {
        case 16: return launch<kI8, 1, 16, true, false, false, true>(st, l.num_sms, prm);
        case 32: return launch<kI8, 1, 32, true, false, false, true>(st, l.num_sms, prm);
        default: return launch<kI8, 1, 64, true, false, false, true>(st, l.num_sms, prm);
        }
    }
    switch (c.bn) {
    case 256: return launch<kI8, 2, 256, false, false, false, true>(st, l.num_sms, prm);
    case 128: return launch<kI8, 2, 128, false, false, false, true>(st, l.num_sms, prm);
    default: return launch<kI8, 1, 64, false, false, false, true>(st, l.num_sms, prm);
    }
}

}  // namespace gvq
