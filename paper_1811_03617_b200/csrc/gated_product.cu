// The gated feed-forward block in 16 bits (gvq.h, "the gated block"):  h = act(x Wg^T) * (x Wu^T).
#include "product.cuh"

namespace gvq {

using namespace product;

cudaError_t launch_gated(const Launch &l, const void *x, int64_t ldx, const void *gate, int64_t ld_gate, const void *up, int64_t ld_up,
                         int dtype, int64_t M, int64_t F, int64_t K, int act, void *h, int64_t ldh, void *g, int64_t ldg, void *u,
                         int64_t ldu)
{
    Params prm = {};
    prm.dtype = dtype;
    prm.bf16 = dtype == GVQ_BF16;
    prm.act = act;
    prm.error_word = l.error_word;
    prm.wait_kcycles = l.wait_kcycles > 0 ? l.wait_kcycles : WAIT_KCYCLES_DEFAULT;
    prm.test_drop = l.test_drop;
    const Cut c = cut(l.num_sms, M, F, true, stages_of(K, k16));
    prm.M = c.few ? F : M;
    prm.N = c.few ? M : F;
    divide(prm, c, k16, true, K, 1, 1);
    CUtensorMap *map_w = c.few ? prm.a : prm.b;
    const int box_w = c.few ? prm.rows_a : c.bn / 2;
    if (!encode(l.encode, map_w, k16, gate, F, K, ld_gate, box_w) || !encode(l.encode, map_w + 1, k16, up, F, K, ld_up, box_w) ||
        !encode(l.encode, c.few ? prm.b : prm.a, k16, x, M, K, ldx, c.few ? c.bn : 128))
        return cudaErrorInvalidValue;
    set_output(prm, 0, h, dtype, ldh);
    set_output(prm, 1, g, dtype, ldg);
    set_output(prm, 2, u, dtype, ldu);
    const cudaStream_t st = l.stream;
    if (c.few) {
        switch (c.bn) {
        case 16: return launch<k16, 1, 16, true, false, false, true>(st, l.num_sms, prm);
        case 32: return launch<k16, 1, 32, true, false, false, true>(st, l.num_sms, prm);
        default: return launch<k16, 1, 64, true, false, false, true>(st, l.num_sms, prm);
        }
    }
    switch (c.bn) {
    case 256: return launch<k16, 2, 256, false, false, false, true>(st, l.num_sms, prm);
    case 128: return launch<k16, 2, 128, false, false, false, true>(st, l.num_sms, prm);
    default: return launch<k16, 1, 64, false, false, false, true>(st, l.num_sms, prm);
    }
}

}  // namespace gvq
