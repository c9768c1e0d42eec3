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
    const Cut c = cut(l.num_sms, M, F, 32);
    prm.M = c.swapped ? F : M;
    prm.N = c.swapped ? M : F;
    divide(prm, l.num_sms, c, k16, c.swapped ? c.bn : c.bn / 2, K, 1, 1);
    CUtensorMap *map_w = c.swapped ? prm.a : prm.b;
    const int box_w = c.swapped || c.cg == 2 ? 128 : 32;
    if (!encode(l.encode, map_w, k16, gate, F, K, ld_gate, box_w) || !encode(l.encode, map_w + 1, k16, up, F, K, ld_up, box_w) ||
        !encode(l.encode, c.swapped ? prm.b : prm.a, k16, x, M, K, ldx, c.swapped ? c.bn : 128))
        return cudaErrorInvalidValue;
    set_output(l.encode, prm, 0, h, dtype, M, F, ldh);
    set_output(l.encode, prm, 1, g, dtype, M, F, ldg);
    set_output(l.encode, prm, 2, u, dtype, M, F, ldu);
    if (c.cg == 2) return launch<k16, 2, 256, 1, false, false, true>(l.stream, l.num_sms, prm);
    if (!c.swapped) return launch<k16, 1, 64, 1, false, false, true>(l.stream, l.num_sms, prm);
    switch (c.bn) {
    case 16: return launch<k16, 1, 16, 2, false, false, true>(l.stream, l.num_sms, prm);
    case 32: return launch<k16, 1, 32, 2, false, false, true>(l.stream, l.num_sms, prm);
    default: return launch<k16, 1, 64, 2, false, false, true>(l.stream, l.num_sms, prm);
    }
}

}  // namespace gvq
