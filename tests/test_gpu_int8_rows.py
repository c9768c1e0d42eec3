"""A row's results do not depend on how many rows come with it, bit for bit: the sums of codes are exact, and the scales are applied in
one order in every form of the kernel."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_1811_03617_b200 import gvq
    return gvq.Context(gvq.HostLayout(4, 4, [0], [4]))


# the weights' outputs and the contraction: narrow, a contraction that a cluster shares, wide
@pytest.mark.parametrize("N,K", [(257, 100), (130, 8200), (5000, 515)])
def test_a_row_has_the_same_bits_among_any_number_of_rows(ctx, N, K):
    from paper_1811_03617_b200 import gvq
    g = torch.Generator().manual_seed(N)
    x, w, v = (torch.randn(r, K, generator=g) * 2.0 ** torch.randint(-3, 3, (r, 1), generator=g) for r in (700, N, N))
    qx, qw, qv = (ctx.i8_quantize(t.cuda()) for t in (x, w, v))

    def some(rows):
        return gvq.I8(rows, K, qx.codes[:rows].contiguous(), qx.scales[:rows].contiguous())

    def product(rows):
        return ctx.i8_matmul(some(rows), qw, torch.empty(rows, N, device="cuda"))

    def block(rows):
        return ctx.i8_gated(some(rows), qw, qv, torch.empty(rows, N, device="cuda"), act="silu")
    for of in (product, block):
        whole = of(700)
        for rows in (1, 7, 16, 17, 40, 64, 65, 130, 300):
            part = of(rows)
            assert torch.equal(part, whole[:rows]), (of.__name__, rows, int((part != whole[:rows]).sum()))
    ctx.device_status()
    # the order that is stated: whole number, a's scale, b's scale
    y = product(5)
    s = (qx.codes[:5, :K].double() @ qw.codes[:, :K].double().T).float()
    assert torch.equal(y, s * qx.scales[:5, None] * qw.scales)
