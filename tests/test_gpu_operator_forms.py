"""Forms of the 4-bit product and of the orthogonalised update that only certain sizes reach: more tiles than CTAs with few
rows, outputs of one column, captures and side streams of an update that takes a launch per product."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def ctx():
    from paper_1811_03617_b200 import gvq
    return gvq.Context(gvq.HostLayout(4, 4, [0], [4]))


# Up to 32 rows against more than 148 x 128 rows of weights, 33 to 64 rows against more than 148 x 64: a CTA goes round its loop
# over tiles (two, three and more times, accumulators in turn).
@pytest.mark.parametrize("m,n,k,dtype,pad", [
    (1, 19000, 33, "f32", 0), (5, 20001, 160, "bf16", 3), (16, 57000, 1100, "f16", 0), (17, 38017, 64, "f32", 1),
    (32, 100003, 257, "bf16", 5), (33, 9601, 500, "f32", 0), (48, 30000, 1000, "bf16", 8), (64, 16384, 256, "f16", 0),
    (64, 75777, 96, "f32", 7)])
def test_product_of_few_rows_with_more_tiles_than_ctas(ctx, m, n, k, dtype, pad):
    g = torch.Generator(device="cuda").manual_seed(m + n)
    a = torch.randn(m, k, generator=g, device="cuda") * 2.0 ** torch.randint(-9, 10, (m, 1), generator=g, device="cuda")
    b = torch.randn(n, k, generator=g, device="cuda") * 2.0 ** torch.randint(-3, 4, (n, 1), generator=g, device="cuda")
    qa, qb = ctx.mx4_quantize(a), ctx.mx4_quantize(b)
    va, vb = ctx.mx4_dequantize(qa).double(), ctx.mx4_dequantize(qb).double()
    buf = torch.full((m, n + pad), 3.0, dtype=DT[dtype], device="cuda")
    ctx.mx4_matmul(qa, qb, buf[:, :n])
    ctx.device_status()
    # the tensor core adds the 64 products of a step into an fp32 accumulator, which it may truncate: 2^-22 of the magnitudes a
    # step, and the output's own rounding
    want, mag = va @ vb.T, va.abs() @ vb.abs().T
    half_ulp = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[DT[dtype]]
    bound = mag * (-(-k // 64) + 2) * 2.0 ** -22 + want.abs() * half_ulp + (6e-8 if dtype == "f16" else 0)
    near = want.abs() + bound < float(torch.finfo(DT[dtype]).max)
    assert bool(((buf[:, :n].double() - want).abs() <= bound)[near].all())
    assert bool((buf[:, n:] == 3.0).all())
    again = torch.empty(m, n, dtype=DT[dtype], device="cuda")
    ctx.mx4_matmul(qa, qb, again)
    assert torch.equal(again, buf[:, :n])


@pytest.mark.parametrize("m", [1, 7, 33, 64, 65, 200])
@pytest.mark.parametrize("dtype", list(DT))
def test_product_with_one_column(ctx, m, dtype):
    """Either side has a single row of codes; rows of the output are one entry apart."""
    k = 700
    a, b = torch.randn(m, k, device="cuda"), torch.randn(1, k, device="cuda")
    qa, qb = ctx.mx4_quantize(a), ctx.mx4_quantize(b)
    buf = torch.full((m + 16,), 3.0, dtype=DT[dtype], device="cuda")
    ctx.mx4_matmul(qa, qb, buf[8:m + 8].view(m, 1))
    ctx.device_status()
    va, vb = ctx.mx4_dequantize(qa).double(), ctx.mx4_dequantize(qb).double()
    want, mag = (va @ vb.T)[:, 0], (va.abs() @ vb.abs().T)[:, 0]
    half_ulp = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[DT[dtype]]
    assert bool(((buf[8:m + 8].double() - want).abs() <= mag * 13 * 2.0 ** -22 + want.abs() * half_ulp + 6e-8).all())
    assert bool((buf[:8] == 3.0).all()) and bool((buf[m + 8:] == 3.0).all())


def made(shapes):
    from paper_1811_03617_b200 import gvq
    lens = [m * n for m, n in shapes]
    off = [sum(-(-x // 4) * 4 for x in lens[:i]) for i in range(len(lens))]
    c = gvq.Context(gvq.HostLayout(64, 4, off, lens))
    return c, gvq.OrthoPlan(c, [m for m, _ in shapes], [n for _, n in shapes])


# a launch a product: 128 x 64 tiles (one matrix with parts of a contraction), and pairs of CTAs
LARGER = [[(300, 400), (40, 3000)], [(129, 2500)], [(1200, 2300), (1025, 1500), (1024, 1700)]]


@pytest.mark.parametrize("shapes", LARGER)
def test_an_update_of_larger_matrices_can_be_captured(shapes):
    c, plan = made(shapes)
    gen = torch.Generator(device="cuda").manual_seed(1)
    g, mo, w = (torch.randn(c.M, generator=gen, device="cuda") for _ in range(3))
    mo2, w2 = mo.clone(), w.clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(3):
            plan.step(g, mo2, w2, lr=0.1, weight_decay=0.01)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        plan.step(g, mo, w, lr=0.1, weight_decay=0.01)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(mo, mo2) and torch.equal(w, w2)
    # a replay reads what is there then
    g.copy_(torch.randn(c.M, generator=gen, device="cuda"))
    graph.replay()
    plan.step(g, mo2, w2, lr=0.1, weight_decay=0.01)
    torch.cuda.synchronize()
    assert torch.equal(mo, mo2) and torch.equal(w, w2)


@pytest.mark.parametrize("shapes", LARGER)
def test_an_update_of_larger_matrices_follows_its_stream(shapes):
    """Inputs that a side stream is still making; the result is read after that stream alone is waited for."""
    c, plan = made(shapes)
    gen = torch.Generator(device="cuda").manual_seed(2)
    g = torch.randn(c.M, generator=gen, device="cuda")
    want, out, late = torch.zeros(c.M, device="cuda"), torch.zeros(c.M, device="cuda"), torch.zeros(c.M, device="cuda")
    plan.orthogonalize(g, want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        big = torch.randn(4096, 4096, device="cuda")
        for _ in range(6):
            big = big @ big * 1e-4
        late.copy_(g)
        plan.orthogonalize(late, out)
    side.synchronize()
    c.device_status()
    assert torch.equal(out, want)
