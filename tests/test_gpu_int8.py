"""8-bit integers on the GPU against their definition in 64 bits: codes and scales bit for bit, products to the roundings that
follow an exact sum, and the refusals."""
import numpy as np
import pytest
import torch

import int8_reference as R

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}      # half a step, relative


@pytest.fixture(scope="module")
def ctx():
    from paper_1811_03617_b200 import gvq
    return gvq.Context(gvq.HostLayout(4, 4, [0], [4]))


def _values_like(rows, cols, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * 10 ** (4 * torch.rand(rows, 1, generator=g) - 3)
    if rows * cols >= 64:
        x.view(-1)[:4] = torch.tensor([0.0, -0.0, 127.0, -63.5])
    if rows > 2:
        x[1] = 0.0                                  # a row without a value
        x[2] = 1e-41                                # below the smallest scale
    if rows > 7 and cols > 40:
        x[3, 5], x[4, 7], x[5, 33], x[6, 1] = float("nan"), float("inf"), float("-inf"), torch.finfo(dtype).max
        x[6, 2] = torch.finfo(dtype).min
        x[7] = torch.arange(cols) % 255 / 2.0 - 63.5    # with a largest entry of 127: every other code is a tie
        x[7, 0] = 127.0
    return x.to(dtype)


def _check(q, x, stochastic=False, seed=0, node=0):
    codes, scales, _ = R.quantize(x, stochastic, seed, node)
    assert torch.equal(q.scales.cpu().view(torch.int32) & 0x7FC00000, scales.view(torch.int32) & 0x7FC00000)
    assert torch.equal(torch.nan_to_num(q.scales.cpu(), -1.0), torch.nan_to_num(scales, -1.0))
    assert torch.equal(q.codes.cpu(), codes)


SIZES = [(1, 1), (1, 15), (3, 16), (7, 64), (128, 128), (129, 130), (33, 515), (260, 77), (9, 1024), (10, 1040), (520, 2100), (1000, 4095), (2500, 1001)]


@pytest.mark.parametrize("stochastic", [False, True])
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("rows,cols", SIZES)
def test_codes_and_scales_bit_exact(ctx, rows, cols, dtype, stochastic):
    x = _values_like(rows, cols, DT[dtype], rows * 1000 + cols)
    kw = dict(stochastic=stochastic, seed=0x1234567890ABCDEF, node=3)
    q, qt = ctx.i8_quantize_both(x.cuda(), **kw)
    _check(q, x, **kw)
    _check(qt, x.t().contiguous(), **kw)
    one, other = ctx.i8_quantize(x.cuda(), **kw), ctx.i8_quantize_transposed(x.cuda(), **kw)
    for a, b in ((one, q), (other, qt)):
        assert torch.equal(a.codes, b.codes) and torch.equal(a.scales.view(torch.int32), b.scales.view(torch.int32))
    values = R.quantize(x, **kw)[2]
    got = ctx.i8_dequantize(q).cpu().double().numpy()      # code * scale, rounded to float32 once
    assert np.array_equal(got, values.astype(np.float32).astype(np.float64), equal_nan=True)


@pytest.mark.parametrize("stochastic", [False, True])
@pytest.mark.parametrize("rows,cols", [(2, 5000), (600, 4096), (3, 9001), (131, 16384), (3, 33000), (2, 70001), (20000, 24), (17000, 3)])
def test_long_rows_and_columns_bit_exact(ctx, rows, cols, stochastic):
    """Rows that more than a warp shares, rows that do not stay in registers, columns of many blocks."""
    x = torch.randn(rows, cols, generator=torch.Generator().manual_seed(cols)).to(torch.bfloat16)
    kw = dict(stochastic=stochastic, seed=77, node=1)
    q, qt = ctx.i8_quantize_both(x.cuda(), **kw)
    _check(q, x, **kw)
    _check(qt, x.t().contiguous(), **kw)
    one = ctx.i8_quantize(x.cuda(), **kw)
    assert torch.equal(one.codes, q.codes) and torch.equal(one.scales, q.scales)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("offset,pad", [(0, 1), (1, 0), (3, 5), (8, 8)])
def test_strides_and_alignment(ctx, dtype, offset, pad):
    rows, cols = 131, 165
    x = _values_like(rows, cols, DT[dtype], 5)
    buf = torch.full((offset + rows * (cols + pad),), float("nan"), dtype=DT[dtype], device="cuda")
    view = torch.as_strided(buf, (rows, cols), (cols + pad, 1), offset)
    view.copy_(x)
    q, qt = ctx.i8_quantize_both(view)
    _check(q, x)
    _check(qt, x.t().contiguous())
    _check(ctx.i8_quantize(view), x)
    out = torch.full((rows, cols + pad), 7.0, device="cuda")
    ctx.i8_dequantize(q, out[:, :cols])
    assert bool((out[:, cols:] == 7.0).all())
    assert torch.equal(torch.nan_to_num(out[:, :cols]), torch.nan_to_num(ctx.i8_dequantize(q)))


@pytest.mark.parametrize("rows,both", [(310, True), (320, False), (336, True)])
def test_first_call_of_a_process_with_nearly_48_kb_of_shared_memory(rows, both):
    """The strips' shared memory and the kernel's own arrays are together more than a kernel has without asking."""
    import subprocess
    import sys
    from pathlib import Path
    code = f"""import torch
from paper_1811_03617_b200 import gvq
ctx = gvq.Context(gvq.HostLayout(4, 4, [0], [4]))
x = torch.randn({rows}, 200, device="cuda", dtype=torch.bfloat16)
q = ctx.i8_quantize_both(x)[1] if {both} else ctx.i8_quantize_transposed(x)
assert torch.equal(q.codes, ctx.i8_quantize(x.t().contiguous()).codes)
"""
    subprocess.run([sys.executable, "-c", code], check=True, cwd=Path(__file__).resolve().parent.parent, timeout=300)


def test_stochastic_rounding_is_unbiased(ctx):
    """4096 roundings of one step have a standard error of at most step / 2 / 64; five of them, the 2^-14 of a step that u
    leaves, and what rounding the scale and the factor to 24 bits moves 127 steps by."""
    n, step = 4096, 6.0 / 127
    x = torch.linspace(-6, 6, 64, device="cuda").repeat(n, 1)
    mean = ctx.i8_dequantize(ctx.i8_quantize(x, stochastic=True, seed=9)).double().mean(0)
    assert bool(((mean - x[0].double()).abs() <= step * (5 * 0.5 / n ** 0.5 + 2.0 ** -14 + 127 * 2.0 ** -22)).all())


def _held(want, dtype):
    """The bound of a result whose sum is exact: converting it to float32 and either scale's product round once each, the output
    once; what lies below the type's smallest step is off by half of that."""
    return want.abs() * (3.01 * 2.0 ** -24 + HALF[dtype]) + (2.0 ** -25 if dtype == torch.float16 else 2.0 ** -126)


def _product(ctx, m, n, k, dtype, pad=0):
    g = torch.Generator(device="cuda").manual_seed(m + n + k)
    a = torch.randn(m, k, generator=g, device="cuda") * 2.0 ** torch.randint(-9, 10, (m, 1), generator=g, device="cuda")
    b = torch.randn(n, k, generator=g, device="cuda") * 2.0 ** torch.randint(-9, 4, (n, 1), generator=g, device="cuda")
    qa, qb = ctx.i8_quantize(a), ctx.i8_quantize(b)
    buf = torch.full((m, n + pad), 3.0, dtype=DT[dtype], device="cuda")
    ctx.i8_matmul(qa, qb, buf[:, :n])
    ctx.device_status()
    sums = qa.codes[:, :k].double() @ qb.codes[:, :k].double().T
    want = sums * qa.scales.double()[:, None] * qb.scales.double()
    bound = _held(want, DT[dtype])
    near = want.abs() + bound < float(torch.finfo(DT[dtype]).max)
    assert bool(near.any())
    assert bool(((buf[:, :n].double() - want).abs() <= bound)[near].all())
    assert bool((buf[:, n:] == 3.0).all())
    again = torch.empty(m, n, dtype=DT[dtype], device="cuda")
    ctx.i8_matmul(qa, qb, again)
    assert torch.equal(again, buf[:, :n])


@pytest.mark.parametrize("m,n,k,dtype,pad", [
    (1, 1, 1, "f32", 0), (1, 7, 33, "bf16", 0), (1, 128, 64, "f32", 0), (2, 130, 2048, "bf16", 0), (16, 300, 96, "f16", 1),
    (17, 129, 700, "f32", 0), (33, 64, 256, "bf16", 3), (64, 1000, 1024, "f32", 0), (65, 65, 65, "f32", 1), (128, 256, 256, "f32", 0),
    (129, 257, 128, "bf16", 0), (200, 515, 1083, "bf16", 5), (385, 1029, 4100, "f32", 0), (1000, 33, 31, "f16", 0)])
def test_product(ctx, m, n, k, dtype, pad):
    _product(ctx, m, n, k, dtype, pad)


@pytest.mark.parametrize("m,n,k,dtype,pad", [
    (1664, 1600, 256, "bf16", 0), (1601, 1611, 1300, "f32", 5), (1700, 1537, 96, "f16", 7), (2304, 2056, 640, "f32", 0),
    (4100, 3000, 2048, "bf16", 8), (1537, 4000, 4128, "bf16", 0)])
def test_large_product(ctx, m, n, k, dtype, pad):
    """Enough 256 x 256 tiles for pairs of CTAs."""
    _product(ctx, m, n, k, dtype, pad)


# Tiles whose contraction a cluster of CTAs shares (2, 4 and 8 parts, the few rows on either side of the tile)
@pytest.mark.parametrize("m,n,k,dtype,pad", [
    (1, 500, 2064, "bf16", 0), (3, 4000, 1100, "f32", 1), (16, 1000, 1283, "f32", 3), (31, 129, 2000, "f16", 1),
    (32, 2049, 5000, "bf16", 8), (33, 70, 8200, "f32", 0), (64, 1000, 4133, "bf16", 8), (100, 300, 4300, "bf16", 5),
    (65, 64, 16500, "f32", 4), (128, 61, 17000, "f16", 8), (150, 260, 4224, "bf16", 4)])
def test_product_of_few_rows_with_a_long_contraction(ctx, m, n, k, dtype, pad):
    _product(ctx, m, n, k, dtype, pad)


@pytest.mark.parametrize("m,n,k,dtype,pad", [
    (1, 19000, 33, "f32", 0), (5, 40001, 160, "bf16", 3), (16, 57000, 1100, "f16", 0), (32, 60003, 257, "bf16", 5),
    (33, 9601, 500, "f32", 0), (64, 45777, 96, "f32", 7)])
def test_product_of_few_rows_with_more_tiles_than_ctas(ctx, m, n, k, dtype, pad):
    _product(ctx, m, n, k, dtype, pad)


@pytest.mark.parametrize("m", [1, 40, 200])
def test_the_longest_contraction_of_the_largest_codes_is_exact(ctx, m):
    """131072 products of 127 x 127: 2114060288, which 32 bits hold; of both signs."""
    k, n = 131072, 130
    a, b = torch.ones(m, k, device="cuda"), torch.ones(n, k, device="cuda")
    b[1::2] = -1
    out = ctx.i8_matmul(ctx.i8_quantize(a), ctx.i8_quantize(b), torch.empty(m, n, device="cuda"))
    ctx.device_status()
    want = torch.full((m, n), float(k * 127 * 127), device="cuda").double() * float(np.float32(1 / 127.0)) ** 2
    want[:, 1::2] *= -1
    assert bool(((out.double() - want).abs() <= _held(want, torch.float32)).all())


@pytest.mark.parametrize("m", [3, 150])
def test_product_writes_inside_the_output_only(ctx, m):
    n, k = 261, 513
    qa, qb = ctx.i8_quantize(torch.randn(m, k).cuda()), ctx.i8_quantize(torch.randn(n, k).cuda())
    for dtype in DT.values():
        buf = torch.full((m + 2, n + 9), 3.0, dtype=dtype, device="cuda")
        ctx.i8_matmul(qa, qb, buf[1:m + 1, 4:n + 4])
        again = torch.empty(m, n, dtype=dtype, device="cuda")
        ctx.i8_matmul(qa, qb, again)
        assert torch.equal(buf[1:m + 1, 4:n + 4], again)
        buf[1:m + 1, 4:n + 4] = 3.0
        assert bool((buf == 3.0).all())


@pytest.mark.parametrize("m", [5, 140, 700])
def test_rows_that_stand_for_nan_make_their_own_results_nan(ctx, m):
    n, k = 500, 200
    a, b = torch.randn(m, k), torch.randn(n, k)
    a[1, 70], b[2, 3] = float("inf"), float("nan")
    out = ctx.i8_matmul(ctx.i8_quantize(a.cuda()), ctx.i8_quantize(b.cuda()), torch.empty(m, n, device="cuda")).cpu()
    want = torch.zeros(m, n, dtype=torch.bool)
    want[1], want[:, 2] = True, True
    assert torch.equal(torch.isnan(out), want)


def test_weights_that_a_program_keeps(ctx):
    """Codes and scales as tensors of one's own."""
    from paper_1811_03617_b200 import gvq
    x, w = torch.randn(5, 70, device="cuda"), torch.randn(33, 70)
    codes, scales, _ = R.quantize(w)
    mine = gvq.I8(33, 70, codes.cuda(), scales.cuda())
    a = ctx.i8_matmul(ctx.i8_quantize(x), mine, torch.empty(5, 33, device="cuda"))
    b = ctx.i8_matmul(ctx.i8_quantize(x), ctx.i8_quantize(w.cuda()), torch.empty(5, 33, device="cuda"))
    assert torch.equal(a, b)


def test_gradients_of_a_linear_layer(ctx):
    """With operands that are whole numbers up to 127, 127 in every row and column, the layer is y = x W^T up to the roundings of
    its scales, so dx and dW are the formula's, and L = sum(dy * y) has them as its differences."""
    t, i, o = 96, 64, 160
    g = torch.Generator().manual_seed(3)

    def whole(r, c):
        v = torch.randint(-127, 128, (r, c), generator=g).float()
        v[:, 0], v[0, :] = 127.0, 127.0
        return v
    x, w, dy = whole(t, i), whole(o, i), whole(t, o)
    qdy, qdy_t = ctx.i8_quantize_both(dy.cuda(), stochastic=True, seed=1)
    dx = ctx.i8_matmul(qdy, ctx.i8_quantize_transposed(w.cuda()), torch.empty(t, i, device="cuda")).cpu().double()
    dw = ctx.i8_matmul(qdy_t, ctx.i8_quantize_transposed(x.cuda()), torch.empty(o, i, device="cuda")).cpu().double()
    assert torch.equal(dx, dy.double() @ w.double()) and torch.equal(dw, dy.double().T @ x.double())     # (a scale of 127 / 127)

    def loss(x, w):
        y = ctx.i8_matmul(ctx.i8_quantize(x.cuda()), ctx.i8_quantize(w.cuda()), torch.empty(t, o, device="cuda"))
        return float((y.cpu().double() * dy.double()).sum())
    for (r, c) in ((5, 7), (40, 33)):
        up, down = x.clone(), x.clone()
        up[r, c], down[r, c] = 2.0, -2.0
        assert loss(up, w) - loss(down, w) == 4.0 * float(dx[r, c])
        up, down = w.clone(), w.clone()
        up[r, c], down[r, c] = 1.0, -1.0
        assert loss(x, up) - loss(x, down) == 2.0 * float(dw[r, c])


def test_calls_follow_their_stream_and_can_be_captured(ctx):
    from paper_1811_03617_b200 import gvq
    x, w = torch.randn(70, 128, device="cuda"), torch.randn(96, 128, device="cuda")
    qx, qw, qt, y = gvq.I8(70, 128), gvq.I8(96, 128), gvq.I8(128, 70), torch.empty(70, 96, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.i8_quantize_both(x, out=qx, out_t=qt)
        ctx.i8_quantize(w, out=qw)
        ctx.i8_matmul(qx, qw, y)
    x.copy_(torch.randn(70, 128))
    graph.replay()
    torch.cuda.synchronize()
    eager = ctx.i8_matmul(ctx.i8_quantize(x), ctx.i8_quantize(w), torch.empty(70, 96, device="cuda"))
    assert torch.equal(y, eager) and torch.equal(qt.codes, ctx.i8_quantize_transposed(x).codes)
    side = torch.cuda.Stream()
    late = torch.empty_like(x)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        big = torch.randn(4096, 4096, device="cuda")
        for _ in range(4):
            big = big @ big * 1e-4
        late.copy_(x)
        out = ctx.i8_matmul(ctx.i8_quantize(late), ctx.i8_quantize(w), torch.empty(70, 96, device="cuda"))
    side.synchronize()
    assert torch.equal(out, eager)


@pytest.mark.parametrize("m,n,k", [(200, 300, 600), (16, 500, 4128), (100, 300, 8200), (1700, 1600, 300)])
def test_a_wait_that_runs_out_is_reported_and_the_context_recovers(ctx, m, n, k):
    from paper_1811_03617_b200 import gvq
    qa, qb = ctx.i8_quantize(torch.randn(m, k, device="cuda")), ctx.i8_quantize(torch.randn(n, k, device="cuda"))
    out = torch.empty(m, n, device="cuda")
    good = ctx.i8_matmul(qa, qb, out).clone()
    ctx.set_limits(wait_cycles=2_000_000)
    ctx.test_drop_load(True)
    try:
        ctx.i8_matmul(qa, qb, out)
        with pytest.raises(gvq.GvqError) as e:
            ctx.device_status()
        assert e.value.status == 9
    finally:
        ctx.test_drop_load(False)
        ctx.set_limits()
    assert torch.equal(ctx.i8_matmul(qa, qb, out), good)
    ctx.device_status()


@pytest.mark.parametrize("dtype", list(DT))
def test_outputs_at_any_place(ctx, dtype):
    """Every offset within a sector and every width of a strip's last piece, exactly: sums of whole numbers below 2^8."""
    t = DT[dtype]
    for m, n in ((130, 1), (130, 2), (130, 13), (130, 31), (130, 33), (260, 63), (260, 200), (2100, 1031), (2100, 1048)):
        k = 16
        g = torch.Generator().manual_seed(n)
        a, b = (torch.randint(-3, 4, (r, k), generator=g, dtype=torch.int8).cuda() for r in (m, n))
        from paper_1811_03617_b200 import gvq
        qa, qb = gvq.I8(m, k, a, torch.ones(m, device="cuda")), gvq.I8(n, k, b, torch.ones(n, device="cuda"))
        want = (a.double() @ b.double().T).to(t)
        for offset, pad in ((0, 0), (1, 0), (0, 1), (3, 2), (8, 8), (5, 16), (2, 4), (16, 7)):
            buf = torch.full((offset + m * (n + pad) + 64,), 77.0, dtype=t, device="cuda")
            out = torch.as_strided(buf, (m, n), (n + pad, 1), offset)
            ctx.i8_matmul(qa, qb, out)
            assert torch.equal(out, want), (m, n, offset, pad)
            out.fill_(77.0)
            assert bool((buf == 77.0).all()), (m, n, offset, pad)
