"""Microscaled 4-bit floating point on the GPU against its definition in 64 bits: codes and scales bit for bit, products
to the bound of their accumulation, the exchange over nodes, and the refusals."""
import numpy as np
import pytest
import torch

import mx4_reference as R
from paper_1811_03617_b200 import workloads as W

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def ctx():
    from paper_1811_03617_b200 import gvq
    return gvq.Context(gvq.HostLayout(4, 4, [0], [4]))


def _values_like(rows, cols, dtype, seed, special=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * 10 ** (4 * torch.rand(rows, 1, generator=g) - 3)
    if special and rows * cols >= 64:
        f = x.view(-1)
        f[0], f[1], f[2] = 0.0, -0.0, 6.0
        f[3:11] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -5.0])    # ties under a scale of 1
        if rows > 2:
            x[1] = 0.0                                  # a row without a value
            x[2] = 1e-41                                # below the smallest scale
            x[2, 0] = -3e-39
        if rows > 6 and cols > 40:
            x[3, 5], x[4, 7], x[5, 33], x[6, 1] = float("nan"), float("inf"), float("-inf"), torch.finfo(dtype).max
            x[6, 2] = torch.finfo(dtype).min
    return x.to(dtype)


def _check_quantized(q, x, stochastic, seed, node):
    codes, scales, _ = R.quantize(x, stochastic, seed, node)
    pc, ps = R.pack(codes, scales)
    assert torch.equal(q.scales.cpu(), ps)
    assert torch.equal(q.codes.cpu(), pc)


@pytest.mark.parametrize("stochastic", [False, True])
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 31), (3, 32), (7, 64), (128, 128), (129, 130), (33, 515), (260, 77)])
def test_codes_and_scales_bit_exact(ctx, rows, cols, dtype, stochastic):
    x = _values_like(rows, cols, DT[dtype], rows * 1000 + cols)
    seed, node = 0x1234567890ABCDEF, 3
    q, qt = ctx.mx4_quantize_both(x.cuda(), stochastic=stochastic, seed=seed, node=node)
    _check_quantized(q, x, stochastic, seed, node)
    _check_quantized(qt, x.t().contiguous(), stochastic, seed, node)
    one = ctx.mx4_quantize(x.cuda(), stochastic=stochastic, seed=seed, node=node)
    other = ctx.mx4_quantize_transposed(x.cuda(), stochastic=stochastic, seed=seed, node=node)
    assert torch.equal(one.codes, q.codes) and torch.equal(one.scales, q.scales)
    assert torch.equal(other.codes, qt.codes) and torch.equal(other.scales, qt.scales)
    # what the codes stand for, exactly
    v = R.quantize(x, stochastic, seed, node)[2]
    got = ctx.mx4_dequantize(q).cpu().double().numpy()
    assert np.array_equal(got, v.astype(np.float32).astype(np.float64), equal_nan=True)


@pytest.mark.parametrize("stochastic", [False, True])
@pytest.mark.parametrize("rows,cols", [(3, 33000), (5, 65600), (40000, 8)])
def test_long_rows_and_columns_bit_exact(ctx, rows, cols, stochastic):
    """Rows of more than 1024 blocks, which are shared among CTAs, and their padding."""
    x = torch.randn(rows, cols, generator=torch.Generator().manual_seed(cols)).to(torch.bfloat16)
    q = ctx.mx4_quantize(x.cuda(), stochastic=stochastic, seed=77, node=1)
    _check_quantized(q, x, stochastic, 77, 1)
    qt = ctx.mx4_quantize_transposed(x.cuda(), stochastic=stochastic, seed=77, node=1)
    _check_quantized(qt, x.t().contiguous(), stochastic, 77, 1)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("offset,pad", [(0, 1), (1, 0), (3, 5), (8, 8)])
def test_strides_and_alignment(ctx, dtype, offset, pad):
    rows, cols = 131, 165
    x = _values_like(rows, cols, DT[dtype], 5)
    buf = torch.full((offset + rows * (cols + pad),), float("nan"), dtype=DT[dtype], device="cuda")
    view = torch.as_strided(buf, (rows, cols), (cols + pad, 1), offset)
    view.copy_(x)
    q, qt = ctx.mx4_quantize_both(view)
    _check_quantized(q, x, False, 0, 0)
    _check_quantized(qt, x.t().contiguous(), False, 0, 0)
    out = torch.full((rows, cols + pad), 7.0, device="cuda")
    ctx.mx4_dequantize(q, out[:, :cols])
    assert bool((out[:, cols:] == 7.0).all())
    assert torch.equal(torch.nan_to_num(out[:, :cols]), torch.nan_to_num(ctx.mx4_dequantize(q)))


def test_stochastic_rounding_is_unbiased(ctx):
    """The mean over independent roundings approaches the entry: 4096 roundings of one step have a standard error of at
    most step / 2 / 64; five of them and the 2^-16 of a step that u leaves."""
    x = torch.linspace(-6, 6, 64, device="cuda").repeat(1, 1)
    total = torch.zeros(1, 64, dtype=torch.float64, device="cuda")
    n = 4096
    big = x.repeat(n, 1).contiguous()
    total = ctx.mx4_dequantize(ctx.mx4_quantize(big, stochastic=True, seed=9)).double().mean(0)
    r = x[0].abs()
    step = torch.where(r < 2, 0.5, torch.where(r < 4, 1.0, 2.0)).double()
    assert bool(((total - x[0].double()).abs() <= step * (5 * 0.5 / n ** 0.5 + 2.0 ** -16)).all())


# The tensor core adds the 64 products of a step into an fp32 accumulator, which it may truncate: every step may lose
# 2^-22 of the sum of magnitudes.  The output's own rounding comes on top.
def _product_bound(a, b, dtype):
    k = a.shape[1]
    mag = np.abs(a) @ np.abs(b).T
    half_ulp = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[dtype]
    return mag * (-(-k // 64) + 2) * 2.0 ** -22 + np.abs(a @ b.T) * half_ulp + (6e-8 if dtype == torch.float16 else 0)


@pytest.mark.parametrize("m,n,k,dtype", [
    (1, 1, 1, "f32"), (1, 7, 33, "bf16"), (1, 128, 64, "f32"), (2, 130, 2048, "bf16"), (16, 300, 96, "f16"),
    (17, 129, 700, "f32"), (33, 64, 256, "bf16"), (64, 1000, 1024, "f32"), (65, 65, 65, "f32"), (128, 256, 256, "f32"),
    (129, 257, 128, "bf16"), (200, 515, 1083, "bf16"), (385, 1029, 4100, "f32"), (1000, 33, 31, "f16"),
    (130, 1500, 2300, "f32"), (1300, 390, 160, "bf16")])
def test_product(ctx, m, n, k, dtype):
    g = torch.Generator().manual_seed(m + n + k)
    # scales that differ from block to block, so that a scale applied to the wrong block shows
    a = torch.randn(m, k, generator=g) * 2.0 ** torch.randint(-6, 7, (m, k), generator=g)
    b = torch.randn(n, k, generator=g) * 2.0 ** torch.randint(-6, 7, (n, k), generator=g)
    for t in (a, b):
        for j in range(0, k, 32):
            t[:, j:j + 32] *= 2.0 ** torch.randint(-8, 9, (t.shape[0], 1), generator=g)
    qa, qb = ctx.mx4_quantize(a.cuda()), ctx.mx4_quantize(b.cuda())
    va, vb = R.quantize(a)[2], R.quantize(b)[2]
    out = torch.full((m, n), float("nan"), dtype=DT[dtype], device="cuda")
    ctx.mx4_matmul(qa, qb, out)
    ctx.device_status()
    want, got = va @ vb.T, out.cpu().double().numpy()
    bound = _product_bound(va, vb, DT[dtype])
    top = float(torch.finfo(DT[dtype]).max)      # beyond it the rounded result is an infinity of the value's sign
    over = np.abs(want) - bound > top * (1 + 2.0 ** -11)
    assert np.array_equal(got[over], np.sign(want[over]) * np.inf)
    near = over | (np.abs(want) + bound >= top)
    err = np.abs(got - want)[~near]
    assert (err <= bound[~near]).all(), float((err / bound[~near]).max())


@pytest.mark.parametrize("m,n,k,dtype,pad", [
    (1664, 1600, 256, "bf16", 0), (1601, 1611, 1300, "f32", 5), (1700, 1537, 96, "f16", 7), (2304, 2056, 640, "f32", 0),
    (4100, 3000, 2048, "bf16", 8), (1537, 4000, 4128, "bf16", 0)])
def test_large_product(ctx, m, n, k, dtype, pad):
    """Enough 256 x 256 tiles for pairs of CTAs; codes and scales made on the GPU (tested bit for bit above), the product
    against float64 of what they stand for."""
    g = torch.Generator(device="cuda").manual_seed(m)
    a = torch.randn(m, k, generator=g, device="cuda") * 2.0 ** torch.randint(-9, 10, (m, 1), generator=g, device="cuda")
    b = torch.randn(n, k, generator=g, device="cuda")
    for t in (a, b):
        for j in range(0, k, 32):
            t[:, j:j + 32] *= 2.0 ** torch.randint(-6, 7, (t.shape[0], 1), generator=g, device="cuda")
    qa, qb = ctx.mx4_quantize(a), ctx.mx4_quantize(b)
    va, vb = ctx.mx4_dequantize(qa).double(), ctx.mx4_dequantize(qb).double()
    buf = torch.full((m, n + pad), 3.0, dtype=DT[dtype], device="cuda")
    ctx.mx4_matmul(qa, qb, buf[:, :n])
    ctx.device_status()
    want, mag = va @ vb.T, va.abs() @ vb.abs().T
    half_ulp = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[DT[dtype]]
    bound = mag * (-(-k // 64) + 2) * 2.0 ** -22 + want.abs() * half_ulp + (6e-8 if dtype == "f16" else 0)
    near = want.abs() + bound < float(torch.finfo(DT[dtype]).max)
    assert bool(((buf[:, :n].double() - want).abs() <= bound)[near].all())
    assert bool((buf[:, n:] == 3.0).all())
    again = torch.empty(m, n, dtype=DT[dtype], device="cuda")
    ctx.mx4_matmul(qa, qb, again)
    assert torch.equal(again, buf[:, :n])


# Tiles of few rows whose contraction a cluster of CTAs shares (2, 4 and 8 parts, with the few rows on either side of the
# tile), last stages that are short, rows of the output that do not start at 16-byte boundaries, tiles that stick out.
@pytest.mark.parametrize("m,n,k,dtype,pad", [
    (1, 500, 4128, "bf16", 0), (3, 4000, 1100, "f32", 1), (16, 1000, 1283, "f32", 3), (31, 129, 2000, "f16", 1),
    (32, 2049, 5000, "bf16", 8), (33, 70, 8200, "f32", 0), (64, 1000, 4133, "bf16", 8), (100, 300, 4300, "bf16", 5),
    (65, 64, 16500, "f32", 4), (128, 61, 17000, "f16", 8), (150, 260, 4224, "bf16", 4)])
def test_product_of_few_rows_with_a_long_contraction(ctx, m, n, k, dtype, pad):
    g = torch.Generator(device="cuda").manual_seed(m + n)
    a = torch.randn(m, k, generator=g, device="cuda") * 2.0 ** torch.randint(-9, 10, (m, 1), generator=g, device="cuda")
    b = torch.randn(n, k, generator=g, device="cuda")
    b[:, k // 2:] *= 2.0 ** torch.randint(-3, 4, (n, 1), generator=g, device="cuda")
    qa, qb = ctx.mx4_quantize(a), ctx.mx4_quantize(b)
    va, vb = ctx.mx4_dequantize(qa).double(), ctx.mx4_dequantize(qb).double()
    buf = torch.full((m, n + pad), 3.0, dtype=DT[dtype], device="cuda")
    ctx.mx4_matmul(qa, qb, buf[:, :n])
    ctx.device_status()
    # the bound of the other products: adding up to eight parts loses less than the steps that each part does not take
    want, mag = va @ vb.T, va.abs() @ vb.abs().T
    half_ulp = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[DT[dtype]]
    bound = mag * (-(-k // 64) + 2) * 2.0 ** -22 + want.abs() * half_ulp + (6e-8 if dtype == "f16" else 0)
    near = want.abs() + bound < float(torch.finfo(DT[dtype]).max)
    assert bool(((buf[:, :n].double() - want).abs() <= bound)[near].all())
    assert bool((buf[:, n:] == 3.0).all())
    for _ in range(3):
        again = torch.empty(m, n, dtype=DT[dtype], device="cuda")
        ctx.mx4_matmul(qa, qb, again)
        assert torch.equal(again, buf[:, :n])


@pytest.mark.parametrize("m", [3, 150])
def test_product_writes_inside_the_output_only_and_repeats_its_bits(ctx, m):
    n, k = 261, 513
    a, b = torch.randn(m, k).cuda(), torch.randn(n, k).cuda()
    qa, qb = ctx.mx4_quantize(a), ctx.mx4_quantize(b)
    for dtype in DT.values():
        buf = torch.full((m + 2, n + 9), 3.0, dtype=dtype, device="cuda")
        ctx.mx4_matmul(qa, qb, buf[1:m + 1, 4:n + 4])
        keep = buf[1:m + 1, 4:n + 4].clone()
        again = torch.empty(m, n, dtype=dtype, device="cuda")
        ctx.mx4_matmul(qa, qb, again)
        assert torch.equal(keep, again)
        buf[1:m + 1, 4:n + 4] = 3.0
        assert bool((buf == 3.0).all())


@pytest.mark.parametrize("m", [5, 140])
def test_product_with_blocks_that_stand_for_nan_and_with_the_extreme_scales(ctx, m):
    """A NaN block makes its whole row NaN and no other; blocks at either end of the scale's range multiply."""
    n, k = 40, 200
    g = torch.Generator().manual_seed(1)
    a, b = torch.randn(m, k, generator=g), torch.randn(n, k, generator=g)
    a[1, 70] = float("inf")
    b[2, 3] = float("nan")
    a[3] *= 1e-30
    a[4] = 3e38
    b[5] *= 1e-38
    qa, qb = ctx.mx4_quantize(a.cuda()), ctx.mx4_quantize(b.cuda())
    out = ctx.mx4_matmul(qa, qb, torch.empty(m, n, device="cuda")).cpu()
    va, vb = R.quantize(a)[2], R.quantize(b)[2]
    nan = np.isnan(va).any(1)[:, None] | np.isnan(vb).any(1)[None, :]
    assert np.array_equal(torch.isnan(out).numpy(), nan)
    want = np.nan_to_num(va) @ np.nan_to_num(vb).T
    bound = _product_bound(np.nan_to_num(va), np.nan_to_num(vb), torch.float32) + 2.0 ** -126   # subnormals may be dropped
    # (where the magnitudes alone pass fp32's range a partial sum may be infinite, whatever the whole sum is)
    fine = ~nan & (np.abs(np.nan_to_num(va)) @ np.abs(np.nan_to_num(vb)).T < 3e38)
    assert fine.sum() > 2 * n
    assert (np.abs(out.double().numpy() - want) <= bound)[fine].all()


def test_gradients_of_a_linear_layer(ctx):
    """dx and dW from the transposed forms against the formula in 64 bits, and against differences of the loss: with the
    operands already on the grid the layer is exactly y = x W^T, so L = sum(dy * y) has exactly these gradients."""
    t, i, o = 96, 64, 160
    g = torch.Generator().manual_seed(3)
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float32)

    def on_grid(r, c):
        v = grid[torch.randint(0, 8, (r, c), generator=g)] * (1 - 2 * torch.randint(0, 2, (r, c), generator=g))
        v[:, ::32] = 6.0      # every block and every column's block has the same scale, so both forms are exact
        v[::32, :] = 6.0
        return v
    x, w, dy = on_grid(t, i), on_grid(o, i), on_grid(t, o)
    qdy, qdy_t = ctx.mx4_quantize_both(dy.cuda(), stochastic=True, seed=1)
    dx = ctx.mx4_matmul(qdy, ctx.mx4_quantize_transposed(w.cuda()), torch.empty(t, i, device="cuda")).cpu().double()
    dw = ctx.mx4_matmul(qdy_t, ctx.mx4_quantize_transposed(x.cuda()), torch.empty(o, i, device="cuda")).cpu().double()
    assert torch.equal(dx, dy.double() @ w.double())
    assert torch.equal(dw, dy.double().T @ x.double())

    def loss(x, w):
        y = ctx.mx4_matmul(ctx.mx4_quantize(x.cuda()), ctx.mx4_quantize(w.cuda()), torch.empty(t, o, device="cuda"))
        return float((y.cpu().double() * dy.double()).sum())
    for (r, c) in ((5, 7), (40, 33)):
        up, down = x.clone(), x.clone()
        up[r, c], down[r, c] = 2.0, -2.0
        assert loss(up, w) - loss(down, w) == 4.0 * float(dx[r, c])
        up, down = w.clone(), w.clone()
        up[r, c], down[r, c] = 1.0, -1.0
        assert loss(x, up) - loss(x, down) == 2.0 * float(dw[r, c])


LAYOUTS = {
    "tiny": (16, [16384], 4),
    "ragged": (64, [100, 40, 6404, 4, 64], 3),
    "short slices": (8, [8, 24, 1000], 2),
    "d12": (12, [12 * 70, 30], 5),
    "wide": (256, [256 * 67 + 12, 512], 9),
    "no slice": (128, [64, 100], 2),
    "one node": (128, [128 * 5], 1),
}


@pytest.mark.parametrize("stochastic", [False, True])
@pytest.mark.parametrize("name", list(LAYOUTS))
def test_exchange(name, stochastic):
    from paper_1811_03617_b200 import gvq
    d, lens, N = LAYOUTS[name]
    w = W.custom(name, 90, d, 4, N, 1, lens, layer_off=list(np.cumsum([0] + [-(-n // 4) * 4 + 8 for n in lens])[:-1]))
    c = gvq.Context(w)
    g = torch.Generator().manual_seed(len(name))
    grads = [torch.randn(w.M, generator=g) * 10 ** (3 * torch.rand(w.M, generator=g) - 3) for _ in range(N)]
    if w.S > 3:
        grads[0][w.layer_off[0]] = float("nan")
    dev = [x.cuda() for x in grads]
    seed, node0 = 77, 5
    total = torch.full((w.M,), -9.0, device="cuda")
    sent = [c.mx4_slices() for _ in range(N)] if w.S else None
    if sent:
        for q in sent:
            q.scales.fill_(0xEE)
    c.mx4_quantize_aggregate(dev, total, stochastic=stochastic, seed=seed, node0=node0, out=sent)
    alone = torch.full((w.M,), -9.0, device="cuda")
    c.mx4_quantize_aggregate(dev, alone, stochastic=stochastic, seed=seed, node0=node0)
    assert torch.equal(torch.nan_to_num(alone, 5.0), torch.nan_to_num(total, 5.0))

    want = torch.full((w.M,), -9.0)
    vals = []
    for n, x in enumerate(grads):
        if not w.S:
            break
        rows = torch.cat([x[o:o + m // d * d].view(-1, d) for o, m in zip(w.layer_off, lens)])
        codes, scales, v = R.quantize(rows, stochastic, seed, node0 + n)
        pc, ps = R.pack(codes, scales)
        assert torch.equal(sent[n].codes.cpu(), pc) and torch.equal(sent[n].scales.cpu(), ps)
        vals.append(torch.from_numpy(v.astype(np.float32)))
    at = 0
    for o, m in zip(w.layer_off, lens):
        f = m // d * d
        if f:
            acc = torch.zeros(f)
            for v in vals:
                acc = acc + v[at:at + f // d].reshape(-1)
            want[o:o + f] = acc
            at += f // d
        if m > f:
            acc = grads[0][o + f:o + m].clone()
            for x in grads[1:]:
                acc = acc + x[o + f:o + m]
            want[o + f:o + m] = acc
    assert torch.equal(torch.nan_to_num(total.cpu(), 5.0), torch.nan_to_num(want, 5.0))
    if sent:
        back = torch.full((w.M,), -9.0, device="cuda")
        c.mx4_dequantize_aggregate(sent, dev, back)
        assert torch.equal(torch.nan_to_num(back.cpu(), 5.0), torch.nan_to_num(want, 5.0))
        # a node's own share: the same bytes as in the call for all of them
        mine = c.mx4_slices()
        c.mx4_quantize_aggregate(dev[-1:], None, stochastic=stochastic, seed=seed, node0=node0 + N - 1, out=[mine])
        assert torch.equal(mine.codes, sent[-1].codes) and torch.equal(mine.scales, sent[-1].scales)


def test_calls_follow_the_stream_they_are_made_on(ctx):
    """Inputs written on a side stream just before the calls; results read after that stream alone is waited for."""
    side = torch.cuda.Stream()
    a, b = torch.randn(300, 400), torch.randn(500, 400)
    want = R.quantize(a)[2] @ R.quantize(b)[2].T
    with torch.cuda.stream(side):
        big = torch.randn(4096, 4096, device="cuda")
        for _ in range(4):
            big = big @ big * 1e-4
        da, db = a.cuda(non_blocking=True), b.cuda(non_blocking=True)
        out = ctx.mx4_matmul(ctx.mx4_quantize(da), ctx.mx4_quantize(db), torch.empty(300, 500, device="cuda"))
    side.synchronize()
    va, vb = R.quantize(a)[2], R.quantize(b)[2]
    assert (np.abs(out.cpu().double().numpy() - want) <= _product_bound(va, vb, torch.float32)).all()


def test_calls_can_be_captured(ctx):
    """No call uploads anything: a graph captured at the first use gives the eager result on new inputs."""
    x, w = torch.randn(70, 128, device="cuda"), torch.randn(96, 128, device="cuda")
    from paper_1811_03617_b200 import gvq
    qx, qw, y = gvq.Mx4(70, 128), gvq.Mx4(96, 128), torch.empty(70, 96, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.mx4_quantize(x, out=qx)
        ctx.mx4_quantize(w, out=qw)
        ctx.mx4_matmul(qx, qw, y)
    x.copy_(torch.randn(70, 128))
    graph.replay()
    torch.cuda.synchronize()
    eager = ctx.mx4_matmul(ctx.mx4_quantize(x), ctx.mx4_quantize(w), torch.empty(70, 96, device="cuda"))
    assert torch.equal(y, eager)


def test_a_wait_that_runs_out_is_reported_and_the_context_recovers(ctx):
    from paper_1811_03617_b200 import gvq
    a, b = torch.randn(200, 600, device="cuda"), torch.randn(300, 600, device="cuda")
    qa, qb = ctx.mx4_quantize(a), ctx.mx4_quantize(b)
    out = torch.empty(200, 300, device="cuda")
    good = ctx.mx4_matmul(qa, qb, out).clone()
    ctx.set_limits(wait_cycles=2_000_000)
    ctx.test_drop_load(True)
    try:
        ctx.mx4_matmul(qa, qb, out)
        with pytest.raises(gvq.GvqError) as e:
            ctx.device_status()
        assert e.value.status == 9
    finally:
        ctx.test_drop_load(False)
        ctx.set_limits()
    assert torch.equal(ctx.mx4_matmul(qa, qb, out), good)
    ctx.device_status()


@pytest.mark.parametrize("m,n,k", [(16, 500, 4128), (100, 300, 8200)])
def test_a_part_whose_wait_runs_out_is_reported_and_the_context_recovers(ctx, m, n, k):
    from paper_1811_03617_b200 import gvq
    qa, qb = ctx.mx4_quantize(torch.randn(m, k, device="cuda")), ctx.mx4_quantize(torch.randn(n, k, device="cuda"))
    out = torch.empty(m, n, device="cuda")
    good = ctx.mx4_matmul(qa, qb, out).clone()
    ctx.set_limits(wait_cycles=2_000_000)
    ctx.test_drop_load(True)
    try:
        ctx.mx4_matmul(qa, qb, out)
        with pytest.raises(gvq.GvqError) as e:
            ctx.device_status()
        assert e.value.status == 9
    finally:
        ctx.test_drop_load(False)
        ctx.set_limits()
    assert torch.equal(ctx.mx4_matmul(qa, qb, out), good)
    ctx.device_status()


def test_refusals(ctx):
    from paper_1811_03617_b200 import gvq
    L = gvq.lib()
    x = torch.zeros(64, 64, device="cuda")
    q = gvq.Mx4(64, 64)
    h, p, c, s = ctx._h, x.data_ptr(), q.codes.data_ptr(), q.scales.data_ptr()

    def quant(p=p, dt=0, r=64, k=64, ld=64, rnd=0, c=c, s=s, ct=None, st=None):
        return L.gvq_mx4_quantize(h, p, dt, r, k, ld, rnd, 0, 0, c, s, ct, st)
    assert quant() == 0
    assert quant(p=None) == 1 and quant(c=None) == 1 and quant(s=None) == 1 and quant(c=None, s=None) == 1
    assert quant(ct=c) == 1 and quant(st=s) == 1
    assert quant(r=0) == 2 and quant(k=0) == 2 and quant(k=-5) == 2 and quant(ld=63) == 2 and quant(dt=3) == 2 and quant(dt=-1) == 2
    assert quant(rnd=2) == 2 and quant(r=1 << 37, k=1 << 20) == 2
    assert quant(c=c + 8) == 3 and quant(s=s + 4) == 3 and quant(p=p + 2) == 3 and quant(p=p + 1, dt=1) == 3
    assert L.gvq_mx4_dequantize(h, c, s, 64, 64, None, 64) == 1 and L.gvq_mx4_dequantize(h, c, s, 64, 64, p, 63) == 2
    assert L.gvq_mx4_dequantize(h, c, s + 1, 64, 64, p, 64) == 3

    def mm(a=c, sa=s, b=c, sb=s, m=64, n=64, k=64, o=p, dt=0, ld=64):
        return L.gvq_mx4_matmul(h, a, sa, b, sb, m, n, k, o, dt, ld)
    assert mm() == 0
    assert mm(a=None) == 1 and mm(sb=None) == 1 and mm(o=None) == 1
    assert mm(m=0) == 2 and mm(n=0) == 2 and mm(k=0) == 2 and mm(ld=63) == 2 and mm(dt=7) == 2 and mm(k=1 << 36) == 2
    assert mm(a=c + 4) == 3 and mm(sb=s + 8) == 3 and mm(o=p + 2) == 3
    g = gvq._ptr_array([x.view(-1)])
    assert L.gvq_mx4_quantize_aggregate(h, g, 1, 0, 0, 0, None, None, None) == 1
    assert L.gvq_mx4_quantize_aggregate(h, g, 0, 0, 0, 0, p, None, None) == 2
    assert L.gvq_mx4_quantize_aggregate(h, g, 1, 0, 5, 0, p, None, None) == 2
    assert L.gvq_mx4_quantize_aggregate(h, g, 1, 0, 0, 0, p, None, None) == 2      # the output is an input
    assert L.gvq_mx4_quantize_aggregate(h, g, 65, 0, 0, 0, p, None, None) == 2
    assert L.gvq_mx4_dequantize_aggregate(h, None, None, None, 1, p) == 1
    torch.cuda.synchronize()
    with pytest.raises(ValueError):
        ctx.mx4_quantize(x[0])
    with pytest.raises(ValueError):
        ctx.mx4_quantize(x.t()[:, ::2])
    with pytest.raises(TypeError):
        ctx.mx4_quantize(x.double())
    with pytest.raises(ValueError):
        ctx.mx4_matmul(q, gvq.Mx4(64, 32), x)
    with pytest.raises(ValueError):
        gvq.Mx4(64, 64, codes=torch.empty(3, dtype=torch.uint8, device="cuda"))
