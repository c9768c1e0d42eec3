"""The gated block on the GPU against its formula in 64 bits: forward, what is kept for the backward pass, the gradients, the
form on 8-bit integers."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}      # half a step, relative
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}   # and where steps are of one size
ACTS = ["silu", "gelu", "gelu_tanh", "relu", "sigmoid"]


@pytest.fixture(scope="module")
def ctx():
    from paper_1811_03617_b200 import gvq
    return gvq.Context(gvq.HostLayout(4, 4, [0], [4]))


def act(name, g):
    """(activation, derivative) in 64 bits."""
    if name == "relu":
        return g * (g > 0), (g > 0).double()
    if name == "gelu":
        cdf = 0.5 * torch.special.erfc(-g / math.sqrt(2))
        return g * cdf, cdf + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        c = 2 * math.sqrt(2 / math.pi)
        s = torch.sigmoid(c * (g + 0.044715 * g ** 3))
        return g * s, s + g * s * (1 - s) * c * (1 + 3 * 0.044715 * g * g)
    s = torch.sigmoid(g)
    return (s, s * (1 - s)) if name == "sigmoid" else (g * s, s + g * s * (1 - s))


# The tensor core adds the 16 products of a step into an fp32 accumulator, which it may truncate: every step may lose 2^-22 of the
# sum of magnitudes.
def _lost(mag, k):
    return mag * (-(-k // 16) + 2) * 2.0 ** -22


def _near(got, want, bound, dtype):
    top = float(torch.finfo(dtype).max)
    near = want.abs() + bound < top
    assert bool(near.any()) and not bool(torch.isnan(got).any())
    assert bool(((got.double() - want).abs() <= bound)[near].all()), float(((got.double() - want).abs() / bound)[near].max())


def _h_bound(name, g, u, eg, eu, dtype):
    """An activation's slope is below 1.13 everywhere, and fp32 computes it to 16 half steps of max(1, |g|) (its exponential, its
    quotient, and for erfc and the cubic the argument's own roundings, each a few)."""
    a = act(name, g)[0].abs()
    ea = 1.13 * eg + 2.0 ** -20 * (1 + g.abs())
    h = a * u.abs()
    return ea * (u.abs() + eu) + a * eu + h * (2.0 ** -23 + HALF[dtype]) + TINY[dtype]


def _rows(g, rows, cols, dtype, pad, scale=1.0, offset=0):
    """A matrix whose rows are `pad` entries further apart than they are long, NaN between them."""
    buf = torch.full((offset + rows * (cols + pad),), float("nan"), dtype=dtype, device="cuda")
    view = torch.as_strided(buf, (rows, cols), (cols + pad, 1), offset)
    view.copy_(torch.randn(rows, cols, generator=g, device="cuda") * scale)
    return view


def _forward(ctx, M, F, K, dtype, name, pad=0, offset=0, kept=True, hpad=0):
    dtype = DT[dtype]
    g = torch.Generator(device="cuda").manual_seed(M + F + K)
    x = _rows(g, M, K, dtype, pad, 1.0, offset)
    wg, wu = (_rows(g, F, K, dtype, pad, 2 / math.sqrt(K), offset) for _ in range(2))
    bufs = [torch.full((M, F + hpad), 3.0, dtype=dtype, device="cuda") for _ in range(3)]
    h, gate, up = (b[:, :F] for b in bufs)
    kw = dict(gate=gate, up=up) if kept else {}
    ctx.gated_forward(x, wg, wu, h, act=name, **kw)
    ctx.device_status()
    xd, gd, ud = x.double(), wg.double(), wu.double()
    want_g, want_u = xd @ gd.T, xd @ ud.T
    eg, eu = _lost(xd.abs() @ gd.abs().T, K), _lost(xd.abs() @ ud.abs().T, K)
    _near(h, act(name, want_g)[0] * want_u, _h_bound(name, want_g, want_u, eg, eu, dtype), dtype)
    if kept:
        for got, want, e in ((gate, want_g, eg), (up, want_u, eu)):
            _near(got, want, e + (want.abs() + e) * HALF[dtype] + TINY[dtype], dtype)
    for b in bufs:
        assert bool((b[:, F:] == 3.0).all())
    again = torch.empty(M, F, dtype=dtype, device="cuda")
    ctx.gated_forward(x, wg, wu, again, act=name)
    assert torch.equal(again, h)          # the same bits, kept or not


# few tokens (tiles as narrow as they are, both matrices' tiles), one CTA a tile, pairs of CTAs, several tiles a pair
@pytest.mark.parametrize("M,F,K,dtype,name", [
    (1, 1, 1, "bf16", "silu"), (1, 300, 64, "f16", "gelu"), (3, 129, 72, "bf16", "relu"), (16, 500, 136, "f16", "gelu_tanh"),
    (17, 1000, 520, "bf16", "sigmoid"), (33, 64, 256, "bf16", "silu"), (64, 5000, 512, "f16", "silu"), (65, 40, 32, "bf16", "gelu"),
    (100, 2000, 304, "f16", "relu"), (128, 32, 64, "bf16", "silu"), (200, 520, 1080, "bf16", "gelu_tanh"), (700, 1100, 520, "f16", "gelu"),
    (1300, 1029, 2104, "bf16", "silu"), (2600, 1300, 640, "bf16", "sigmoid"), (300, 5001, 72, "f16", "silu")])
def test_forward(ctx, M, F, K, dtype, name):
    _forward(ctx, M, F, K, dtype, name)


@pytest.mark.parametrize("M,F,K", [(1, 200, 4100), (5, 1000, 2056), (16, 130, 8200), (40, 300, 5000), (64, 600, 2120), (130, 90, 4200)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_forward_with_a_long_contraction(ctx, M, F, K, dtype):
    """A cluster of CTAs shares a tile's contraction."""
    _forward(ctx, M, F, K, dtype, "silu")


@pytest.mark.parametrize("M", [1, 7, 40, 150, 900])
@pytest.mark.parametrize("pad,offset,hpad", [(1, 0, 0), (0, 1, 1), (5, 3, 8), (8, 8, 3)])
def test_forward_with_rows_at_any_place(ctx, M, pad, offset, hpad):
    _forward(ctx, M, 333, 165, "bf16", "silu", pad, offset, True, hpad)
    _forward(ctx, M, 328, 160, "f16", "gelu", pad, offset, False, hpad)


def test_more_tiles_of_few_tokens_than_ctas(ctx):
    for M, F in ((1, 40000), (20, 60001), (50, 30010)):
        _forward(ctx, M, F, 40, "bf16", "silu")


def test_activations_over_their_whole_range(ctx):
    """x is one column: g takes every size, u is 1, so h is the activation itself; infinities and NaN stay in their row."""
    g = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 0.5, -0.5, 3.0, -3.0, 9.0, -9.0, 30.0, -30.0, 89.0, -89.0, 1e4, -1e4, 1e15, -1e15, 3e38, -3e38],
                     dtype=torch.bfloat16, device="cuda")
    one = torch.ones(1, 1, dtype=torch.bfloat16, device="cuda")
    for rows in (len(g), 200):
        x = torch.stack([g, torch.ones_like(g)], 1)
        x = torch.cat([x, torch.zeros(rows - len(g), 2, dtype=x.dtype, device="cuda")])
        wg, wu = torch.tensor([[1.0, 0.0]], device="cuda").bfloat16(), torch.tensor([[0.0, 1.0]], device="cuda").bfloat16()
        for name in ACTS:
            h, gate, up = (torch.empty(rows, 1, dtype=torch.bfloat16, device="cuda") for _ in range(3))
            ctx.gated_forward(x, wg, wu, h, act=name, gate=gate, up=up)
            assert torch.equal(gate[:len(g), 0], g) and bool((up[:len(g)] == 1).all())
            want, slope = act(name, g.double().clamp(-1e30, 1e30))
            want = torch.where(g.double().abs() > 1e30, torch.where(g > 0, g.double() if name != "sigmoid" else want, want * 0), want)
            _near(h[:len(g), 0], want, want.abs() * 2.0 ** -8 + 2.0 ** -20, torch.bfloat16)
            dw, dh = torch.empty(1, 2, device="cuda"), torch.ones(rows, 1, dtype=torch.bfloat16, device="cuda")
            dx = torch.empty(rows, 2, dtype=torch.bfloat16, device="cuda")
            ctx.gated_backward(dh, gate, up, x, wg, wu, act=name, dx=dx)
            slope = torch.nan_to_num(slope, 0.0)
            far = g.double().abs() > 1e14      # the derivative there: 1 or 0
            slope = torch.where(far, ((g > 0) & (name != "sigmoid")).double(), slope)
            _near(dx[:len(g), 0], slope, slope.abs() * 2.0 ** -7 + 2.0 ** -18, torch.bfloat16)
    x = torch.randn(150, 64, device="cuda").bfloat16()
    w = torch.randn(40, 64, device="cuda").bfloat16()
    x[3, 5], x[9, 9] = float("nan"), float("inf")
    h = ctx.gated_forward(x, w, w, torch.empty(150, 40, dtype=torch.bfloat16, device="cuda"))
    ok = torch.isfinite(h).all(1)
    assert not bool(ok[3]) and not bool(ok[9]) and int(ok.sum()) == 148
    assert one.item() == 1


def _backward(ctx, M, F, K, dtype, name, pad=0, offset=0, dw="f32", opad=0, which=("dx", "dw_gate", "dw_up")):
    dtype, dw = DT[dtype], DT[dw]
    g = torch.Generator(device="cuda").manual_seed(M + 2 * F + K)
    x = _rows(g, M, K, dtype, pad, 1.0, offset)
    wg, wu = (_rows(g, F, K, dtype, pad, 1 / math.sqrt(K), offset) for _ in range(2))
    gate, up, dh = (_rows(g, M, F, dtype, pad, 1.0, offset) for _ in range(3))
    bufs = {"dx": torch.full((M, K + opad), 3.0, dtype=dtype, device="cuda"), "dw_gate": torch.full((F, K + opad), 3.0, dtype=dw, device="cuda"),
            "dw_up": torch.full((F, K + opad), 3.0, dtype=dw, device="cuda")}
    outs = {k: v[:, :K] for k, v in bufs.items() if k in which}
    ctx.gated_backward(dh, gate, up, x if set(which) - {"dx"} else None, wg if "dx" in which else None, wu if "dx" in which else None, act=name, **outs)
    ctx.device_status()
    a, slope = act(name, gate.double())
    dg, du = dh.double() * up.double() * slope, dh.double() * a
    # dg and du: fp32 (the activation as in the forward pass, its slope twice that), rounded to the operands' type
    eg = (dh.double() * up.double()).abs() * 2.0 ** -19 * (1 + gate.double().abs()) + dg.abs() * HALF[dtype] + TINY[dtype]
    eu = dh.double().abs() * 2.0 ** -20 * (1 + gate.double().abs()) + du.abs() * HALF[dtype] + TINY[dtype]
    want = {"dx": dg @ wg.double() + du @ wu.double(), "dw_gate": dg.T @ x.double(), "dw_up": du.T @ x.double()}
    mag = {"dx": (dg.abs() + eg) @ wg.double().abs() + (du.abs() + eu) @ wu.double().abs(), "dw_gate": (dg.abs() + eg).T @ x.double().abs(),
           "dw_up": (du.abs() + eu).T @ x.double().abs()}
    err = {"dx": eg @ wg.double().abs() + eu @ wu.double().abs(), "dw_gate": eg.T @ x.double().abs(), "dw_up": eu.T @ x.double().abs()}
    for k, got in outs.items():
        t = got.dtype
        e = err[k] + _lost(mag[k], 2 * F + 64 if k == "dx" else M)
        _near(got, want[k], e + (want[k].abs() + e) * HALF[t] + TINY[t], t)
    for k, v in bufs.items():
        assert bool((v[:, K if k in which else 0:] == 3.0).all())
    return outs


@pytest.mark.parametrize("M,F,K,dtype,name,dw", [
    (1, 1, 1, "bf16", "silu", "f32"), (1, 300, 64, "f16", "gelu", "f16"), (3, 129, 72, "bf16", "relu", "bf16"), (16, 504, 136, "f16", "gelu_tanh", "f32"),
    (17, 1000, 520, "bf16", "sigmoid", "f16"), (33, 64, 256, "bf16", "silu", "f32"), (64, 512, 9600, "f16", "silu", "f16"),
    (65, 40, 32, "bf16", "gelu", "f32"), (200, 520, 1080, "bf16", "gelu_tanh", "bf16"), (700, 1104, 520, "f16", "gelu", "f32"),
    (1300, 1032, 2104, "bf16", "silu", "f32"), (2600, 1304, 1640, "bf16", "silu", "bf16"), (5000, 72, 3000, "bf16", "relu", "f32")])
def test_backward(ctx, M, F, K, dtype, name, dw):
    _backward(ctx, M, F, K, dtype, name, dw=dw)


@pytest.mark.parametrize("M", [1, 20, 50, 150, 1300])
@pytest.mark.parametrize("pad,offset,opad", [(1, 0, 0), (0, 1, 1), (5, 3, 8), (8, 8, 3)])
def test_backward_with_rows_at_any_place(ctx, M, pad, offset, opad):
    _backward(ctx, M, 333, 165, "bf16", "silu", pad, offset, "f32", opad)
    _backward(ctx, M, 336, 1160, "f16", "gelu", pad, offset, "f16", opad)


@pytest.mark.parametrize("which", [("dx",), ("dw_gate",), ("dw_up",), ("dx", "dw_up"), ("dw_gate", "dw_up")])
@pytest.mark.parametrize("M,F,K", [(9, 200, 100), (300, 520, 264), (1000, 2001, 1111)])
def test_backward_of_what_is_wanted(ctx, which, M, F, K):
    some = _backward(ctx, M, F, K, "bf16", "silu", which=which)
    everything = _backward(ctx, M, F, K, "bf16", "silu")
    for k, v in some.items():
        assert torch.equal(v, everything[k])


@pytest.mark.parametrize("M,F,K", [(1, 300, 4200), (16, 2056, 130), (40, 3000, 200), (100, 2500, 90), (20, 8200, 300)])
def test_backward_with_a_long_contraction(ctx, M, F, K):
    _backward(ctx, M, F, K, "bf16", "silu")


def test_gradients_are_the_differences_of_a_loss(ctx):
    """L = sum(dh * h) in 64 bits, moved along a random direction of every input: the quotient of differences of a smooth function is
    off by step^2 times its third derivative, the gradients by their roundings; 1 % of the sum of magnitudes covers both."""
    M, F, K = 70, 96, 80
    g = torch.Generator(device="cuda").manual_seed(4)
    x, wg, wu, dh = (torch.randn(r, c, generator=g, device="cuda").bfloat16() * s for r, c, s in
                     ((M, K, 1.0), (F, K, 0.125), (F, K, 0.125), (M, F, 1.0)))
    for name in ("silu", "gelu", "gelu_tanh", "sigmoid"):
        h, gate, up, dx = (torch.empty(r, c, dtype=torch.bfloat16, device="cuda") for r, c in ((M, F), (M, F), (M, F), (M, K)))
        ctx.gated_forward(x, wg, wu, h, act=name, gate=gate, up=up)
        dwg, dwu = torch.empty(F, K, device="cuda"), torch.empty(F, K, device="cuda")
        ctx.gated_backward(dh, gate, up, x, wg, wu, act=name, dx=dx, dw_gate=dwg, dw_up=dwu)

        def loss(x, wg, wu):
            return float((dh.double() * act(name, x @ wg.T)[0] * (x @ wu.T)).sum())
        ins, grads = [t.double() for t in (x, wg, wu)], (dx, dwg, dwu)
        for j in range(3):
            d = torch.randn(ins[j].shape, generator=g, device="cuda").double()
            e = 1e-4
            moved = [[t + (s * e * d if i == j else 0) for i, t in enumerate(ins)] for s in (1, -1)]
            want = (loss(*moved[0]) - loss(*moved[1])) / (2 * e)
            terms = grads[j].double() * d
            assert abs(float(terms.sum()) - want) <= 0.01 * float(terms.abs().sum())


def _gated8(ctx, M, F, K, dtype, name, pad=0):
    dtype = DT[dtype]
    g = torch.Generator(device="cuda").manual_seed(M + F + K)
    x = torch.randn(M, K, generator=g, device="cuda") * 2.0 ** torch.randint(-3, 2, (M, 1), generator=g, device="cuda")
    wg, wu = (torch.randn(F, K, generator=g, device="cuda") * 2.0 ** torch.randint(-2, 2, (F, 1), generator=g, device="cuda") / math.sqrt(K)
              for _ in range(2))
    qx, qg, qu = (ctx.i8_quantize(t) for t in (x, wg, wu))
    buf = torch.full((M, F + pad), 3.0, dtype=dtype, device="cuda")
    ctx.i8_gated(qx, qg, qu, buf[:, :F], act=name)
    ctx.device_status()

    def product(q):      # whole numbers are summed exactly, and a sum may be 0: the scales come after it
        return (qx.codes[:, :K].double() @ q.codes[:, :K].double().T) * qx.scales.double()[:, None] * q.scales.double()
    want_g, want_u = product(qg), product(qu)
    # exact sums: their conversion and two scales round (a cancelled sum is exact too)
    eg, eu = want_g.abs() * 3.01 * 2.0 ** -24 + 2.0 ** -126, want_u.abs() * 3.01 * 2.0 ** -24 + 2.0 ** -126
    _near(buf[:, :F], act(name, want_g)[0] * want_u, _h_bound(name, want_g, want_u, eg, eu, dtype), dtype)
    assert bool((buf[:, F:] == 3.0).all())
    again = torch.empty(M, F, dtype=dtype, device="cuda")
    assert torch.equal(ctx.i8_gated(qx, qg, qu, again, act=name), buf[:, :F])


@pytest.mark.parametrize("M,F,K,dtype,name,pad", [
    (1, 1, 1, "f32", "silu", 0), (1, 300, 64, "bf16", "gelu", 1), (3, 129, 70, "f16", "relu", 0), (16, 500, 2130, "bf16", "gelu_tanh", 8),
    (17, 1000, 515, "f32", "sigmoid", 3), (33, 64, 4256, "bf16", "silu", 0), (64, 5000, 512, "f16", "silu", 8), (65, 40, 33, "f32", "gelu", 0),
    (100, 2000, 300, "bf16", "relu", 4), (200, 515, 1083, "bf16", "silu", 5), (700, 1100, 520, "f32", "gelu", 0),
    (1300, 1029, 2100, "bf16", "silu", 3), (2600, 1304, 640, "f16", "sigmoid", 0), (130, 60, 9000, "f32", "silu", 0)])
def test_gated_8_bit(ctx, M, F, K, dtype, name, pad):
    _gated8(ctx, M, F, K, dtype, name, pad)


@pytest.mark.parametrize("M,F,K", [(8, 520, 264), (50, 5008, 136), (150, 200, 136), (1000, 2000, 520)])
def test_calls_follow_their_stream_and_can_be_captured(ctx, M, F, K):
    """Rows that need copies too: the copies' room belongs to the graph."""
    bf = torch.bfloat16
    for odd in (0, 1):
        x, wg, wu, dh = (torch.randn(r, c, device="cuda").to(bf) for r, c in ((M, K - odd), (F, K - odd), (F, K - odd), (M, F)))

        def room():
            return [torch.empty(M, F, dtype=bf, device="cuda") for _ in range(3)] + [torch.empty(M, K - odd, dtype=bf, device="cuda")] + \
                   [torch.empty(F, K - odd, device="cuda") for _ in range(2)]

        def step(o, x):
            ctx.gated_forward(x, wg, wu, o[0], gate=o[1], up=o[2])
            ctx.gated_backward(dh, o[1], o[2], x, wg, wu, dx=o[3], dw_gate=o[4], dw_up=o[5])
        captured, eager, late = room(), room(), room()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(captured, x)
        x.copy_(torch.randn(M, K - odd))
        graph.replay()
        step(eager, x)
        torch.cuda.synchronize()
        for a, b in zip(captured, eager):
            assert torch.equal(a, b)
        side, x2 = torch.cuda.Stream(), torch.empty_like(x)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            big = torch.randn(4096, 4096, device="cuda")
            for _ in range(4):
                big = big @ big * 1e-4
            x2.copy_(x)
            step(late, x2)
        side.synchronize()
        for a, b in zip(late, eager):
            assert torch.equal(a, b)


@pytest.mark.parametrize("M,F,K", [(8, 500, 4200), (150, 200, 400), (1300, 1029, 304)])
def test_a_wait_that_runs_out_is_reported_and_the_context_recovers(ctx, M, F, K):
    from paper_1811_03617_b200 import gvq
    x, wg, wu = (torch.randn(r, K, device="cuda").bfloat16() for r in (M, F, F))
    h = torch.empty(M, F, dtype=torch.bfloat16, device="cuda")
    good = ctx.gated_forward(x, wg, wu, h).clone()
    ctx.set_limits(wait_cycles=2_000_000)
    ctx.test_drop_load(True)
    try:
        ctx.gated_forward(x, wg, wu, h)
        with pytest.raises(gvq.GvqError) as e:
            ctx.device_status()
        assert e.value.status == 9
    finally:
        ctx.test_drop_load(False)
        ctx.set_limits()
    assert torch.equal(ctx.gated_forward(x, wg, wu, h), good)
    ctx.device_status()


# dx and the weights' gradients in one launch: an SM a tile, some with a shared contraction, pairs of SMs with 128 and 256 columns
@pytest.mark.parametrize("M,F,K,dtype,dw,pad,opad", [
    (150, 200, 136, "bf16", "bf16", 0, 0), (100, 2500, 90, "f16", "f32", 3, 1), (300, 520, 264, "bf16", "f16", 0, 2), (1100, 700, 700, "f16", "f16", 1, 0),
    (1100, 704, 720, "bf16", "f32", 0, 8), (2100, 1030, 1000, "bf16", "bf16", 0, 0), (600, 600, 2101, "f16", "f32", 0, 3), (520, 1029, 2050, "bf16", "bf16", 0, 6)])
def test_backward_in_one_launch(ctx, M, F, K, dtype, dw, pad, opad):
    _backward(ctx, M, F, K, dtype, "gelu", pad, dw=dw, opad=opad)
    _backward(ctx, M, F, K, dtype, "relu", pad, dw=dw, opad=opad, which=("dx", "dw_up"))


@pytest.mark.parametrize("M,F,K", [(150, 200, 136), (300, 520, 264), (600, 600, 2104), (20, 300, 200)])
def test_a_wait_of_the_backward_pass_that_runs_out(ctx, M, F, K):
    from paper_1811_03617_b200 import gvq
    x, wg, wu, dh, g, u = (torch.randn(r, c, device="cuda").bfloat16() for r, c in ((M, K), (F, K), (F, K), (M, F), (M, F), (M, F)))
    out = {"dx": torch.empty_like(x), "dw_gate": torch.empty_like(wg), "dw_up": torch.empty_like(wu)}
    ctx.gated_backward(dh, g, u, x, wg, wu, **out)
    good = [t.clone() for t in out.values()]
    ctx.set_limits(wait_cycles=2_000_000)
    ctx.test_drop_load(True)
    try:
        ctx.gated_backward(dh, g, u, x, wg, wu, **out)
        with pytest.raises(gvq.GvqError) as e:
            ctx.device_status()
        assert e.value.status == 9
    finally:
        ctx.test_drop_load(False)
        ctx.set_limits()
    ctx.gated_backward(dh, g, u, x, wg, wu, **out)
    ctx.device_status()
    for a, b in zip(good, out.values()):
        assert torch.equal(a, b)


# outputs whose rows start anywhere in a sector, of every width of a strip's last piece
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hpad", [0, 1, 2, 5, 8, 16])
def test_outputs_at_any_place(ctx, dtype, hpad):
    for F in (1, 15, 30, 31, 47, 64, 66, 97, 129, 250):
        _forward(ctx, 140, F, 40, dtype, "silu", hpad=hpad)
    for F in (1029, 1040):
        _forward(ctx, 2100, F, 24, dtype, "gelu", hpad=hpad)


@pytest.mark.parametrize("M,F,K,dtype,name", [
    (1, 40, 24, "bf16", "silu"), (20, 300, 130, "f16", "gelu"), (64, 200, 700, "bf16", "relu"), (90, 50, 46, "f16", "silu"), (300, 333, 165, "bf16", "gelu_tanh"),
    (1400, 50, 46, "f16", "gelu"), (400, 600, 250, "bf16", "sigmoid"), (250, 2100, 100, "f16", "relu")])
def test_short_products_do_not_round_the_slopes(ctx, M, F, K, dtype, name):
    """Up to 2^26 multiply-adds dg and du are two halves each: what is off by half a step of dtype above is off by half a step of half
    a step, and with fp16 by no more than half its smallest step."""
    t = DT[dtype]
    g = torch.Generator(device="cuda").manual_seed(M + F + K)
    x, wg, wu = (_rows(g, r, K, t, 0, s) for r, s in ((M, 1.0), (F, 1 / math.sqrt(K)), (F, 1 / math.sqrt(K))))
    gate, up, dh = (_rows(g, M, F, t, 0) for _ in range(3))
    out = {"dx": torch.empty(M, K, device="cuda", dtype=t), "dw_gate": torch.empty(F, K, device="cuda"), "dw_up": torch.empty(F, K, device="cuda")}
    ctx.gated_backward(dh, gate, up, x, wg, wu, act=name, **out)
    ctx.device_status()
    a, slope = act(name, gate.double())
    dg, du = dh.double() * up.double() * slope, dh.double() * a
    eg = (dh.double() * up.double()).abs() * 2.0 ** -19 * (1 + gate.double().abs()) + dg.abs() * HALF[t] ** 2 + TINY[t]
    eu = dh.double().abs() * 2.0 ** -20 * (1 + gate.double().abs()) + du.abs() * HALF[t] ** 2 + TINY[t]
    x, wg, wu = x.double(), wg.double(), wu.double()
    want = {"dx": dg @ wg + du @ wu, "dw_gate": dg.T @ x, "dw_up": du.T @ x}
    mag = {"dx": dg.abs() @ wg.abs() + du.abs() @ wu.abs(), "dw_gate": dg.abs().T @ x.abs(), "dw_up": du.abs().T @ x.abs()}
    err = {"dx": eg @ wg.abs() + eu @ wu.abs(), "dw_gate": eg.T @ x.abs(), "dw_up": eu.T @ x.abs()}
    for k, got in out.items():
        e = err[k] + 1.01 * _lost(mag[k], 2 * (2 * F + 64) if k == "dx" else 2 * (M + 64))
        _near(got, want[k], e + (want[k].abs() + e) * HALF[got.dtype] + TINY[got.dtype], got.dtype)
    if M == 1:      # an infinite slope stays one, and its row's alone
        dh[0, 3] = float("inf")
        ctx.gated_backward(dh, gate, up, x.to(t), None, None, act=name, dw_gate=out["dw_gate"], dw_up=out["dw_up"])
        other = torch.arange(F, device="cuda") != 3
        assert bool(torch.isfinite(out["dw_up"][other]).all()) and bool(torch.isinf(out["dw_up"][3]).all())
