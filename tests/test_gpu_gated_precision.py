"""How exact the gated block's gradients are where it is easily lost."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

BF, F16, F32 = torch.bfloat16, torch.float16, torch.float32
HALF = {BF: 2.0 ** -8, F16: 2.0 ** -11, F32: 2.0 ** -24}      # half a step, relative


@pytest.fixture(scope="module")
def ctx():
    from paper_1811_03617_b200 import gvq
    return gvq.Context(gvq.HostLayout(4, 4, [0], [4]))


def act(name, g):
    """(activation, derivative) in 64 bits, without differences of nearly equal numbers."""
    if name == "relu":
        return g * (g > 0), (g > 0).double()
    if name == "gelu":
        cdf = 0.5 * torch.special.erfc(-g / math.sqrt(2))
        return g * cdf, cdf + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        c = 2 * math.sqrt(2 / math.pi)
        z = c * (g + 0.044715 * g ** 3)
        s = torch.sigmoid(z)
        return g * s, s + g * s * torch.sigmoid(-z) * c * (1 + 3 * 0.044715 * g * g)
    s, r = torch.sigmoid(g), torch.sigmoid(-g)
    return (s, s * r) if name == "sigmoid" else (g * s, s + g * s * r)


def _of_one_token(ctx, g, name):
    """(du, dg) of gates g with dh = u = 1, as the kernels form them: one token, x = 1, so that the weights' gradients in fp32 are du and
    dg themselves, of which what rounding to 16 bits leaves is multiplied too (2^26 multiply-adds are far off)."""
    n = len(g)
    gate, ones = g.view(1, n), torch.ones(1, n, dtype=g.dtype, device="cuda")
    dw = [torch.empty(n, 1, device="cuda") for _ in range(2)]
    ctx.gated_backward(ones, gate, ones, torch.ones(1, 1, dtype=g.dtype, device="cuda"), None, None, act=name, dw_gate=dw[0], dw_up=dw[1])
    ctx.device_status()
    return dw[1][:, 0].double(), dw[0][:, 0].double()


@pytest.mark.parametrize("dtype", [BF, F16])
def test_sigmoid_keeps_its_digits_where_it_saturates(ctx, dtype):
    """Relative errors: two halves of dg 2^-16 or 2^-22 of it; the exponential's argument has three roundings (the constant, the product,
    the unit's), each 2^-24 of |g|, and what follows is a few steps of fp32, 2^-20 with room."""
    g = torch.linspace(0.25, 30 if dtype == BF else 12, 300, device="cuda").to(dtype)
    g = torch.cat([g, -g])
    value, slope = act("sigmoid", g.double())
    for got, want in zip(_of_one_token(ctx, g, "sigmoid"), (value, slope)):
        bound = HALF[dtype] ** 2 + 3 * g.double().abs() * 2.0 ** -24 + 2.0 ** -20
        if dtype == F16:      # (half of half precision's smallest step, 2^-25, where the largest entry, 1 here, is held as 2^15, or 32752 where that overflows)
            bound = bound + 2.0 ** -39 / want
        off = ((got - want).abs() / want / bound)
        assert float(off.max()) <= 1, (float(off.max()), float(g[off.argmax()]))


def test_the_tail_of_gelu_keeps_its_digits(ctx):
    """Relative errors from -3 to -12: the fit 1.2e-7; exponents g^2 / 2, four roundings of 2^-24 of it; the fit's polynomial, whose ten steps
    sum to less than 8, 80 roundings of 2^-25; two halves of a bfloat16.  The derivative is cdf - |g| density, the second at least 9 times
    the first, so that nothing cancels (twice the bound covers both terms' errors)."""
    g = torch.linspace(-3, -12, 400, device="cuda").to(BF)
    value, slope = act("gelu", g.double())
    bound = 1.2e-7 + g.double() ** 2 / 2 * 4 * 2.0 ** -24 + 80 * 2.0 ** -25 + 2.0 ** -16
    for got, want, times in zip(_of_one_token(ctx, g, "gelu"), (value, slope), (1, 2)):
        off = ((got - want) / want).abs() / (times * bound)
        assert float(off.max()) <= 1, (float(off.max()), float(g[off.argmax()]))
    # past where the density is a normal number: nothing, and nothing wrong
    for far in _of_one_token(ctx, torch.tensor([-14.0, -20.0, -1e4, -3e38], device="cuda").to(BF), "gelu"):
        assert bool((far.abs() < 2.0 ** -120).all())


# sizes on both sides of 2^26 multiply-adds; one token, few, tiles, one launch for all gradients, pairs of SMs, rows at any place
SIZES = [(1, 300, 264), (20, 333, 165), (300, 333, 165), (700, 520, 264), (64, 2056, 1032), (1300, 1029, 520)]


def _gradients(ctx, M, F, K, dtype, name, dh_size, up_size=1.0, **kw):
    """Outputs, and for each (wanted value, sum of magnitudes, what errors of dg and du relative to themselves make of it)."""
    gen = torch.Generator(device="cuda").manual_seed(M + F + K)

    def made(rows, cols, size=1.0):
        return (torch.randn(rows, cols, generator=gen, device="cuda") * size).to(dtype)
    x, wg, wu = made(M, K), made(F, K, 1 / math.sqrt(K)), made(F, K, 1 / math.sqrt(K))
    gate, up, dh = made(M, F), made(M, F, up_size), made(M, F) * 1.0
    dh = (dh.float() * dh_size).to(dtype)
    out = {"dx": torch.empty(M, K, device="cuda", dtype=dtype), "dw_gate": torch.empty(F, K, device="cuda"), "dw_up": torch.empty(F, K, device="cuda")}
    ctx.gated_backward(dh, gate, up, x, wg, wu, act=name, **out, **kw)
    ctx.device_status()
    a, slope = act(name, gate.double())
    dhu = dh.double() * up.double()
    dg, du = dhu * slope, dh.double() * a
    x, wg, wu = x.double(), wg.double(), wu.double()
    want = {"dx": dg @ wg + du @ wu, "dw_gate": dg.T @ x, "dw_up": du.T @ x}

    def spread(eg, eu):
        return {"dx": eg @ wg.abs() + eu @ wu.abs(), "dw_gate": eg.T @ x.abs(), "dw_up": eu.T @ x.abs()}
    top = max(float(dg.abs().max()), float(du.abs().max()))
    # fp32: the activation 16 half steps of max(1, |g|), its slope twice that (of dh u, as |slope| < 1.13)
    fp32 = (dhu.abs() * 2.0 ** -19 * (1 + gate.double().abs()), dh.double().abs() * 2.0 ** -20 * (1 + gate.double().abs()))
    return out, want, spread(dg.abs(), du.abs()), spread(*fp32), spread(torch.ones_like(dg) * top, torch.ones_like(dg) * top)


def _check(out, want, mag, fp32, top, M, F, dtype, operand, names):
    """operand: what rounding leaves of dg and du, relative; half precision: half its smallest step, 2^-25, where the largest
    entry is held as 2^15 to 2^16, or half of that where it overflows."""
    for k in names:
        got, t = out[k], out[k].dtype
        steps = (2 * 2 * F if k == "dx" else 2 * M) // 16 + 8      # of 16 terms, each of which may lose 2^-22 of the sum of magnitudes
        e = mag[k] * (operand + steps * 2.0 ** -22) + fp32[k] + (top[k] * 2.0 ** -39 if dtype == F16 else 0)
        tiny = 2.0 ** -25 if t == F16 else 0.0
        bound = e + (want[k].abs() + e) * HALF[t] + tiny
        assert bool(torch.isfinite(got).all()), k
        off = (got.double() - want[k]).abs() / bound
        assert float(off.max()) <= 1, (k, float(off.max()))


@pytest.mark.parametrize("M,F,K", SIZES)
@pytest.mark.parametrize("dh_size", [1.0, 1e-4, 2e-6])
def test_small_gradients_in_half_precision_keep_their_digits(ctx, M, F, K, dh_size):
    """dg and du of 1e-6 are among half precision's subnormal numbers, whose steps are 6e-8: they are held at another power of two."""
    r = _gradients(ctx, M, F, K, F16, "silu", dh_size)
    _check(*r, M, F, F16, HALF[F16], ("dx", "dw_gate", "dw_up"))


@pytest.mark.parametrize("M,F,K", SIZES)
def test_large_gradients_in_half_precision_do_not_overflow(ctx, M, F, K):
    """dh u act'(g) of a million is past half precision; the weights' gradients in fp32 hold its products."""
    r = _gradients(ctx, M, F, K, F16, "gelu_tanh", 300.0, 3000.0)
    _check(*r, M, F, F16, HALF[F16], ("dw_gate", "dw_up"))


def test_infinities_and_zeros_in_half_precision(ctx):
    """The power of two is that of the finite entries: a row with an infinity makes its own results infinite or NaN, and the other tokens'
    have the bits that they have without it; of gradients that are all 0 everything is 0."""
    M, F, K = 300, 333, 168
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, wg, wu, gate, up, dh = (torch.randn(r, c, generator=gen, device="cuda").half() for r, c in ((M, K), (F, K), (F, K), (M, F), (M, F), (M, F)))
    dh *= 1e-3
    dh[7] = 0

    def gradients():
        out = {"dx": torch.empty(M, K, device="cuda", dtype=F16), "dw_gate": torch.empty(F, K, device="cuda"), "dw_up": torch.empty(F, K, device="cuda")}
        ctx.gated_backward(dh, gate, up, x, wg, wu, act="silu", **out)
        ctx.device_status()
        return out
    want = gradients()
    dh[7, 5], gate[7, 5] = float("inf"), 1.0
    got = gradients()
    others = torch.arange(M, device="cuda") != 7
    assert torch.equal(got["dx"][others], want["dx"][others]) and not bool(torch.isfinite(got["dx"][7]).any())
    columns = torch.arange(F, device="cuda") != 5
    for k in ("dw_gate", "dw_up"):
        assert torch.equal(got[k][columns], want[k][columns]) and not bool(torch.isfinite(got[k][5]).any())
    dh.zero_()
    assert all(bool((t == 0).all()) for t in gradients().values())


@pytest.mark.parametrize("M,F,K", [(20, 333, 165), (300, 520, 264), (1300, 1029, 520)])
def test_a_captured_backward_pass_takes_its_power_of_two_from_its_own_inputs(ctx, M, F, K):
    gen = torch.Generator(device="cuda").manual_seed(2)
    x, wg, wu, gate, up, dh = (torch.randn(r, c, generator=gen, device="cuda").half() for r, c in ((M, K), (F, K), (F, K), (M, F), (M, F), (M, F)))

    def room():
        return {"dx": torch.empty_like(x), "dw_gate": torch.empty(F, K, device="cuda"), "dw_up": torch.empty(F, K, device="cuda")}
    captured, eager = room(), room()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.gated_backward(dh, gate, up, x, wg, wu, **captured)
    for size in (1.0, 2.0 ** -18, 2.0 ** 10):
        dh.copy_(torch.randn(M, F, generator=gen, device="cuda") * size)
        graph.replay()
        ctx.gated_backward(dh, gate, up, x, wg, wu, **eager)
        torch.cuda.synchronize()
        for k in eager:
            assert torch.equal(captured[k], eager[k]) and bool((eager[k] != 0).any())


# on both sides of 2^26 multiply-adds
@pytest.mark.parametrize("M,F,K", SIZES + [(64, 2056, 511), (64, 2056, 510), (2100, 1030, 1000)])
@pytest.mark.parametrize("dtype", [BF, F16])
def test_the_caller_says_how_exact_the_products_operands_are(ctx, M, F, K, dtype):
    """precise: what is off by half a step of dg and du is off by half a step of half a step, at every size."""
    names = ("dx", "dw_gate", "dw_up")
    exact, rounded, auto = (_gradients(ctx, M, F, K, dtype, "silu", 1.0, precise=p) for p in (True, False, None))
    _check(*exact, M, F, dtype, HALF[dtype] ** 2, names)
    _check(*rounded, M, F, dtype, HALF[dtype], names)
    for k in names:
        assert torch.equal(auto[0][k], (exact if M * F * K <= 2 ** 26 else rounded)[0][k])
    if dtype == BF and M > 1:      # (of these sums of roundings fp32 keeps far more)
        want = rounded[1]["dw_gate"]
        off = [float((r[0]["dw_gate"].double() - want).norm() / want.norm()) for r in (exact, rounded)]
        assert off[0] < 2.0 ** -14 and off[1] > 2.0 ** -11


@pytest.mark.parametrize("precise", [True, False, None])
def test_both_ways_of_the_binding_take_what_the_caller_says(ctx, precise, monkeypatch):
    from paper_1811_03617_b200 import gvq
    assert gvq._short is not None
    short = _gradients(ctx, 700, 520, 264, BF, "gelu", 1.0, precise=precise)[0]
    monkeypatch.setattr(gvq, "_short", None)
    for k, t in _gradients(ctx, 700, 520, 264, BF, "gelu", 1.0, precise=precise)[0].items():
        assert torch.equal(t, short[k])


def test_gradients_along_themselves_are_the_differences_of_a_loss(ctx):
    """L = sum(dh * h) in 64 bits, each input moved along its own gradient, so that all terms have one sign: the quotient of differences is
    off by step^2 times a third derivative (1e-8 of it), and a gradient's length by less than its roundings: gate, up, dg, du and the
    gradient itself to 2^-8 each at most, as they average out, and 1 % covers them.  1.1 times a gradient would be ten times that off."""
    M, F, K = 70, 96, 80
    g = torch.Generator(device="cuda").manual_seed(4)
    x, wg, wu, dh = ((torch.randn(r, c, generator=g, device="cuda") * s).to(BF) for r, c, s in
                     ((M, K, 1.0), (F, K, 0.125), (F, K, 0.125), (M, F, 1.0)))
    for name in ("silu", "gelu", "gelu_tanh", "relu", "sigmoid"):
        h, gate, up, dx = (torch.empty(r, c, dtype=BF, device="cuda") for r, c in ((M, F), (M, F), (M, F), (M, K)))
        ctx.gated_forward(x, wg, wu, h, act=name, gate=gate, up=up)
        dwg, dwu = torch.empty(F, K, device="cuda"), torch.empty(F, K, device="cuda")
        ctx.gated_backward(dh, gate, up, x, wg, wu, act=name, dx=dx, dw_gate=dwg, dw_up=dwu)

        def loss(x, wg, wu):
            return float((dh.double() * act(name, x @ wg.T)[0] * (x @ wu.T)).sum())
        ins = [t.double() for t in (x, wg, wu)]
        for j, grad in enumerate((dx, dwg, dwu)):
            norm = float(grad.double().norm())
            d = grad.double() / norm
            e = 1e-4
            moved = [[t + (s * e * d if i == j else 0) for i, t in enumerate(ins)] for s in (1, -1)]
            want = (loss(*moved[0]) - loss(*moved[1])) / (2 * e)
            assert abs(norm - want) <= 0.01 * want, (name, j, norm, want)
