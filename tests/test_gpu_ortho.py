"""The orthogonalised update on the GPU against the formula in 64 bits: shapes and orientations, what a call must not
touch, precision, refusals."""
import math

import numpy as np
import pytest
import torch

from paper_1811_03617_b200 import workloads as W

pytestmark = pytest.mark.gpu

A, B, C, EPS = 3.4445, -4.7750, 2.0315, 1e-7
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -9, torch.float16: 2.0 ** -12}


def exact(u):
    """Five steps in 64 bits on the shorter side."""
    x = u.double()
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    x = x / (x.norm() + EPS)
    for _ in range(5):
        g = x @ x.t()
        x = A * x + (B * g + C * g @ g) @ x
    return x.t() if tall else x


# Half-precision operands: each rounding is 2^-12 / sqrt(3) (rms) of an entry; the steps' condition and number made of it
# up to 2.1e-3 of the result's norm in a simulation of the roundings on Gaussian, low-rank and decaying spectra of sides 64
# to 1024.  Twice that is the bar; a side below 64 averages over few singular values and may sit where the step's slope
# is largest: five times.
def bar(m, n):
    return 4.2e-3 if min(m, n) >= 64 else 1.05e-2


def kinds(m, n, seed, kind):
    g = torch.Generator().manual_seed(seed)
    if kind == "gauss":
        return torch.randn(m, n, generator=g)
    k = min(8, m, n)
    return torch.randn(m, k, generator=g) @ torch.randn(k, n, generator=g) + 0.1 * torch.randn(m, n, generator=g)


def layout_of(shapes, gap=8):
    off, at = [], 0
    for m, n in shapes:
        off.append(at)
        at += -(-m * n // 4) * 4 + gap
    return W.custom("ortho", 91, 64, 4, 2, 1, [m * n for m, n in shapes], layer_off=off)


def make(shapes, rows=None, cols=None, **kw):
    from paper_1811_03617_b200 import gvq
    w = layout_of(shapes)
    ctx = gvq.Context(w)
    return w, gvq.OrthoPlan(ctx, rows or [m for m, _ in shapes], cols or [n for _, n in shapes], **kw)


SHAPES = [(1, 1), (1, 7), (9, 1), (5, 7), (16, 27), (64, 64), (64, 576), (100, 64), (129, 65), (128, 128), (257, 255), (255, 600),
          (515, 1027), (1152, 128), (1027, 515), (300, 300), (8, 5000), (5000, 3), (640, 641)]


@pytest.mark.parametrize("kind", ["gauss", "lowrank"])
def test_orthogonalize_all_shapes_in_one_call(kind):
    w, plan = make(SHAPES)
    flat = torch.full((w.M,), float("nan"))
    mats = []
    for i, ((m, n), o) in enumerate(zip(SHAPES, w.layer_off)):
        u = kinds(m, n, i, kind) * 10.0 ** (i % 7 - 4)
        mats.append(u)
        flat[o:o + m * n] = u.reshape(-1)
    g = flat.cuda()
    for dtype in DT.values():
        out = torch.full((w.M,), 7.0, dtype=dtype, device="cuda")
        plan.orthogonalize(g, out)
        plan.ctx.device_status()
        got = out.cpu()
        for u, (m, n), o in zip(mats, SHAPES, w.layer_off):
            want = exact(u)
            err = float((got[o:o + m * n].view(m, n).double() - want).norm() / want.norm())
            assert err <= bar(m, n) + 2 * HALF_ULP[dtype], (m, n, err)
            got[o:o + m * n] = 7.0
        assert bool((got == 7.0).all())                      # nothing outside the matrices was written
        again = torch.empty_like(out)
        plan.orthogonalize(g, again)
        at = torch.cat([torch.arange(o, o + m * n) for (m, n), o in zip(SHAPES, w.layer_off)]).cuda()
        assert torch.equal(out[at], again[at])               # the same bits every time


# plans whose matrices all fit one SM: both rooms for the short side (64 and 128), both orientations, one block of 64 columns
# to thirteen, single rows and columns
SMALL = [[(1, 1), (1, 7), (9, 1), (5, 7), (16, 27), (64, 64), (63, 65), (64, 576), (576, 64), (3, 800), (832, 64), (33, 257)],
         [(128, 128), (65, 1), (100, 300), (320, 128), (127, 129), (96, 257), (1, 320), (66, 64)], [(64, 64)], [(300, 100)]]


@pytest.mark.parametrize("shapes", SMALL)
@pytest.mark.parametrize("dtype", list(DT))
def test_small_matrices(shapes, dtype):
    w, plan = make(shapes)
    gen = torch.Generator().manual_seed(9)
    g = torch.randn(w.M, generator=gen)
    for i, ((m, n), o) in enumerate(zip(shapes, w.layer_off)):
        if i % 3 == 1:
            g[o:o + m * n] = kinds(m, n, i, "lowrank").reshape(-1) * 1e-3
    g = g.cuda()
    out = torch.full((w.M,), 7.0, dtype=DT[dtype], device="cuda")
    plan.orthogonalize(g, out)
    mo = torch.randn(w.M, generator=gen).cuda()
    mo0 = mo.clone()
    wt = torch.full((w.M,), 2.0, dtype=DT[dtype], device="cuda")
    plan.step(g, mo, wt, lr=0.5, weight_decay=0.5, beta=0.5, nesterov=True)
    plan.ctx.device_status()
    rest = torch.ones(w.M, dtype=torch.bool, device="cuda")
    for (m, n), o in zip(shapes, w.layer_off):
        sl = slice(o, o + m * n)
        rest[sl] = False
        want = exact(g[sl].view(m, n)).reshape(-1)
        err = float((out[sl].double() - want).norm() / want.norm())
        assert err <= bar(m, n) + 2 * HALF_ULP[DT[dtype]], (m, n, err)
        mom = 0.5 * mo0[sl].double() + g[sl].double()
        assert bool(((mo[sl].double() - mom).abs() <= mom.abs() * 2.0 ** -24).all())
        want = exact((g[sl].double() + 0.5 * mom).view(m, n)).reshape(-1)
        s = math.sqrt(max(1.0, m / n))
        new = 0.75 * 2.0 - 0.5 * s * want
        err = float((wt[sl].double() - new).norm())
        assert err <= 0.5 * s * float(want.norm()) * bar(m, n) + float(new.norm()) * (2 * HALF_ULP[DT[dtype]] + 2.0 ** -22), (m, n)
    assert bool((out[rest] == 7.0).all()) and bool((wt[rest] == 2.0).all()) and torch.equal(mo[rest], mo0[rest])
    again = torch.empty_like(out)
    plan.orthogonalize(g, again)
    assert torch.equal(out[~rest], again[~rest])


# Plans whose matrices are shared by the CTAs of a cluster: two, four and eight of them, long sides that leave the last ones
# little or nothing, either orientation, rows of whole quads and others.
CLUSTER = [[(64, 1500), (64, 1), (7, 100)], [(20, 3333)], [(3333, 50), (50, 65)], [(37, 801), (802, 37), (64, 640)], [(128, 1000), (5, 7), (90, 321)],
           [(500, 100)], [(63, 5001)]]


@pytest.mark.parametrize("shapes", CLUSTER)
@pytest.mark.parametrize("dtype", list(DT))
def test_matrices_that_a_cluster_shares(shapes, dtype):
    w, plan = make(shapes)
    gen = torch.Generator().manual_seed(5)
    g = torch.randn(w.M, generator=gen)
    mo, wt = torch.randn(w.M, generator=gen), torch.randn(w.M, generator=gen).to(DT[dtype])
    out = torch.full((w.M,), 7.0, dtype=DT[dtype], device="cuda")
    plan.orthogonalize(g.cuda(), out)
    dm, dw = mo.cuda(), wt.cuda()
    plan.step(g.cuda(), dm, dw, lr=0.5, weight_decay=0.1, beta=0.9)
    plan.ctx.device_status()
    got, gm, gw = out.cpu(), dm.cpu(), dw.cpu()
    inside = torch.zeros(w.M, dtype=torch.bool)
    for (m, n), o in zip(shapes, w.layer_off):
        at = slice(o, o + m * n)
        inside[at] = True
        want = exact(g[at].view(m, n))
        err = float((got[at].view(m, n).double() - want).norm() / want.norm())
        assert err <= bar(m, n) + 2 * HALF_ULP[DT[dtype]], (m, n, err)
        new_m = 0.9 * mo[at].double() + g[at].double()
        assert float((gm[at].double() - new_m).abs().max()) <= 1e-6
        want = exact((g[at].double() + 0.9 * new_m).view(m, n)) * math.sqrt(max(1.0, m / n)) * 0.5
        moved = wt[at].view(m, n).double() * (1 - 0.5 * 0.1) - gw[at].view(m, n).double()
        slack = 2 * HALF_ULP[DT[dtype]] * float(wt[at].double().norm() + want.norm())
        assert float((moved - want).norm()) <= (bar(m, n) * float(want.norm()) + slack), (m, n)
    assert bool((got[~inside] == 7.0).all()) and torch.equal(gm[~inside], mo[~inside]) and torch.equal(gw[~inside], wt[~inside])
    again = torch.full((w.M,), 7.0, dtype=DT[dtype], device="cuda")
    plan.orthogonalize(g.cuda(), again)
    assert torch.equal(again, out)


def test_a_small_plan_gives_what_a_larger_one_gives():
    """The same matrix alone (one SM) and next to one that does not fit (tiles): two summation orders of one algorithm."""
    w1, one = make([(64, 320)])
    w2, two = make([(64, 320), (400, 400)])
    g = torch.randn(w2.M, device="cuda")
    a, b = torch.empty(w1.M, device="cuda"), torch.empty(w2.M, device="cuda")
    one.orthogonalize(g[:w1.M].clone(), a)
    two.orthogonalize(g, b)
    x, y = a[:64 * 320].double(), b[:64 * 320].double()
    assert float((x - y).norm() / y.norm()) <= 2 * bar(64, 320)


@pytest.mark.parametrize("shape", [(40, 200), (128, 200)])
def test_small_zero_and_non_finite(shape):
    m, n = shape
    w, plan = make([shape] * 3)
    g = torch.randn(w.M)
    o = w.layer_off
    g[o[0]:o[0] + m * n] = 0.0
    g[o[1] + 5] = float("inf")
    out = torch.empty(w.M, device="cuda")
    plan.orthogonalize(g.cuda(), out)
    plan.ctx.device_status()
    assert bool((out[o[0]:o[0] + m * n] == 0).all())
    got = out[o[1]:o[1] + m * n]
    assert not bool((torch.isfinite(got) & (got != 0)).any())
    want = exact(g[o[2]:o[2] + m * n].view(m, n))
    assert float((out[o[2]:o[2] + m * n].view(m, n).cpu().double() - want).norm() / want.norm()) <= bar(m, n)


@pytest.mark.parametrize("dtype", list(DT))
def test_many_large_matrices(dtype):
    """Enough 256 x 256 tiles for pairs of CTAs: wide, tall and square matrices with ragged edges in one plan."""
    shapes = [(1030, 2100)] * 2 + [(1500, 700)] * 2 + [(900, 900)] * 3 + [(24, 3000), (2999, 40), (257, 1030)]
    shapes += [(1285, 1281)] * 2 + [(64, 576), (1024, 1024), (512, 4608)]
    w, plan = make(shapes)
    gen = torch.Generator(device="cuda").manual_seed(8)
    g = torch.randn(w.M, generator=gen, device="cuda")
    for i, ((m, n), o) in enumerate(zip(shapes, w.layer_off)):
        if i % 2:       # a few strong directions
            g[o:o + m * n] = (torch.randn(m, 6, generator=gen, device="cuda") @ torch.randn(6, n, generator=gen, device="cuda")).view(-1) + 0.1 * g[o:o + m * n]
    out = torch.full((w.M,), 7.0, dtype=DT[dtype], device="cuda")
    plan.orthogonalize(g, out)
    plan.ctx.device_status()
    mo = torch.zeros(w.M, device="cuda")
    wt = torch.full((w.M,), 2.0, dtype=DT[dtype], device="cuda")
    plan.step(g, mo, wt, lr=0.5, weight_decay=0.5, beta=0.5, nesterov=False)
    rest = torch.ones(w.M, dtype=torch.bool, device="cuda")
    for (m, n), o in zip(shapes, w.layer_off):
        sl = slice(o, o + m * n)
        rest[sl] = False
        want = exact(g[sl].view(m, n)).reshape(-1)
        err = float((out[sl].double() - want).norm() / want.norm())
        assert err <= bar(m, n) + 2 * HALF_ULP[DT[dtype]], (m, n, err)
        s = math.sqrt(max(1.0, m / n))
        new = 0.75 * 2.0 - 0.5 * s * want
        err = float((wt[sl].double() - new).norm())
        assert err <= 0.5 * s * float(want.norm()) * bar(m, n) + float(new.norm()) * (2 * HALF_ULP[DT[dtype]] + 2.0 ** -22), (m, n)
    assert bool((out[rest] == 7.0).all()) and bool((wt[rest] == 2.0).all())
    assert torch.equal(mo[~rest], g[~rest])


@pytest.mark.parametrize("shape", [(8, 900001), (900001, 5)])
def test_a_matrix_of_very_many_tiles(shape):
    """More tiles than a CTA keeps the descriptions of."""
    m, n = shape
    w, plan = make([shape])
    u = kinds(m, n, 3, "lowrank")
    g = torch.zeros(w.M)
    g[:m * n] = u.reshape(-1)
    out = torch.empty(w.M, device="cuda")
    plan.orthogonalize(g.cuda(), out)
    plan.ctx.device_status()
    want = exact(u)
    err = float((out[:m * n].view(m, n).cpu().double() - want).norm() / want.norm())
    assert err <= bar(m, n) + 2 * HALF_ULP[torch.float32], err


# Short sides' factors are sums of two halves: a simulation of the roundings on Gaussian matrices and on eight strong directions
# over noise gave at most 1.35e-3 up to 48 (A and P both) and 1.7e-3 up to 128 (A alone); long sides up to 64 take part whole,
# and what is left there is fp32's.  The bars are half as much again.
@pytest.mark.parametrize("kind", ["gauss", "lowrank"])
@pytest.mark.parametrize("shapes", [
    [(8, 8), (8, 12), (12, 8), (16, 64), (64, 16), (33, 60), (64, 64)], [(8, 300), (300, 12), (16, 100), (32, 500), (48, 400), (600, 40)],
    [(64, 96), (200, 64), (100, 300), (128, 320), (320, 90)], [(8, 4000), (3000, 32), (48, 1500), (30, 2000)],
    [(64, 3000), (1440, 90), (128, 1000), (800, 128), (120, 200)]])
def test_short_sides_keep_their_precision(shapes, kind):
    w, plan = make(shapes)
    flat = torch.zeros(w.M)
    mats = [kinds(m, n, 11 * i + m, kind) for i, (m, n) in enumerate(shapes)]
    for u, o in zip(mats, w.layer_off):
        flat[o:o + u.numel()] = u.reshape(-1)
    out = torch.empty(w.M, device="cuda")
    plan.orthogonalize(flat.cuda(), out)
    plan.ctx.device_status()
    whole = all(max(s) <= 320 or min(s) <= 64 and max(s) <= 832 for s in shapes)      # (one SM)
    for u, (m, n), o in zip(mats, shapes, w.layer_off):
        want = exact(u)
        err = float((out[o:o + m * n].view(m, n).cpu().double() - want).norm() / want.norm())
        limit = 1e-4 if whole and max(m, n) <= 64 else 2e-3 if min(m, n) <= 48 else 2.6e-3
        assert err <= limit, (m, n, err)


def test_singular_values_end_near_one():
    shapes = [(192, 320), (700, 96)]
    w, plan = make(shapes)
    g = torch.zeros(w.M)
    for (m, n), o in zip(shapes, w.layer_off):
        g[o:o + m * n] = torch.randn(m * n)
    out = torch.zeros(w.M, device="cuda")
    plan.orthogonalize(g.cuda(), out)
    for (m, n), o in zip(shapes, w.layer_off):
        s = torch.linalg.svdvals(out[o:o + m * n].view(m, n).double())
        assert 0.6 < float(s.min()) and float(s.max()) < 1.3


def test_invariant_to_the_scale_of_the_gradient_by_powers_of_two():
    w, plan = make([(130, 200)])
    g = torch.randn(w.M, device="cuda")
    one, other = torch.empty(w.M, device="cuda"), torch.empty(w.M, device="cuda")
    plan.orthogonalize(g, one)
    plan.orthogonalize(g * 2.0 ** 20, other)    # eps = 1e-7 against a norm of 161: below fp32's resolution
    assert torch.equal(one[:130 * 200], other[:130 * 200])


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("dtype", list(DT))
def test_step(dtype, nesterov):
    shapes = [(64, 576), (300, 128), (7, 9), (129, 257)]
    scales = [1.0, 0.5, 2.0, 0.25]
    w, plan = make(shapes, scales=scales)
    gen = torch.Generator().manual_seed(4)
    g, mo, wt = torch.randn(w.M, generator=gen), torch.randn(w.M, generator=gen), torch.randn(w.M, generator=gen) * 0.1
    wt = wt.to(DT[dtype])
    lr, wd, beta = 0.02, 0.1, 0.9
    dg, dmo, dw = g.cuda(), mo.cuda(), wt.cuda()
    plan.step(dg, dmo, dw, lr=lr, weight_decay=wd, beta=beta, nesterov=nesterov)
    assert torch.equal(dg.cpu(), g)
    gm, gw = dmo.cpu(), dw.cpu()
    keep = torch.ones(w.M, dtype=torch.bool)
    for (m, n), o, s in zip(shapes, w.layer_off, scales):
        sl = slice(o, o + m * n)
        keep[sl] = False
        mom = beta * mo[sl].double() + g[sl].double()
        # beta is a float in the call; one fused multiply-add
        assert bool(((gm[sl].double() - mom).abs() <= mom.abs() * 2.0 ** -24 + mo[sl].double().abs() * 2.0 ** -25).all())
        u = g[sl].double() + beta * mom if nesterov else mom
        o_ = exact(u.view(m, n)).reshape(-1)
        want = (1 - lr * wd) * wt[sl].double() - lr * s * o_
        err = (gw[sl].double() - want).norm()
        # the update's error, the weights' rounding, and fp32's in the sum
        assert float(err) <= lr * s * float(o_.norm()) * bar(m, n) + float(want.norm()) * (2 * HALF_ULP[DT[dtype]] + 2.0 ** -22)
    assert torch.equal(gm[keep], mo[keep]) and torch.equal(gw[keep], wt[keep])


def test_default_scale_and_layers_left_alone():
    shapes = [(64, 16), (10, 30), (16, 64)]
    w, plan = make(shapes, rows=[64, 0, 16], cols=[16, 0, 64])
    g = torch.randn(w.M, device="cuda")
    mo, wt = torch.zeros(w.M, device="cuda"), torch.zeros(w.M, device="cuda")
    plan.step(g, mo, wt, lr=1.0, beta=0.0, nesterov=False)
    o = torch.zeros(w.M, device="cuda")
    plan.orthogonalize(g, o)
    at = w.layer_off
    assert torch.allclose(wt[at[0]:at[0] + 1024], -2.0 * o[at[0]:at[0] + 1024], rtol=1e-6, atol=0)      # sqrt(64 / 16)
    assert torch.allclose(wt[at[2]:at[2] + 1024], -o[at[2]:at[2] + 1024], rtol=1e-6, atol=0)
    assert bool((wt[at[1]:at[1] + 300] == 0).all()) and bool((mo[at[1]:at[1] + 300] == 0).all())


def test_zero_and_non_finite_matrices_stay_apart():
    shapes = [(70, 140), (64, 64), (200, 100), (33, 90)]
    w, plan = make(shapes)
    g = torch.randn(w.M)
    o = w.layer_off
    g[o[1]:o[1] + 64 * 64] = 0.0
    g[o[2] + 77] = float("nan")
    out = torch.empty(w.M, device="cuda")
    plan.orthogonalize(g.cuda(), out)
    got = out.cpu()
    assert bool((got[o[1]:o[1] + 64 * 64] == 0).all())
    assert bool(torch.isnan(got[o[2]:o[2] + 200 * 100]).all())
    for i in (0, 3):
        m, n = shapes[i]
        want = exact(g[o[i]:o[i] + m * n].view(m, n))
        assert float((got[o[i]:o[i] + m * n].view(m, n).double() - want).norm() / want.norm()) <= bar(m, n)
    # the next call is not touched by what the last one left behind
    g[o[2] + 77] = 0.0
    plan.orthogonalize(g.cuda(), out)
    assert bool(torch.isfinite(out[o[2]:o[2] + 200 * 100]).all())


def test_step_after_the_exchange_on_one_stream_and_in_a_graph():
    """decompress' output feeds the step on a side stream, captured and replayed."""
    shapes = [(64, 64), (128, 96)]
    w, plan = make(shapes)
    side = torch.cuda.Stream()
    g, mo, wt = torch.randn(w.M).cuda(), torch.zeros(w.M, device="cuda"), torch.randn(w.M).cuda()
    mo2, wt2 = mo.clone(), wt.clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(3):
            plan.step(g, mo2, wt2, lr=0.1)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        plan.step(g, mo, wt, lr=0.1)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for (m, n), o in zip(shapes, w.layer_off):
        assert torch.equal(mo[o:o + m * n], mo2[o:o + m * n]) and torch.equal(wt[o:o + m * n], wt2[o:o + m * n])


@pytest.mark.parametrize("shape", [(300, 400), (60, 100), (1600, 1600)])
def test_a_wait_that_runs_out_is_reported_and_the_plan_recovers(shape):
    from paper_1811_03617_b200 import gvq
    w, plan = make([shape])
    n = shape[0] * shape[1]
    g, out = torch.randn(w.M, device="cuda"), torch.empty(w.M, device="cuda")
    plan.orthogonalize(g, out)
    good = out[:n].clone()
    plan.ctx.set_limits(wait_cycles=2_000_000)
    plan.ctx.test_drop_load(True)
    try:
        plan.orthogonalize(g, out)
        with pytest.raises(gvq.GvqError) as e:
            plan.ctx.device_status()
        assert e.value.status == 9
    finally:
        plan.ctx.test_drop_load(False)
        plan.ctx.set_limits()
    plan.orthogonalize(g, out)
    plan.ctx.device_status()
    assert torch.equal(out[:n], good)


def test_a_wait_of_a_pair_that_runs_out_is_reported_and_the_plan_recovers():
    """The same with tiles of CTA pairs."""
    test_a_wait_that_runs_out_is_reported_and_the_plan_recovers((2000, 2000))


def test_a_cluster_whose_wait_runs_out_is_reported_and_the_plan_recovers():
    from paper_1811_03617_b200 import gvq
    shape = (64, 1500)
    w, plan = make([shape])
    g = torch.randn(w.M).cuda()
    good, out = torch.zeros(w.M, device="cuda"), torch.zeros(w.M, device="cuda")
    plan.orthogonalize(g, good)
    plan.ctx.device_status()
    plan.ctx.set_limits(wait_cycles=2_000_000)
    plan.ctx.test_drop_load(True)
    try:
        plan.orthogonalize(g, out)
        with pytest.raises(gvq.GvqError) as e:
            plan.ctx.device_status()
        assert e.value.status == 9
    finally:
        plan.ctx.test_drop_load(False)
        plan.ctx.set_limits()
    plan.orthogonalize(g, out)
    plan.ctx.device_status()
    assert torch.equal(out, good)


def test_a_plan_can_be_destroyed_after_its_context():
    """As garbage collection may order it."""
    w, plan = make([(16, 32)])
    plan.ctx.close()
    plan.close()
    _, plan = make([(16, 32)])
    out = torch.empty(w.M, device="cuda")
    plan.orthogonalize(torch.randn(w.M, device="cuda"), out)
    plan.ctx.device_status()


def test_refusals():
    import ctypes
    from paper_1811_03617_b200 import gvq
    L = gvq.lib()
    w = layout_of([(8, 16), (4, 4)])
    ctx = gvq.Context(w)
    lay = ctypes.byref(ctx.layout.c)
    i2 = ctypes.c_int32 * 2

    def need(r, c):
        return L.gvq_ortho_workspace_bytes(lay, i2(*r), i2(*c))
    n = need((8, 4), (16, 4))
    assert n > 0 and need((8, 0), (16, 0)) < n
    assert need((8, 4), (16, 5)) == -1 and need((8, -4), (16, -4)) == -1 and need((0, 4), (16, 4)) == -1
    assert need((8, 16), (16, 1)) > 0 and L.gvq_ortho_workspace_bytes(lay, None, i2(16, 4)) == -1
    big = gvq.HostLayout(64, 4, [0], [40000 * 40000])
    assert L.gvq_ortho_workspace_bytes(ctypes.byref(big.c), (ctypes.c_int32 * 1)(40000), (ctypes.c_int32 * 1)(40000)) == -1
    ws = torch.empty(n + 256, dtype=torch.uint8, device="cuda")
    p = ctypes.c_void_p()

    def create(ctx_h=ctx._h, r=(8, 4), c=(16, 4), s=None, at=ws.data_ptr(), size=n):
        st = L.gvq_ortho_create(ctypes.byref(p), ctx_h, i2(*r), i2(*c), s, at, size)
        if st == 0:
            L.gvq_ortho_destroy(p)
        return st
    assert create() == 0
    assert create(ctx_h=None) == 1 and create(r=(8, 5)) == 2 and create(size=n - 1) == 5 and create(at=None) == 5
    assert create(at=ws.data_ptr() + 16) == 3
    assert create(s=(ctypes.c_float * 2)(1.0, float("nan"))) == 2
    plan = gvq.OrthoPlan(ctx, [8, 4], [16, 4])
    g = torch.zeros(w.M, device="cuda")
    mo, wt = torch.zeros_like(g), torch.zeros_like(g)
    a, b, c = g.data_ptr(), mo.data_ptr(), wt.data_ptr()
    step = L.gvq_ortho_step
    assert step(plan._h, a, b, 0.9, 1, c, 0, 0.1, 0.0) == 0
    assert step(None, a, b, 0.9, 1, c, 0, 0.1, 0.0) == 1 and step(plan._h, None, b, 0.9, 1, c, 0, 0.1, 0.0) == 1
    assert step(plan._h, a, None, 0.9, 1, c, 0, 0.1, 0.0) == 1 and step(plan._h, a, b, 0.9, 1, None, 0, 0.1, 0.0) == 1
    assert step(plan._h, a, b, 1.0, 1, c, 0, 0.1, 0.0) == 2 and step(plan._h, a, b, -0.1, 1, c, 0, 0.1, 0.0) == 2
    assert step(plan._h, a, b, float("nan"), 1, c, 0, 0.1, 0.0) == 2 and step(plan._h, a, b, 0.9, 1, c, 0, float("inf"), 0.0) == 2
    assert step(plan._h, a, b, 0.9, 1, c, 3, 0.1, 0.0) == 2 and step(plan._h, a, a, 0.9, 1, c, 0, 0.1, 0.0) == 2
    assert step(plan._h, a, b, 0.9, 1, b, 0, 0.1, 0.0) == 2 and step(plan._h, a + 4, b, 0.9, 1, c, 0, 0.1, 0.0) == 3
    assert L.gvq_orthogonalize(plan._h, a, a, 0) == 2 and L.gvq_orthogonalize(plan._h, a, None, 0) == 1
    assert L.gvq_orthogonalize(plan._h, a, c + 2, 1) == 3 and L.gvq_orthogonalize(plan._h, a, c, 9) == 2
    torch.cuda.synchronize()
    with pytest.raises(ValueError):
        plan.step(g[:-1], mo, wt, lr=0.1)
    with pytest.raises(TypeError):
        plan.step(g.half(), mo, wt, lr=0.1)
    with pytest.raises(TypeError):
        plan.orthogonalize(g, wt.double())
    with pytest.raises(ValueError):
        gvq.OrthoPlan(ctx, [8], [16])
    # a plan without matrices does nothing
    none = gvq.OrthoPlan(ctx, [0, 0], [0, 0])
    wt.fill_(3.0)
    none.step(g, mo, wt, lr=0.1)
    assert bool((wt == 3.0).all())
