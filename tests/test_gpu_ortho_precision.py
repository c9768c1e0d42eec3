"""The bounds that gvq.h states for the orthogonalised update's error, for spectra that are hard for it, in all of its
forms.  The bounds were set from a simulation of the roundings in 64 bits: at most 2.8e-3, 3.6e-3, 1.04e-2 and 1.05e-4."""
import pytest
import torch

from paper_1811_03617_b200 import workloads as W

pytestmark = pytest.mark.gpu

A, B, C, EPS = 3.4445, -4.7750, 2.0315, 1e-7
FACTORS, RANDOM, ALIKE, WHOLE = 3.2e-3, 4e-3, 1.5e-2, 2e-4


def exact(u):
    x = u.double()
    x = x / (x.norm() + EPS)
    for _ in range(5):
        g = x @ x.t()
        x = A * x + (B * g + C * g @ g) @ x
    return x


def families(r, c, gen):
    """(name, bound, r x c matrix) for 8 <= r <= c, as many for every size."""
    def randn(*s):
        return torch.randn(s, generator=gen, device="cuda", dtype=torch.double)

    def zeros():
        return torch.zeros((r, c), device="cuda", dtype=torch.double)
    yield "gauss", FACTORS, randn(r, c)
    yield "uniform", FACTORS, torch.rand((r, c), generator=gen, device="cuda", dtype=torch.double) - 0.5
    for k in (1, 2, 4, 8, r // 2, r):
        for noise in (0.0, 1e-3, 1e-2, 1e-1):
            yield f"rank {k}, noise {noise}", FACTORS, randn(r, k) @ randn(k, c) + noise * randn(r, c)
    u, v = torch.linalg.qr(randn(r, r))[0], torch.linalg.qr(randn(c, r))[0].t()
    yield "orthogonal", RANDOM, v
    for e in (1, 2, 4, 8):
        yield f"decay {e}", RANDOM, (u * torch.logspace(0, -e, r, device="cuda", dtype=torch.double)) @ v
    for k in (1, 2, 3, 5, 16):
        k = min(k, r // 2)
        x, y = zeros(), zeros()
        x[:k], y[:, :k] = randn(k, c), randn(r, k)
        yield f"{k} rows", ALIKE, x
        yield f"{k} columns", ALIKE, y
    yield "ones", ALIKE, zeros() + 1
    yield "nearly ones", ALIKE, 1 + 0.01 * randn(r, c)
    yield "signs of rank 1", ALIKE, randn(r, 1).sign() @ randn(1, c).sign()
    yield "signs", ALIKE, randn(r, c).sign()
    for k in (1, 2, r // 4, r // 2, r):
        x = zeros()
        x[:k, :k] = torch.eye(k, device="cuda")
        yield f"identity of {k}", ALIKE, x
    x = zeros()
    x[0] = 1
    yield "a row of ones", ALIKE, x


# every matrix of the first two plans fits an SM; a cluster shares those of the next three; the rest take a launch a product, the
# last ones on pairs of CTAs
PLANS = [[(8, 12), (16, 64), (24, 60), (64, 64), (16, 144), (48, 400), (64, 576)], [(50, 100), (128, 128), (128, 320)],
         [(64, 3000)], [(40, 1500), (64, 576)], [(128, 1000), (90, 321)],
         [(8, 12), (40, 500), (64, 576), (128, 1100), (129, 257)], [(256, 512), (300, 700)], [(515, 1027)], [(700, 700)], [(512, 4608)],
         [(1024, 1024)] * 2, [(2000, 2000)], [(1300, 2500), (129, 400)]]


@pytest.mark.parametrize("shapes", PLANS, ids=lambda s: "+".join("%dx%d" % x for x in s))
@pytest.mark.parametrize("tall", [False, True])
def test_errors_stay_within_the_stated_bounds(shapes, tall):
    from paper_1811_03617_b200 import gvq
    lens = [m * n for m, n in shapes]
    off = [0]
    for n in lens[:-1]:
        off.append(off[-1] + -(-n // 4) * 4)
    w = W.custom("precision", 92, 64, 4, 2, 1, lens, layer_off=off)
    ctx = gvq.Context(w)
    rows, cols = [m for m, _ in shapes], [n for _, n in shapes]
    plan = gvq.OrthoPlan(ctx, cols, rows) if tall else gvq.OrthoPlan(ctx, rows, cols)
    whole = all(r <= 64 and c <= 832 or r <= 128 and c <= 320 for r, c in shapes) and (max(rows) <= 64 or max(cols) <= 320)
    gen = torch.Generator(device="cuda").manual_seed(sum(lens))
    out, worst = torch.empty(w.M, device="cuda"), {}
    for members in zip(*[list(families(r, c, gen)) for r, c in shapes]):
        g = torch.zeros(w.M, device="cuda")
        for (r, c), o, (_, _, u) in zip(shapes, off, members):
            u = u * 10.0 ** float(torch.randint(-6, 3, (1,), generator=gen, device="cuda"))
            g[o:o + r * c] = (u.t() if tall else u).float().reshape(-1)
        plan.orthogonalize(g, out)
        for (r, c), o, (name, bound, _) in zip(shapes, off, members):
            def of(flat):
                return flat[o:o + r * c].view(c, r).t() if tall else flat[o:o + r * c].view(r, c)
            want = exact(of(g))
            err = float((of(out).double() - want).norm() / want.norm())
            if whole and c <= 64:
                bound = WHOLE
            worst[(r, c), bound] = max(worst.get(((r, c), bound), (0.0, "")), (err, name))
    ctx.device_status()
    print({k: ("%.2e" % v[0], v[1]) for k, v in worst.items()})
    assert all(err <= bound for (_, bound), (err, _) in worst.items()), worst


@pytest.mark.parametrize("shapes", [[(64, 576)], [(515, 1027)]])
@pytest.mark.parametrize("norm", [1e-10, 1e-8, 1e-7, 1e15])
def test_errors_stay_within_the_bound_for_small_and_large_gradients(shapes, norm):
    from paper_1811_03617_b200 import gvq
    (r, c), = shapes
    ctx = gvq.Context(gvq.HostLayout(64, 4, [0], [r * c]))
    plan = gvq.OrthoPlan(ctx, [r], [c])
    gen = torch.Generator(device="cuda").manual_seed(r)
    u = torch.randn((r, 4), generator=gen, device="cuda") @ torch.randn((4, c), generator=gen, device="cuda")
    u += 0.01 * torch.randn((r, c), generator=gen, device="cuda")
    u *= norm / u.norm()
    out = torch.empty(r * c, device="cuda")
    plan.orthogonalize(u.view(-1), out)
    want = exact(u)
    assert float((out.view(r, c).double() - want).norm() / want.norm()) <= FACTORS


@pytest.mark.parametrize("outputs,inputs", [(192, 64), (64, 576), (300, 129)])
def test_a_layer_in_flatten_order_moves_as_its_transpose(outputs, inputs):
    """[outputs][inputs] by default and [inputs][filters] with `flattened`: the same update of the same layer."""
    from paper_1811_03617_b200 import gvq
    gen = torch.Generator(device="cuda").manual_seed(outputs)
    g, w = (torch.randn((outputs, inputs), generator=gen, device="cuda") for _ in range(2))
    moved = []
    for flat in (False, True):
        ctx = gvq.Context(gvq.HostLayout(64, 4, [0], [outputs * inputs]))
        shape = (inputs, outputs) if flat else (outputs, inputs)
        plan = gvq.OrthoPlan(ctx, [shape[0]], [shape[1]], flattened=flat)
        gf, wf = [(x.t() if flat else x).clone(memory_format=torch.contiguous_format).view(-1) for x in (g, w)]
        plan.step(gf, torch.zeros_like(gf), wf, lr=0.5, beta=0.0, nesterov=False)
        moved.append((wf.view(shape).t() if flat else wf.view(shape)) - w)
    assert float((moved[0] - moved[1]).norm() / moved[0].norm()) <= 2 * FACTORS
    want = -0.5 * max(1.0, outputs / inputs) ** 0.5 * (exact(g) if outputs <= inputs else exact(g.t()).t())
    assert float((moved[1].double() - want).norm() / want.norm()) <= FACTORS + 1e-6
