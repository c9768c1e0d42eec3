"""The gated block's operators and the 8-bit products together, as a program uses them, and what only such use reaches: refusals of
the entry points, two contexts at once, outputs whose offsets pass 32 bits."""
import math

import pytest
import torch

import int8_reference as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_1811_03617_b200 import gvq
    return gvq.Context(gvq.HostLayout(4, 4, [0], [4]))


def _example():
    import sys
    from pathlib import Path
    sys.path.insert(0, str(Path(__file__).resolve().parent.parent / "examples"))
    import train_gated_block
    return train_gated_block


def test_training_steps_run():
    losses, block = _example().train(steps=3)
    assert len(losses) == 3 and all(math.isfinite(v) for v in losses)
    assert bool(torch.isfinite(block.weights.float()).all()) and bool((block.grad != 0).any())


def test_gradients_of_a_training_step():
    """dh and dW of the last projection are products of what their codes stand for (fp32 roundings aside), dx and the two gradients in front of
    it those of the formula at the dh, gate and up that the step made (dg and du are off by half a step of bfloat16, and so is dx)."""
    example = _example()
    block = example.GatedBlock(3)
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(200, example.D, generator=gen, device="cuda").bfloat16()
    dy = torch.randn(200, example.D, generator=gen, device="cuda").bfloat16()
    y = block.forward(x)
    dx = block.backward(dy, seed=9)
    block.ctx.device_status()
    ctx = block.ctx

    def values(q):
        return q.codes[:, :q.cols].double() * q.scales.double()[:, None]
    h8, w8 = values(ctx.i8_quantize(block.h)), values(ctx.i8_quantize(block.w_down))
    half = 2.0 ** -8
    assert bool(((y.double() - h8 @ w8.T).abs() <= (h8 @ w8.T).abs() * (half + 2.0 ** -22) + 1e-12 * (h8.abs() @ w8.abs().T)).all())
    dy8, dy8_t = ctx.i8_quantize_both(dy, stochastic=True, seed=9)
    want = values(dy8_t) @ values(block.h8_t).T
    assert bool(((block.d_down.double() - want).abs() <= want.abs() * 2.0 ** -22 + 1e-12 * (values(dy8_t).abs() @ values(block.h8_t).abs().T)).all())
    g, u, dh = block.g.double(), block.u.double(), block.dh.double()
    s = torch.sigmoid(g)
    dg, du = dh * u * (s + g * s * (1 - s)), dh * g * s
    wg, wu = block.w_gate.double(), block.w_up.double()
    # (2 % on top of the half steps covers the sums' truncation of 2^-22 of the magnitudes a step of 16 terms, and fp32's activation)
    for got, want, mag, out in ((dx, dg @ wg + du @ wu, dg.abs() @ wg.abs() + du.abs() @ wu.abs(), half),
                                (block.d_gate, dg.T @ x.double(), dg.abs().T @ x.double().abs(), 0),
                                (block.d_up, du.T @ x.double(), du.abs().T @ x.double().abs(), 0)):
        assert bool(((got.double() - want).abs() <= mag * half * 1.02 + want.abs() * out + 1e-9 * mag.max()).all())


@pytest.mark.parametrize("tokens", [1, 7, 64, 200])
def test_an_answer_in_8_bits(tokens):
    example = _example()
    block = example.GatedBlock(5)
    kept = block.kept()
    x = torch.randn(tokens, example.D, device="cuda").bfloat16()
    y = block.answer(x, kept)
    one = torch.cat([block.answer(x[i:i + 1], kept) for i in range(tokens)])
    block.ctx.device_status()
    # a token's codes and its sums depend on its own row alone; the sums are exact, so tokens answered together or one by one agree to the
    # order in which scales are applied (2^-23), which may move an activation, its code and the result's own rounding by a step
    assert float((y.double() - one.double()).norm() / y.double().norm()) <= 2.0 ** -7
    h = torch.nn.functional.silu(x.float() @ block.w_gate.float().T) * (x.float() @ block.w_up.float().T)
    full = h @ block.w_down.float().T
    # 8 bits with a scale a row: an entry is off by half a step, 1 / 254 of its row's largest, which is about 4 times a random row's rms
    assert float((y.float() - full).norm() / full.norm()) <= 4 * 4 / 254 / math.sqrt(3) + 2.0 ** -8


def test_two_contexts_on_two_streams_replay_their_graphs_at_once():
    """Rows that need copies, so that each graph has a workspace of its own."""
    from paper_1811_03617_b200 import gvq
    M, F, K = 300, 515, 333
    made = []
    for i in range(2):
        c, st = gvq.Context(gvq.HostLayout(4, 4, [0], [4])), torch.cuda.Stream()
        gen = torch.Generator(device="cuda").manual_seed(i)
        x, wg, wu = (torch.randn(r, K, generator=gen, device="cuda").bfloat16() for r in (M, F, F))
        h, g, u = (torch.empty(M, F, dtype=torch.bfloat16, device="cuda") for _ in range(3))
        dx, dg, du = torch.empty(M, K, dtype=torch.bfloat16, device="cuda"), torch.empty(F, K, device="cuda"), torch.empty(F, K, device="cuda")

        def step(c=c, x=x, wg=wg, wu=wu, h=h, g=g, u=u, dx=dx, dg=dg, du=du):
            c.gated_forward(x, wg, wu, h, gate=g, up=u)
            c.gated_backward(h, g, u, x, wg, wu, dx=dx, dw_gate=dg, dw_up=du)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            step()
        with torch.cuda.stream(st):
            graph.replay()
        st.synchronize()
        made.append((graph, st, (h, dx, dg, du), [t.clone() for t in (h, dx, dg, du)], step))      # (what the graph reads lives with it)
    for _ in range(20):
        for graph, st, *_ in made:
            with torch.cuda.stream(st):
                graph.replay()
    torch.cuda.synchronize()
    for _, _, outs, want, _ in made:
        for a, b in zip(outs, want):
            assert torch.equal(a, b)


def test_offsets_past_32_bits(ctx):
    """2.3 billion outputs, and 8-bit operands whose codes pass 2^31 bytes along the rows."""
    m, n, k = 70001, 32776, 32
    a, b = torch.randn(m, k, device="cuda"), torch.randn(n, k, device="cuda")
    qa, qb = ctx.i8_quantize(a), ctx.i8_quantize(b)
    out = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    ctx.i8_matmul(qa, qb, out)
    ctx.device_status()
    rows = torch.tensor([0, 1, 40000, 65535, 65536, 69999, 70000], device="cuda")
    want = (qa.codes[rows].double() @ qb.codes.double().T) * qa.scales[rows].double()[:, None] * qb.scales.double()
    assert bool(((out[rows].double() - want).abs() <= want.abs() * (2.0 ** -8 + 2.0 ** -22) + 1e-38).all())
    del out
    rows, cols = 70001, 32000
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    x[-1] = torch.linspace(-3, 3, cols, device="cuda")
    x[:, -1] = torch.linspace(-5, 5, rows, device="cuda").bfloat16()
    q, qt = ctx.i8_quantize_both(x)
    ctx.device_status()
    assert torch.equal(q.codes[-1:].cpu(), R.quantize(x[-1:])[0])      # (by the definition: a factor of 127 / 5 in 64 bits has other ties)
    top = float(x[:, -1].float().abs().max())
    got = qt.codes[-1, :rows].double() * float(qt.scales[-1])
    assert bool(((got - x[:, -1].double()).abs() <= top / 127 * 0.5001).all())
    assert bool((qt.codes[-1, rows:] == 0).all()) and qt.codes.shape == (cols, (rows + 15) // 16 * 16)


def test_refusals(ctx):
    from paper_1811_03617_b200 import gvq
    L, h = gvq.lib(), ctx._h
    x = torch.zeros(64, 64, device="cuda")
    q = gvq.I8(64, 64)
    p, c, s = x.data_ptr(), q.codes_ptr, q.scales_ptr

    def quant(p=p, dt=0, r=64, k=64, ld=64, rnd=0, c=c, s=s, ct=None, st=None, sc=None, n=0):
        return L.gvq_i8_quantize(h, p, dt, r, k, ld, rnd, 0, 0, c, s, ct, st, sc, n)
    assert quant() == 0
    assert quant(p=None) == 1 and quant(c=None) == 1 and quant(s=None) == 1 and quant(c=None, s=None) == 1 and quant(ct=c) == 1
    assert quant(r=0) == 2 and quant(k=0) == 2 and quant(k=-5) == 2 and quant(ld=63) == 2 and quant(dt=3) == 2 and quant(rnd=2) == 2
    assert quant(r=1 << 31, ld=64) == 2
    assert quant(c=c + 8) == 3 and quant(s=s + 2) == 3 and quant(p=p + 2) == 3 and quant(p=p + 1, dt=1) == 3
    assert quant(r=4000, k=1, ld=1, ct=c, st=s) == 5 and quant(r=4000, k=1, ld=1, ct=c, st=s, sc=c, n=3) == 5
    assert L.gvq_i8_dequantize(h, c, s, 64, 64, None, 64) == 1 and L.gvq_i8_dequantize(h, c, s, 64, 64, p, 63) == 2
    assert L.gvq_i8_dequantize(h, c + 1, s, 64, 64, p, 64) == 3

    def mm(a=c, sa=s, b=c, sb=s, m=64, n=64, k=64, o=p, dt=0, ld=64):
        return L.gvq_i8_matmul(h, a, sa, b, sb, m, n, k, o, dt, ld)

    def gated8(a=c, sa=s, b=c, sb=s, m=64, n=64, k=64, o=p, dt=0, ld=64, act=0):
        return L.gvq_i8_gated(h, a, sa, b, sb, b, sb, m, n, k, act, o, dt, ld)
    for f in (mm, gated8):
        assert f() == 0
        assert f(a=None) == 1 and f(sb=None) == 1 and f(o=None) == 1
        assert f(m=0) == 2 and f(n=0) == 2 and f(k=0) == 2 and f(ld=63) == 2 and f(dt=7) == 2 and f(k=131073) == 2 and f(m=1 << 31) == 2
        assert f(a=c + 4) == 3 and f(sb=s + 2) == 3 and f(o=p + 2) == 3
    assert gated8(act=5) == 2 and gated8(act=-1) == 2

    def fwd(x=p, wg=p, wu=p, ldx=64, ldg=64, ldu=64, dt=1, m=32, f=32, k=32, act=0, h_=c, ldh=64, g=None, u=None, ws=None, n=0):
        return L.gvq_gated_forward(h, x, ldx, wg, ldg, wu, ldu, dt, m, f, k, act, h_, ldh, g, 64, u, 64, ws, n)
    x.zero_()
    room = torch.empty(32, 64, dtype=torch.bfloat16, device="cuda").data_ptr()
    assert fwd(h_=room) == 0
    assert fwd(x=None) == 1 and fwd(wu=None) == 1 and fwd(h_=None) == 1 and fwd(g=room) == 1 and fwd(u=room) == 1
    assert fwd(dt=0) == 2 and fwd(m=0) == 2 and fwd(f=-1) == 2 and fwd(ldx=31) == 2 and fwd(ldh=31) == 2 and fwd(act=9) == 2 and fwd(ldg=8) == 2
    assert fwd(x=p + 1) == 3 and fwd(h_=room + 1) == 3
    assert fwd(x=p + 2) == 5 and fwd(ldg=33) == 5 and fwd(x=p + 2, ws=room, n=64) == 5 and fwd(x=p + 2, ws=room + 2, n=1 << 20) == 3

    def bwd(dh=p, g=p, u=p, x=p, wg=p, wu=p, dx=room, dg=None, du=None, dt=1, dwt=0, m=8, f=8, k=8, act=0, ws=c, n=4096, ld=64):
        return L.gvq_gated_backward(h, dh, ld, g, ld, u, ld, x, ld, wg, ld, wu, ld, dt, m, f, k, act, dx, ld, dg, ld, du, ld, dwt, ws, n)
    assert bwd() == 0
    assert bwd(dx=None) == 1 and bwd(dh=None) == 1 and bwd(wg=None) == 1 and bwd(x=None, dg=room) == 1
    assert bwd(x=None) == 0 and bwd(wg=None, wu=None, dx=None, du=room) == 0
    assert bwd(m=0) == 2 and bwd(dt=0) == 2 and bwd(act=7) == 2 and bwd(ld=7) == 2 and bwd(dg=room, dwt=5) == 2
    assert bwd(dh=p + 1) == 3 and bwd(dg=room + 2, dwt=0) == 3 and bwd(ws=c + 8) == 3
    assert bwd(ws=None) == 5 and bwd(n=100) == 5 and bwd(wg=p + 2, n=256) == 5
    ctx.device_status()
    with pytest.raises(ValueError):
        ctx.i8_quantize(x[0])
    with pytest.raises(TypeError):
        ctx.i8_quantize(x.double())
    with pytest.raises(ValueError):
        ctx.i8_matmul(q, gvq.I8(64, 32), x)
    with pytest.raises(ValueError):
        gvq.I8(64, 64, codes=torch.empty(3, dtype=torch.int8, device="cuda"), scales=torch.empty(64, device="cuda"))
    with pytest.raises(ValueError):
        gvq.I8(64, 64, codes=torch.empty(64, 64, dtype=torch.int8, device="cuda"))


def test_both_ways_of_the_binding_give_the_same_bits(ctx, monkeypatch):
    """The long way, which the short one leaves to whatever is not plainly right, makes the same calls."""
    from paper_1811_03617_b200 import gvq

    def everything():
        gen = torch.Generator(device="cuda").manual_seed(0)
        x, wg, wu, dh = (torch.randn(r, c, generator=gen, device="cuda").bfloat16() for r, c in ((70, 129), (200, 129), (200, 129), (70, 200)))
        out = []
        for kw in (dict(), dict(stochastic=True, seed=2 ** 64 - 3, node=5)):
            both = ctx.i8_quantize_both(x, **kw)
            out += [t for q in (*both, ctx.i8_quantize(x, **kw), ctx.i8_quantize_transposed(x, **kw)) for t in (q.codes, q.scales)]
        q, g, u = ctx.i8_quantize(x), ctx.i8_quantize(wg), ctx.i8_quantize(wu)
        kept = gvq.I8(g.rows, g.cols, g.codes, g.scales)
        assert kept.codes is g.codes and kept.scales is g.scales and (kept.rows, kept.cols, kept.device) == (200, 129, 0)
        out.append(ctx.i8_matmul(q, kept, torch.empty(70, 200, device="cuda")))
        assert (q.rows, q.cols, q.device) == (70, 129, 0) and q.codes.dtype is torch.int8 and q.codes.shape == (70, 144) and q.scales.shape == (70,)
        out.append(ctx.i8_matmul(q, g, torch.empty(70, 200, device="cuda")))
        out.append(ctx.i8_gated(q, g, u, torch.empty(70, 200, device="cuda"), act="gelu"))
        h, gate, up = (torch.empty(70, 200, dtype=torch.bfloat16, device="cuda") for _ in range(3))
        out += [ctx.gated_forward(x, wg, wu, h, act="gelu_tanh", gate=gate, up=up), gate, up]
        dx, dg, du = torch.empty_like(x), torch.empty(200, 129, device="cuda"), torch.empty(200, 129, device="cuda")
        ctx.gated_backward(dh, gate, up, x, wg, wu, act="gelu_tanh", dx=dx, dw_gate=dg, dw_up=du)
        du2 = torch.empty_like(du)
        ctx.gated_backward(dh, gate, up, x, None, None, act="gelu_tanh", dw_up=du2)
        return out + [dx, dg, du, du2]
    short = everything()
    assert gvq._short is not None
    monkeypatch.setattr(gvq, "_short", None)
    for a, b in zip(short, everything()):
        assert torch.equal(a, b)


def test_the_short_way_leaves_errors_to_the_long_one(ctx):
    from paper_1811_03617_b200 import gvq
    x, q = torch.zeros(64, 64, device="cuda"), gvq.I8(64, 64)
    h, bf = ctx._address, x.bfloat16()
    s = gvq._short
    assert s.i8_quantize(h, 0, x, True, False, False, 0, 0) is not None
    for args in ((0, 0, x), (h, 0, x[0]), (h, 0, x.t()[:, ::2]), (h, 0, x.double()), (h, 0, x.cpu()), (h, 0, None), (h, 0, x[:0]), (h, 0, x.expand(64, 64)[:1, :0])):
        assert s.i8_quantize(*args, True, False, False, 0, 0) is None
    assert s.i8_quantize(h, 0, x, True, False, False, "1", 0) is None and s.i8_quantize(h, 0, x) is None
    assert s.i8_quantize(h, 0, x[:1].expand(64, 64), True, True, False, 0, 0) is None          # rows 0 entries apart
    assert not s.i8_matmul(h, 0, q, q, x.double()) and not s.i8_matmul(h, 0, q, gvq.I8(64, 32), x) and not s.i8_matmul(h, 0, q, object(), x)
    assert not s.i8_matmul(h, 0, gvq.I8.__new__(gvq.I8), q, x) and not s.i8_matmul(0, 0, q, q, x)
    assert not s.i8_gated(h, 0, q, q, q, x, -1) and not s.i8_gated(h, 0, q, q, gvq.I8(32, 64), x, 0)
    assert not s.gated_forward(h, 0, x, x, x, x, 0, None, None) and not s.gated_forward(h, 0, bf, bf, bf, x, 0, None, None)
    assert not s.gated_forward(h, 0, bf, bf, bf, bf, 0, bf, None) and not s.gated_forward(h, 0, bf, bf[:, :32], bf, bf, 0, None, None)
    assert not s.gated_backward(h, 0, bf, bf, bf, bf, bf, bf, 0, None, None, None)
    assert not s.gated_backward(h, 0, bf, bf, bf, None, bf, bf, 0, None, x, None) and not s.gated_backward(h, 0, bf, bf, bf, bf, None, bf, 0, bf, None, None)
    assert not s.gated_backward(h, 0, bf, bf, bf, bf, bf, bf, 0, None, x, bf) and not s.gated_backward(h, 0, bf, bf, bf, bf, bf, bf, 9, bf, None, None)
    c, w = torch.zeros(64, 64, dtype=torch.int8, device="cuda"), torch.ones(64, device="cuda")
    for args in ((q, 64, 64, c, w[:32]), (q, 64, 64, c.t(), w[::2]), (q, 64, 60, c.cpu(), w), (q, 64, 64, c.byte(), w), (q, 64, 64, c, w.double()), (q, 0, 64, c, w),
                 (q, 64, 1 << 40, c, w), (q, 64.0, 64, c, w), (q, 64, 64, c, None), (object(), 64, 64, c, w), (q, 64, 80, c, w)):
        assert not s.i8_fill(*args)
    assert q.codes is not c and s.i8_fill(q, 64, 64, c, w) and q.codes is c and q.scales is w
    for args in ((64, 64, c, w[:32]), (64, 64, c, None), (64, 80, c, w), (64, 64, c.byte(), w)):
        with pytest.raises(ValueError):
            gvq.I8(*args)
    assert gvq.I8(64.0, 64, c, w).rows == 64
    ctx.device_status()
    with pytest.raises(ValueError):
        ctx.i8_matmul(q, gvq.I8(64, 32), x)
    with pytest.raises(gvq.GvqError):
        ctx.i8_quantize(x[:1].expand(64, 64))
    closed = gvq.Context(gvq.HostLayout(4, 4, [0], [4]))
    closed.close()
    with pytest.raises(gvq.GvqError):
        closed.i8_quantize(x)


def test_threads_quantize_columns_of_different_lengths_at_once():
    """Strips of different sizes in shared memory, whose limit the first launches raise, from threads with a context each."""
    import threading
    from paper_1811_03617_b200 import gvq
    rows, got = (450, 900, 1500, 2900), {}
    xs = {r: torch.randn(r, 130, generator=torch.Generator().manual_seed(r)).half() for r in rows}

    def work(r):
        ctx, x = gvq.Context(gvq.HostLayout(4, 4, [0], [4])), xs[r].cuda()
        with torch.cuda.stream(torch.cuda.Stream()):
            x.record_stream(torch.cuda.current_stream())
            torch.cuda.current_stream().wait_stream(torch.cuda.default_stream())
            q = [ctx.i8_quantize_transposed(x) for _ in range(5)][-1]
            got[r] = q.codes.cpu(), q.scales.cpu()
    threads = [threading.Thread(target=work, args=(r,)) for r in rows]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for r in rows:
        codes, scales, _ = R.quantize(xs[r].t().contiguous())
        assert torch.equal(got[r][0], codes) and torch.equal(got[r][1], scales)
