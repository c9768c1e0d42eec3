"""What the binding of the 4-bit exchange and of the orthogonalised update refuses before anything reaches the library.
Host only: the library is a stand-in that counts calls, and no pointer is followed."""
from types import SimpleNamespace

import pytest
import torch


class Library:
    """Counts the calls of every entry point; all succeed."""

    def __init__(self):
        self.calls = []

    def gvq_status_string(self, status):
        return b"refused"

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 0
        return call

    def names(self):
        return [n for n, _ in self.calls if n != "gvq_set_stream"]


class Device(SimpleNamespace):
    """A CUDA tensor as far as the binding looks at one."""

    def __init__(self, numel, dtype=torch.float32, contiguous=True, cuda=True, device=0, shape=None):
        super().__init__(dtype=dtype, is_cuda=cuda, shape=shape or (numel,), device=f"cuda:{device}")
        self._n, self._c, self._device = numel, contiguous, device

    def numel(self):
        return self._n

    def is_contiguous(self):
        return self._c

    def data_ptr(self):
        return 4096

    def get_device(self):
        return self._device if self.is_cuda else -1

    def stride(self):
        return self.shape[1], 1


def matrix(rows, cols, device=0):
    return SimpleNamespace(rows=rows, cols=cols, codes_ptr=256, scales_ptr=512, device=device)


@pytest.fixture
def made(monkeypatch):
    """(context of 100 slices of 16 and a tail of 8, stand-in library)"""
    from paper_1811_03617_b200 import gvq
    ctx = object.__new__(gvq.Context)
    ctx._h, ctx.device, ctx.S, ctx.d, ctx.M, ctx.n_layers = 1, 0, 100, 16, 1608, 1
    ctx._raw_stream = lambda: 0
    fake = Library()
    monkeypatch.setattr(gvq, "lib", lambda: fake)
    yield ctx, fake
    ctx._h = None        # nothing to destroy


def test_exchange_takes_one_matrix_of_slices_per_node(made):
    ctx, fake = made
    g = [Device(1608) for _ in range(3)]
    total, q = Device(1608), [matrix(100, 16) for _ in range(3)]
    ctx.mx4_quantize_aggregate(g, total, out=q)
    ctx.mx4_quantize_aggregate(g, None, out=q)
    ctx.mx4_quantize_aggregate(g, total)
    assert fake.names() == ["gvq_mx4_quantize_aggregate"] * 3
    for bad in (q[:2], q + q[:1], [], q[:2] + [matrix(99, 16)], q[:2] + [matrix(100, 8)], [matrix(16, 100)] * 3):
        with pytest.raises(ValueError):
            ctx.mx4_quantize_aggregate(g, total, out=bad)
    assert len(fake.names()) == 3


def test_exchange_takes_flat_float32_gradients(made):
    ctx, fake = made
    good = Device(1608)
    for bad, error in ((Device(1607), ValueError), (Device(1608, contiguous=False), ValueError),
                       (Device(1608, cuda=False), ValueError), (Device(1608, torch.bfloat16), TypeError)):
        with pytest.raises(error):
            ctx.mx4_quantize_aggregate([good, bad], good)
        with pytest.raises(error):
            ctx.mx4_quantize_aggregate([good, good], bad)
        with pytest.raises(error):
            ctx.mx4_dequantize_aggregate([matrix(100, 16)] * 2, [good, bad], good)
        with pytest.raises(error):
            ctx.mx4_dequantize_aggregate([matrix(100, 16)] * 2, [good, good], bad)
    assert fake.names() == []


def test_receiver_takes_the_slices_and_the_gradients_of_the_same_nodes(made):
    ctx, fake = made
    g, total, q = [Device(1608)] * 2, Device(1608), [matrix(100, 16)] * 2
    ctx.mx4_dequantize_aggregate(q, g, total)
    ctx.mx4_dequantize_aggregate(q, None, total)
    assert fake.names() == ["gvq_mx4_dequantize_aggregate"] * 2
    for bad_q, bad_g in ((q[:1], g), (q + q, g), (q, g[:1]), (q, g + g), ([matrix(100, 16), matrix(50, 32)], g), ([matrix(101, 16)] * 2, g)):
        with pytest.raises(ValueError):
            ctx.mx4_dequantize_aggregate(bad_q, bad_g, total)
    assert len(fake.names()) == 2


@pytest.mark.parametrize("closed", ["context", "plan"])
def test_a_plan_is_not_used_after_its_context_or_itself_was_closed(made, closed):
    from paper_1811_03617_b200 import gvq
    ctx, fake = made
    plan = object.__new__(gvq.OrthoPlan)
    plan.ctx, plan._h = ctx, 2
    g, mo, w = Device(1608), Device(1608), Device(1608)
    plan.step(g, mo, w, lr=0.1)
    plan.orthogonalize(g, w)
    assert fake.names() == ["gvq_ortho_step", "gvq_orthogonalize"]
    (ctx if closed == "context" else plan).close()
    for call in (lambda: plan.step(g, mo, w, lr=0.1), lambda: plan.orthogonalize(g, w)):
        with pytest.raises(gvq.GvqError) as e:
            call()
        assert e.value.status == 1
    assert not [n for n in fake.names()[2:] if n in ("gvq_ortho_step", "gvq_orthogonalize")]
    plan._h = None


def test_a_stream_that_somebody_else_set_does_not_stay(made):
    """gvq_set_stream is public: a call made through the binding goes to torch's current stream all the same."""
    from paper_1811_03617_b200 import gvq
    ctx, fake = made

    def stream_of_the_library():
        return [args[1] for name, args in fake.calls if name == "gvq_set_stream"][-1]
    ctx.mx4_quantize_aggregate([Device(1608)], Device(1608))
    gvq.lib().gvq_set_stream(ctx._h, 77)
    ctx.mx4_quantize_aggregate([Device(1608)], Device(1608))
    assert stream_of_the_library() == 0
    ctx._raw_stream = lambda: 5
    ctx.mx4_quantize_aggregate([Device(1608)], Device(1608))
    assert stream_of_the_library() == 5


def test_operands_are_on_the_context_s_device(made):
    """What lies on another device would be read or written through a pointer that this one may not follow."""
    ctx, fake = made
    here, there = Device(12800, shape=(100, 128)), Device(12800, shape=(100, 128), device=1)
    out = Device(10000, shape=(100, 100))
    q, q_t, far, far_t = matrix(100, 128), matrix(128, 100), matrix(100, 128, 1), matrix(128, 100, 1)
    ctx.mx4_quantize_both(here, out=q, out_t=q_t)
    ctx.mx4_dequantize(q, here)
    ctx.mx4_matmul(q, q, out)
    assert len(fake.names()) == 3
    flat, flat_there = Device(1608), Device(1608, device=1)
    for call in (lambda: ctx.mx4_quantize(there), lambda: ctx.mx4_quantize(here, out=far),
                 lambda: ctx.mx4_quantize_transposed(here, out=far_t), lambda: ctx.mx4_dequantize(far, here),
                 lambda: ctx.mx4_dequantize(q, there), lambda: ctx.mx4_matmul(far, q, out), lambda: ctx.mx4_matmul(q, far, out),
                 lambda: ctx.mx4_matmul(q, q, Device(10000, shape=(100, 100), device=1)),
                 lambda: ctx.mx4_quantize_aggregate([flat, flat_there], flat),
                 lambda: ctx.mx4_quantize_aggregate([flat], flat_there),
                 lambda: ctx.mx4_quantize_aggregate([flat], flat, out=[matrix(100, 16, 1)]),
                 lambda: ctx.mx4_dequantize_aggregate([matrix(100, 16, 1)], None, flat)):
        with pytest.raises(ValueError):
            call()
    assert len(fake.names()) == 3


def test_scales_of_layers_in_flatten_order(made, monkeypatch):
    """[inputs][filters]: the factor grows with the columns.  Otherwise the library's default, rows over columns, is left alone."""
    from paper_1811_03617_b200 import gvq
    ctx, fake = made
    ctx.n_layers = 4
    ctx.layout = SimpleNamespace(c=gvq._Layout())
    monkeypatch.setattr(torch, "empty", lambda *a, **k: Device(256))

    def scales(**kw):
        plan = gvq.OrthoPlan(ctx, [64, 16, 0, 10], [16, 64, 0, 10], **kw)
        plan._h = None
        got = [args for name, args in fake.calls if name == "gvq_ortho_create"][-1][4]
        return None if got is None else list(got)
    assert scales() is None
    assert scales(flattened=True) == [1.0, 2.0, 1.0, 1.0]
    assert scales(flattened=[True, False, True, False]) == [1.0, 1.0, 1.0, 1.0]
    assert scales(flattened=[False, True, False, True]) == [2.0, 2.0, 1.0, 1.0]
    assert scales(scales=[3.0, 1.0, 1.0, 0.5]) == [3.0, 1.0, 1.0, 0.5]
    for bad in (dict(flattened=[True]), dict(flattened=True, scales=[1.0] * 4)):
        with pytest.raises(ValueError):
            scales(**bad)
