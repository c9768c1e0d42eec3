"""Host-only parts of the 8-bit format and of the gated block: sizes, what the entry points and the binding refuse before anything
reaches a GPU, and pins of the reference that the GPU tests compare with."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch

import int8_reference as R
from test_operator_refusals import Device, Library

BF, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def gvq():
    from paper_1811_03617_b200 import build, gvq as _gvq
    build.build()
    return _gvq


def test_sizes(gvq):
    L = gvq.lib()
    for rows, cols in ((1, 1), (1, 16), (7, 33), (515, 1083), (4096, 16384)):
        assert L.gvq_i8_codes_bytes(rows, cols) == rows * -(-cols // 16) * 16
        assert L.gvq_i8_scratch_bytes(rows, cols) >= 0
    assert L.gvq_i8_scratch_bytes(2900, 10 ** 6) == 0 and L.gvq_i8_scratch_bytes(3200, 10) > 0
    for rows, cols in ((0, 1), (1, 0), (-1, 5), (1 << 31, 1), (1, (1 << 31) - 1000), (1 << 30, 1 << 30)):
        assert L.gvq_i8_codes_bytes(rows, cols) == -1 and L.gvq_i8_scratch_bytes(rows, cols) == -1
        with pytest.raises(ValueError):
            gvq.I8(rows, cols)
    need = L.gvq_gated_workspace_bytes
    assert need(5, 7, 9, 0, 1) == 0
    assert need(5, 7, 9, 1, 1) >= 2 * 5 * 8 * 2
    assert need(5, 7, 9, 0, 0) >= (5 + 2 * 7) * 16 * 2 and need(5, 7, 9, 1, 0) == need(5, 7, 9, 1, 1) + need(5, 7, 9, 0, 0)
    assert need(0, 7, 9, 1, 1) == -1 and need(5, -7, 9, 1, 1) == -1 and need(5, 7, 1 << 31, 0, 0) == -1


def test_null_arguments_are_refused_without_a_gpu(gvq):
    L, n = gvq.lib(), None
    assert L.gvq_i8_quantize(n, n, 0, 1, 1, 1, 0, 0, 0, n, n, n, n, n, 0) == 1
    assert L.gvq_i8_dequantize(n, n, n, 1, 1, n, 1) == 1
    assert L.gvq_i8_matmul(n, n, n, n, n, 1, 1, 1, n, 0, 1) == 1
    assert L.gvq_i8_gated(n, n, n, n, n, n, n, 1, 1, 1, 0, n, 0, 1) == 1
    assert L.gvq_gated_forward(n, n, 1, n, 1, n, 1, 1, 1, 1, 1, 0, n, 1, n, 0, n, 0, n, 0) == 1
    assert L.gvq_gated_backward(n, n, 1, n, 1, n, 1, n, 1, n, 1, n, 1, 1, 1, 1, 1, 0, n, 1, n, 1, n, 1, 0, n, 0) == 1


class Matrix(Device):
    """A CUDA matrix as far as the binding looks at one."""

    def __init__(self, rows, cols, dtype=BF, device=0, stride=None, at=4096):
        super().__init__(rows * cols, dtype, device=device, shape=(rows, cols))
        self._stride, self._at = stride or (cols, 1), at

    def stride(self):
        return self._stride

    def data_ptr(self):
        return self._at

    def element_size(self):
        return 4 if self.dtype is F32 else 2

    def new_empty(self, n):
        return Device(n, self.dtype, device=self._device)


def quantized(rows, cols, device=0):
    return SimpleNamespace(rows=rows, cols=cols, codes_ptr=256, scales_ptr=512, device=device)


@pytest.fixture
def made(gvq, monkeypatch):
    ctx = object.__new__(gvq.Context)
    ctx._h, ctx.device = 1, 0
    ctx._raw_stream = lambda: 0
    fake = Library()
    fake.gvq_i8_scratch_bytes = lambda r, c: 0
    fake.gvq_gated_workspace_bytes = lambda *a: 4096
    monkeypatch.setattr(gvq, "lib", lambda: fake)
    monkeypatch.setattr(torch, "empty", lambda *a, **k: Device(4096))
    yield ctx, fake
    ctx._h = None


def test_8_bit_operands(made):
    ctx, fake = made
    x, out = Matrix(100, 128), Matrix(100, 70, F32)
    a, b = quantized(100, 128), quantized(70, 128)
    ctx.i8_quantize(x)
    ctx.i8_quantize_both(x, out=quantized(100, 128), out_t=quantized(128, 100))
    ctx.i8_dequantize(quantized(100, 70), out)
    ctx.i8_matmul(a, b, out)
    ctx.i8_gated(a, b, b, out, act="relu")
    good = ["gvq_i8_quantize", "gvq_i8_quantize", "gvq_i8_dequantize", "gvq_i8_matmul", "gvq_i8_gated"]
    assert fake.names() == good
    for call in (lambda: ctx.i8_quantize(Matrix(100, 128, device=1)), lambda: ctx.i8_quantize(Device(128)),
                 lambda: ctx.i8_quantize(Matrix(100, 128, stride=(1, 100))), lambda: ctx.i8_quantize(x, out=quantized(99, 128)),
                 lambda: ctx.i8_quantize(x, out=quantized(100, 128, 1)), lambda: ctx.i8_quantize_transposed(x, out=quantized(100, 128)),
                 lambda: ctx.i8_dequantize(quantized(100, 71), out), lambda: ctx.i8_dequantize(quantized(100, 70), Matrix(100, 70)),
                 lambda: ctx.i8_dequantize(quantized(100, 70, 1), out), lambda: ctx.i8_matmul(a, quantized(70, 127), out),
                 lambda: ctx.i8_matmul(a, quantized(71, 128), out), lambda: ctx.i8_matmul(quantized(99, 128), b, out),
                 lambda: ctx.i8_matmul(a, quantized(70, 128, 1), out), lambda: ctx.i8_matmul(a, b, Matrix(100, 70, F32, 1)),
                 lambda: ctx.i8_gated(a, b, quantized(71, 128), out), lambda: ctx.i8_gated(a, b, quantized(70, 128, 1), out),
                 lambda: ctx.i8_gated(a, b, b, Matrix(100, 71)), lambda: ctx.i8_gated(a, b, b, out, act="tanh")):
        with pytest.raises((ValueError, TypeError)):
            call()
    with pytest.raises(TypeError):
        ctx.i8_quantize(Matrix(100, 128, torch.float64))
    with pytest.raises(TypeError):
        ctx.i8_matmul(a, b, Matrix(100, 70, torch.float64))
    assert fake.names() == good


def test_gated_operands(made):
    ctx, fake = made
    M, F, K = 10, 24, 16
    x, w, h = Matrix(M, K), Matrix(F, K), Matrix(M, F)
    ctx.gated_forward(x, w, w, h)
    ctx.gated_forward(x, w, w, h, gate=h, up=h)
    assert fake.calls[-1][1][-1] == 0          # rows at 16-byte boundaries: no workspace
    for odd in (Matrix(M, K, stride=(K + 1, 1)), Matrix(M, K, at=4098)):
        ctx.gated_forward(odd, w, w, h)
        assert fake.calls[-1][1][-1] == 4096
    ctx.gated_forward(Matrix(1, K, stride=(K + 1, 1)), w, w, Matrix(1, F))
    assert fake.calls[-1][1][-1] == 0          # (one row alone)
    n = len(fake.names())
    for args, kw in (((x, w, Matrix(F, K + 1), h), {}), ((x, Matrix(F, K + 1), w, h), {}), ((x, w, w, Matrix(M, F + 1)), {}),
                     ((x, w, Matrix(F + 1, K), h), {}), ((x, w, w, h), dict(gate=h)), ((x, w, w, h), dict(up=h)),
                     ((x, w, w, h), dict(gate=h, up=Matrix(M + 1, F))), ((x, w, w, h), dict(act="swish")),
                     ((Matrix(M, K, device=1), w, w, h), {}), ((x, Matrix(F, K, device=1), w, h), {}),
                     ((x, w, w, Matrix(M, F, stride=(1, M))), {})):
        with pytest.raises(ValueError):
            ctx.gated_forward(*args, **kw)
    for args in ((Matrix(M, K, F32), w, w, h), (x, Matrix(F, K, F16), w, h), (x, w, w, Matrix(M, F, F32))):
        with pytest.raises(TypeError):
            ctx.gated_forward(*args)

    dx, dw = Matrix(M, K), Matrix(F, K, F32)
    ctx.gated_backward(h, h, h, x, w, w, dx=dx, dw_gate=dw, dw_up=dw)
    ctx.gated_backward(h, h, h, None, w, w, dx=dx)
    ctx.gated_backward(h, h, h, x, None, None, dw_up=dw)
    assert len(fake.names()) == n + 3
    for args, kw in (((h, h, h, x, w, w), {}), ((h, h, h, None, w, w), dict(dw_up=dw)), ((h, h, h, x, None, w), dict(dx=dx)),
                     ((h, h, Matrix(M, F + 1), x, w, w), dict(dx=dx)), ((h, h, h, Matrix(M + 1, K), w, w), dict(dw_up=dw)),
                     ((h, h, h, x, w, w), dict(dx=Matrix(M + 1, K))), ((h, h, h, x, w, w), dict(dx=dx, dw_gate=Matrix(F, K + 1, F32))),
                     ((h, h, h, x, w, w), dict(dx=dx, act="none")), ((h, h, h, x, w, w), dict(dx=Matrix(M, K, device=1)))):
        with pytest.raises(ValueError):
            ctx.gated_backward(*args, **kw)
    for kw in (dict(dx=Matrix(M, K, F32)), dict(dw_gate=dw, dw_up=Matrix(F, K, BF)), dict(dw_gate=Matrix(F, K, torch.float64))):
        with pytest.raises(TypeError):
            ctx.gated_backward(h, h, h, x, w, w, **kw)
    assert len(fake.names()) == n + 3


# ---- pins of the reference the GPU tests compare with

def test_reference_factor_is_the_largest_that_holds_the_row():
    rng = np.random.default_rng(1)
    for top in [127.0, 1.0, 2.0 ** -100, 3.4e38, 1e-20] + list(np.float32(rng.uniform(0.5, 2, 50)).astype(float)):
        r = R.factor(top)
        assert r * top <= 127.0 and float(np.nextafter(np.float32(r), np.float32(np.inf))) * top > 127.0


def test_reference_codes():
    x = torch.tensor([[127.0, 0.5, 1.5, -0.5, -2.5, 63.0], [0.0, -0.0, 0.0, 0.0, 0.0, 0.0], [1.0, float("nan"), 0, 0, 0, 0]])
    codes, scales, values = R.quantize(x)
    assert codes.shape == (3, 16) and codes[0, :6].tolist() == [127, 0, 2, 0, -2, 63] and not codes[0, 6:].any()
    assert scales[0] == 1.0 and not codes[1:].any() and torch.isnan(scales[2]) and np.isnan(values[2]).all()
    # 4096 roundings of 0.3 of a step: their mean is off by less than five standard errors and the 2^-14 that u leaves
    x = torch.full((4096, 2), 0.3)
    x[:, 1] = 127.0
    mean = R.quantize(x, True, 5)[0][:, 0].double().mean()
    assert abs(float(mean) - 0.3) <= 5 * (0.3 * 0.7 / 4096) ** 0.5 + 2.0 ** -14
