"""Host-only parts of the 4-bit format and of the orthogonalised update (no GPU)."""
import ctypes

import numpy as np
import pytest
import torch

import mx4_reference as R


@pytest.fixture(scope="module")
def gvq():
    from paper_1811_03617_b200 import build, gvq as _gvq
    build.build()
    return _gvq


def test_sizes_of_a_quantized_matrix(gvq):
    L = gvq.lib()
    for rows, cols in ((1, 1), (1, 32), (7, 33), (128, 128), (129, 130), (515, 1083), (4096, 16384)):
        nb = -(-cols // 32)
        assert L.gvq_mx4_codes_bytes(rows, cols) == rows * nb * 16
        assert L.gvq_mx4_scales_bytes(rows, cols) == -(-rows // 128) * -(-nb // 4) * 512
    for rows, cols in ((0, 1), (1, 0), (-1, 5), (1 << 38, 1), (1 << 30, 1 << 30)):
        assert L.gvq_mx4_codes_bytes(rows, cols) == -1 and L.gvq_mx4_scales_bytes(rows, cols) == -1
    with pytest.raises(ValueError):
        gvq.Mx4(0, 5)
    with pytest.raises(ValueError):
        gvq.Mx4(4, 4, codes=torch.zeros(64, dtype=torch.uint8))


def test_null_arguments_are_refused_without_a_gpu(gvq):
    L = gvq.lib()
    assert L.gvq_mx4_quantize(None, None, 0, 1, 1, 1, 0, 0, 0, None, None, None, None) == 1
    assert L.gvq_mx4_dequantize(None, None, None, 1, 1, None, 1) == 1
    assert L.gvq_mx4_matmul(None, None, None, None, None, 1, 1, 1, None, 0, 1) == 1
    assert L.gvq_mx4_quantize_aggregate(None, None, 1, 0, 0, 0, None, None, None) == 1
    assert L.gvq_mx4_dequantize_aggregate(None, None, None, None, 1, None) == 1
    p = ctypes.c_void_p()
    assert L.gvq_ortho_create(None, None, None, None, None, None, 0) == 1
    assert L.gvq_ortho_create(ctypes.byref(p), None, None, None, None, None, 0) == 1
    assert L.gvq_ortho_destroy(None) == 0
    assert L.gvq_ortho_step(None, None, None, 0.9, 1, None, 0, 0.1, 0.0) == 1
    assert L.gvq_orthogonalize(None, None, None, 0) == 1


def test_workspace_of_the_update(gvq):
    i2 = ctypes.c_int32 * 2
    lay = gvq.HostLayout(64, 4, [0, 1000], [960, 12])
    need = gvq.lib().gvq_ortho_workspace_bytes
    both, one = need(ctypes.byref(lay.c), i2(24, 3), i2(40, 4)), need(ctypes.byref(lay.c), i2(24, 0), i2(40, 0))
    assert both > one > 0 and need(ctypes.byref(lay.c), i2(0, 0), i2(0, 0)) == 0
    assert need(ctypes.byref(lay.c), i2(24, 3), i2(41, 4)) == -1 and need(ctypes.byref(lay.c), i2(-24, 3), i2(-40, 4)) == -1
    assert need(None, i2(24, 3), i2(40, 4)) == -1 and need(ctypes.byref(lay.c), None, i2(40, 4)) == -1


# ---- pins of the reference the GPU tests compare with

def test_reference_scale_is_the_smallest_that_holds_the_block():
    x = torch.tensor([[6.0], [6.0000005], [3.0], [1e-45], [0.0], [3.4e38]]).repeat(1, 32)
    _, s, v = R.quantize(x)
    assert list(s[:, 0]) == [127, 128, 126, 0, 0, 253]
    assert v[0, 0] == 6.0 and v[2, 0] == 3.0 and v[4, 0] == 0.0


def test_reference_rounds_ties_to_the_even_code():
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0] + [0.0] * 24)[None]
    codes, s, v = R.quantize(ties)
    assert s[0, 0] == 127 and list(v[0, :8]) == [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0]
    assert list(R.quantize(-ties)[0][0, :8]) == [8, 10, 10, 12, 12, 14, 14, 15]


def test_reference_stochastic_rounding_is_unbiased_and_stays_between_neighbours():
    x = torch.linspace(-6, 6, 128).view(1, 128).repeat(2000, 1)
    x[:, ::32] = 6.0
    _, _, v = R.quantize(x, True, 5, 1)
    r = x[0].abs().numpy()
    step = np.where(r < 2, 0.5, np.where(r < 4, 1.0, 2.0))
    assert (np.abs(v - x.numpy()) < step).all()
    # five standard errors of a rounding (at most half a step) and the resolution of u
    assert (np.abs(v.mean(0) - x[0].numpy()) <= step * (5 * 0.5 / 2000 ** 0.5 + 2.0 ** -16)).all()


def test_reference_random_numbers_look_uniform():
    u = R.u16(12345, 2, 64, 512).astype(np.float64) / 65536
    n = u.size
    assert abs(u.mean() - 0.5) < 5 * (1 / 12 / n) ** 0.5
    assert abs(np.corrcoef(u[:, 0::2].ravel(), u[:, 1::2].ravel())[0, 1]) < 5 / (n / 2) ** 0.5
    assert abs(np.corrcoef(u[:-1].ravel(), u[1:].ravel())[0, 1]) < 5 / n ** 0.5


def test_running_out_of_host_memory_is_an_error_code():
    """No exception leaves a C entry: 4 million layers under a limit of the address space that their tables exceed."""
    import subprocess
    import sys
    from pathlib import Path
    code = """
import ctypes, resource
import numpy as np
from paper_1811_03617_b200 import gvq
L, n = gvq.lib(), 4_000_000
off, length, rows = np.arange(n, dtype=np.int64) * 4, np.full(n, 4, dtype=np.int64), np.full(n, 2, dtype=np.int32)
p = lambda a, t: a.ctypes.data_as(ctypes.POINTER(t))
layout = gvq._Layout(64, 4, n, p(off, ctypes.c_int64), p(length, ctypes.c_int64))
need = lambda: L.gvq_ortho_workspace_bytes(ctypes.byref(layout), p(rows, ctypes.c_int32), p(rows, ctypes.c_int32))
held = int(open('/proc/self/statm').read().split()[0]) * resource.getpagesize()
resource.setrlimit(resource.RLIMIT_AS, (held + (200 << 20), resource.RLIM_INFINITY))
less = need()
resource.setrlimit(resource.RLIMIT_AS, (resource.RLIM_INFINITY, resource.RLIM_INFINITY))
print('less', less, 'enough', need() > 0)
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=Path(__file__).resolve().parent.parent)
    assert r.returncode == 0, r.stderr[-500:]
    assert r.stdout.split() == ["less", "-1", "enough", "True"]
