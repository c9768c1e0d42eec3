"""8-bit integers with a scale a row, in 64 bits, on the CPU, from the definition in gvq.h."""
import numpy as np
import torch

from mx4_reference import u16


def factor(top):
    """The largest float32 r with r * top <= 127, by steps from the rounded quotient."""
    r = np.float32(127.0 / top)
    while float(r) * top > 127.0:
        r = np.nextafter(r, np.float32(0))
    while float(np.nextafter(r, np.float32(np.inf))) * top <= 127.0:
        r = np.nextafter(r, np.float32(np.inf))
    return float(r)


def quantize(x, stochastic=False, seed=0, node=0):
    """x [rows, cols] (any float tensor) -> (codes int8 [rows, pitch], scales float32 [rows], values float64 [rows, cols])."""
    x = x.double().cpu().numpy()
    rows, cols = x.shape
    codes = np.zeros((rows, -(-cols // 16) * 16), dtype=np.int8)
    scales = np.empty(rows, dtype=np.float32)
    u = u16(seed, node, rows, cols) >> 2 if stochastic else None
    for i in range(rows):
        if not np.isfinite(x[i]).all():
            scales[i] = np.nan
            continue
        top = max(float(np.abs(x[i]).max()), 2.0 ** -100)
        at = x[i] * factor(top)              # 24 bits times 24: exact
        if stochastic:
            codes[i, :cols] = (np.floor(at * 16384).astype(np.int64) + u[i]) >> 14
        else:
            codes[i, :cols] = np.rint(at)
        scales[i] = np.float32(top / 127.0)
    return torch.from_numpy(codes), torch.from_numpy(scales), codes[:, :cols].astype(np.float64) * scales[:, None].astype(np.float64)
