"""Microscaled 4-bit floating point in 64 bits, on the CPU, from the definition in gvq.h."""
import math

import numpy as np
import torch

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
M64 = (1 << 64) - 1


def _mix(z):
    z ^= z >> 30
    z = z * 0xBF58476D1CE4E5B9 & M64
    z ^= z >> 27
    z = z * 0x94D049BB133111EB & M64
    return z ^ (z >> 31)


def u16(seed, node, rows, cols):
    """The 16-bit random numbers of a [rows, cols] matrix."""
    out = np.empty((rows, cols), dtype=np.int64)
    p = np.arange((cols + 1) // 2, dtype=np.uint64)
    h0 = _mix((seed + 0x9E3779B97F4A7C15 * (node + 1)) & M64)
    for i in range(rows):
        h = _mix(h0 ^ (0xD1B54A32D192ED03 * (i + 1) & M64))
        x = np.uint64(h >> 32) ^ ((np.uint64(h & 0xFFFFFFFF) + np.uint64(0x9E3779B9) * (p + np.uint64(1))) & np.uint64(0xFFFFFFFF))
        m = np.uint64(0xFFFFFFFF)
        x ^= x >> np.uint64(16)
        x = x * np.uint64(0x7FEB352D) & m
        x ^= x >> np.uint64(15)
        x = x * np.uint64(0x846CA68B) & m
        x ^= x >> np.uint64(16)
        both = np.stack(((x & np.uint64(0xFFFF)), x >> np.uint64(16)), 1).reshape(-1)[:cols]
        out[i] = both.astype(np.int64)
    return out


def quantize(x, stochastic=False, seed=0, node=0):
    """x [rows, cols] (any float tensor) -> (codes uint8 [rows, cols], scale bytes uint8 [rows, nb], values float64)."""
    x = x.double().cpu().numpy()
    rows, cols = x.shape
    nb = -(-cols // 32)
    codes = np.zeros((rows, cols), dtype=np.uint8)
    scales = np.zeros((rows, nb), dtype=np.uint8)
    values = np.zeros((rows, cols))
    u = u16(seed, node, rows, cols) if stochastic else None
    for b in range(nb):
        c = slice(32 * b, min(cols, 32 * b + 32))
        v = x[:, c]
        top = np.abs(v).max(1)
        bad = ~np.isfinite(v).all(1)
        s = np.zeros(rows, dtype=np.int64)
        for r in range(rows):
            if not bad[r] and top[r] > 0:
                s[r] = max(0, math.frexp(top[r] / 6.0)[1] + 126)          # an upper candidate: 2^(s - 127) >= top / 6 / 2
                while s[r] > 0 and top[r] <= 6.0 * 2.0 ** (s[r] - 1 - 127):
                    s[r] -= 1
                while top[r] > 6.0 * 2.0 ** (s[r] - 127):
                    s[r] += 1
        q = np.where(bad[:, None], 0.0, np.abs(np.where(bad[:, None], 0.0, v)) / 2.0 ** (s[:, None] - 127.0))
        if stochastic:
            step = np.where(q < 2, 0.5, np.where(q < 4, 1.0, 2.0))
            level = (np.floor(65536 * q / step).astype(np.int64) + u[:, c]) >> 16
            idx = np.searchsorted(GRID, level * step)
        else:
            hi = np.clip(np.searchsorted(GRID, q), 1, 7)
            lo = hi - 1
            mid = (GRID[lo] + GRID[hi]) / 2
            idx = np.where((q > mid) | ((q == mid) & (lo % 2 == 1)), hi, lo)
        neg = np.signbit(v) & ~bad[:, None]
        codes[:, c] = idx + 8 * neg
        scales[:, b] = np.where(bad, 255, s)
        val = GRID[idx] * 2.0 ** (s[:, None] - 127.0) * np.where(neg, -1.0, 1.0)
        values[:, c] = np.where(bad[:, None], np.nan, val)
    return codes, scales, values


def pack(codes, scales):
    """The library's layout of quantize()'s codes and scale bytes (bytes outside the matrix 0)."""
    rows, cols = codes.shape
    nb = scales.shape[1]
    full = np.zeros((rows, nb * 32), dtype=np.uint8)
    full[:, :cols] = codes
    packed = (full[:, 0::2] | (full[:, 1::2] << 4)).reshape(-1)
    rt, kt = -(-rows // 128), -(-nb // 4)
    out = np.zeros(rt * kt * 512, dtype=np.uint8)
    for r in range(rows):
        for b in range(nb):
            out[((r // 128) * kt + b // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + b % 4] = scales[r, b]
    return torch.from_numpy(packed), torch.from_numpy(out)
