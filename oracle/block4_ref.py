"""Oracle of the 4-bit form of a matrix and of layers of blocks whose operands are in it: numpy, 64 bits."""
from __future__ import annotations

import numpy as np

from oracle import grouped_ref as G

WORTH = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def row_bytes(k: int):
    """bytes of a row of codes and of scales"""
    return (k + 127) // 128 * 64, (k + 511) // 512 * 16


def number(q: float) -> int:
    """The nearest of WORTH to q >= 0, halfway the one of even number."""
    off = np.abs(WORTH - q)
    near = np.flatnonzero(off == off.min())
    return int(near[0] if len(near) == 1 or near[0] % 2 == 0 else near[1])


def pack(x):
    """x [rows][k] float32 -> codes uint8 [rows][64 ceil(k / 128)], scale uint8 [rows][16 ceil(k / 512)]."""
    x = np.asarray(x, np.float64)
    rows, k = x.shape
    nc, ns = row_bytes(k)
    code, scale = np.zeros((rows, 2 * nc), np.uint8), np.zeros((rows, ns), np.uint8)
    for r in range(rows):
        for b in range((k + 31) // 32):
            v = x[r, 32 * b:min(32 * b + 32, k)]
            if not np.isfinite(v).all():
                scale[r, b] = 255
                continue
            top, e = np.abs(v).max(), -126
            if top > 0:
                e = max(int(np.floor(np.log2(top))) - 4, -126)
                while top / 2.0 ** e >= 7 and e < 125:               # 4 * 2^126 would be no float32
                    e += 1
                scale[r, b] = e + 127
            code[r, 32 * b:32 * b + len(v)] = [number(abs(t) / 2.0 ** e) | (8 if np.signbit(t) else 0) for t in v]
    return code[:, 0::2] | code[:, 1::2] << 4, scale


def unpack(codes, scale, k: int):
    rows, nc = codes.shape
    code = np.stack([codes & 15, codes >> 4], axis=-1).reshape(rows, 2 * nc)[:, :k]
    step = np.where(scale == 255, np.nan, 2.0 ** (scale.astype(np.float64) - 127))
    return np.where(code & 8, -1.0, 1.0) * WORTH[code & 7] * np.repeat(step, 32, axis=1)[:, :k]


def forward(x4, w4, offsets, k: int, bias=None, relu: bool = False):
    """x4 = (codes, scale) of [rows][k], w4 of [blocks n][k] -> (y, magnitude)."""
    x, w = unpack(*x4, k), unpack(*w4, k)
    blocks = len(offsets) - 1
    return G.forward(x, w.reshape(blocks, -1, k), offsets, bias, relu)
