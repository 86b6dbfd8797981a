"""Oracle of the grouped perceptron layers and their 8-bit checkpoints: numpy, 64 bits, one block after the other.

Every result comes with the sum of the magnitudes it was added up from, which is what an error bound of a
32-bit sum is stated in."""
from __future__ import annotations

import numpy as np


def blocks_of(offsets, rows: int):
    """(begin, end) of every block; offsets above `rows` count as `rows`."""
    edge = [min(int(o), rows) for o in offsets]
    return list(zip(edge, [max(a, b) for a, b in zip(edge, edge[1:])]))


def forward(x, w, offsets, bias=None, relu=False):
    """x [rows][k], w [blocks][n][k] -> (y, magnitude), both [rows][n]; rows of no block are 0."""
    x, w = np.asarray(x, np.float64), np.asarray(w, np.float64)
    y, mag = np.zeros((x.shape[0], w.shape[1])), np.zeros((x.shape[0], w.shape[1]))
    with np.errstate(invalid="ignore", over="ignore"):
        for g, (a, b) in enumerate(blocks_of(offsets, x.shape[0])):
            add = 0.0 if bias is None else np.asarray(bias[g], np.float64)
            y[a:b] = x[a:b] @ w[g].T + add
            mag[a:b] = np.abs(x[a:b]) @ np.abs(w[g].T) + np.abs(add)
        if relu:
            y = np.where(y < 0, 0.0, y)
    return y, mag


def backward(dy, x, w, offsets, gate=False):
    """-> dx, dw, db and their magnitudes."""
    dy, x, w = (np.asarray(v, np.float64) for v in (dy, x, w))
    dx, dw, db = np.zeros(x.shape), np.zeros(w.shape), np.zeros(w.shape[:2])
    mx, mw, mb = np.zeros(x.shape), np.zeros(w.shape), np.zeros(w.shape[:2])
    with np.errstate(invalid="ignore", over="ignore"):
        for g, (a, b) in enumerate(blocks_of(offsets, x.shape[0])):
            dx[a:b], mx[a:b] = dy[a:b] @ w[g], np.abs(dy[a:b]) @ np.abs(w[g])
            dw[g], mw[g] = dy[a:b].T @ x[a:b], np.abs(dy[a:b].T) @ np.abs(x[a:b])
            db[g], mb[g] = dy[a:b].sum(0), np.abs(dy[a:b]).sum(0)
    if gate:
        shut = x <= 0
        dx, mx = np.where(shut, 0.0, dx), np.where(shut, 0.0, mx)
    return (dx, dw, db), (mx, mw, mb)


def pack(x):
    """x [rows][k] float32 -> codes int8 [rows][kp], scale uint8 [rows][kp / 32]."""
    x = np.asarray(x, np.float64)
    rows, k = x.shape
    kp = (k + 31) // 32 * 32
    codes, scale = np.zeros((rows, kp), np.int8), np.zeros((rows, kp // 32), np.uint8)
    for r in range(rows):
        for q in range(kp // 32):
            v = x[r, 32 * q:min(32 * q + 32, k)]
            if not np.isfinite(v).all():
                scale[r, q] = 255
                continue
            top = np.abs(v).max()
            if top == 0:
                continue
            e = -126
            while top / 2.0 ** e >= 127.5 and e < 121:          # 64 * 2^122 would be no float32
                e += 1
            c = np.minimum(np.rint(np.abs(v) / 2.0 ** e), 127)
            c = np.where((c == 0) & (v != 0), 1, c) * np.sign(v)
            scale[r, q] = e + 127
            codes[r, 32 * q:32 * q + len(v)] = c.astype(np.int8)
    return codes, scale


def unpack(codes, scale, k: int):
    step = np.where(scale == 255, np.nan, 2.0 ** (scale.astype(np.float64) - 127))
    return (codes.astype(np.float64) * np.repeat(step, 32, axis=1))[:, :k]
