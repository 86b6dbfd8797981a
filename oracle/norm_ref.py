"""Oracle of the layer norms of blocks and their gradients: numpy, 64 bits.

Every result comes with a bound of what 32 bits may be off by (u = 2^-24).  No value goes through more than M = 96 additions on its way
into a sum over a row (64 in a lane, 6 over a wavefront, 16 over wavefronts), so with dm = (M + 2) u mean|x| the mean is off by dm at
most; the squares are of x less that mean, whose own offset enters the variance squared only (the true differences add up to nothing),
so 1 / deviation is off by a share rs = (M / 2 + 10) u + (dm s)^2 of itself; the rest are single roundings of single operations."""
from __future__ import annotations

import numpy as np

from oracle.grouped_ref import blocks_of

U = 2.0 ** -24


def _rows(x, eps: float):
    """h, s and the bounds of h (element) and s (share)."""
    k, m = x.shape[1], min(x.shape[1], 96)
    mean = x.mean(1, keepdims=True)
    s = 1.0 / np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + eps)
    h = (x - mean) * s
    dm = (m + 2) * U * np.abs(x).mean(1, keepdims=True)
    rs = (m / 2 + 10) * U + (dm * s) ** 2
    return h, s, s * dm + np.abs(h) * (rs + 2 * U), rs, m


def forward(x, offsets, gain=None, shift=None, eps: float = 1e-5):
    """x [rows][k], gain and shift [blocks][k] -> (y, bound); rows of no block are 0."""
    x = np.asarray(x, np.float64)
    y, bound = np.zeros(x.shape), np.zeros(x.shape)
    with np.errstate(invalid="ignore", over="ignore"):
        for g, (a, b) in enumerate(blocks_of(offsets, x.shape[0])):
            if a == b:
                continue
            h, _, dh, _, _ = _rows(x[a:b], eps)
            w = 1.0 if gain is None else np.asarray(gain[g], np.float64)
            t = 0.0 if shift is None else np.asarray(shift[g], np.float64)
            y[a:b] = w * h + t
            bound[a:b] = np.abs(w) * dh + 2 * U * (np.abs(w * h) + np.abs(t))
    return y, bound


def backward(dy, x, offsets, gain=None, eps: float = 1e-5):
    """-> (dx, dgain, dshift) and their bounds."""
    dy, x = np.asarray(dy, np.float64), np.asarray(x, np.float64)
    blocks, k = len(offsets) - 1, x.shape[1]
    dx, ex = np.zeros(x.shape), np.zeros(x.shape)
    dgain, eg, dshift, es = (np.zeros((blocks, k)) for _ in range(4))
    mean = lambda v: v.mean(1, keepdims=True)
    with np.errstate(invalid="ignore", over="ignore"):
        for g, (a, b) in enumerate(blocks_of(offsets, x.shape[0])):
            if a == b:
                continue
            h, s, dh, rs, m = _rows(x[a:b], eps)
            d = dy[a:b] * (1.0 if gain is None else np.asarray(gain[g], np.float64))
            level, along = mean(d), mean(d * h)
            dx[a:b] = s * (d - level - h * along)
            parts = np.abs(d) + mean(np.abs(d)) + np.abs(h) * mean(np.abs(d * h))
            e_level = (m + 3) * U * mean(np.abs(d))
            e_along = (m + 6 + rs / U) * U * mean(np.abs(d * h)) + mean(np.abs(d) * dh)
            ex[a:b] = s * (e_level + np.abs(h) * e_along + dh * mean(np.abs(d * h)) + (rs + 6 * U) * parts)
            rows = b - a
            dgain[g], dshift[g] = (dy[a:b] * h).sum(0), dy[a:b].sum(0)
            eg[g] = (np.abs(dy[a:b]) * dh).sum(0) + (rows + 2) * U * np.abs(dy[a:b] * h).sum(0)
            es[g] = (rows + 2) * U * np.abs(dy[a:b]).sum(0)
    return (dx, dgain, dshift), (ex, eg, es)
