"""Oracle of the gated layers of blocks and their gradients: numpy, 64 bits, one block after the other.

Every result comes with a bound of what 32 bits may be off by (u = 2^-24):
  a and u, sums of k products: (k + 3) u times the sum of the magnitudes.
  The activation moves by at most 1.13 of what a moves (the steepest slope of the three), its slope by 0.8 of it.
  SiLU: e^-a as a power of two of a rounded product is off by (2 |a| + 2) u of itself, sum, reciprocal and product by 6 u more.
  GELU: the normal distribution and its density are off by 12 u of themselves, each product or sum behind them by one more.
  ReLU: exact, but for the slope of an a that may as well be on the other side of 0.
`half`: the roundings of both projections' gradients to bfloat16, 2^-8 of each, on their way into dx and dw."""
from __future__ import annotations

import numpy as np

from oracle.grouped_ref import blocks_of

U = 2.0 ** -24
STEEP, BENT = 1.13, 0.8


def normal(a):
    """The normal distribution, from the standard library's error function."""
    import math
    return 0.5 * np.vectorize(math.erfc, otypes=[np.float64])(-np.asarray(a, np.float64) / math.sqrt(2.0))


def activation(a, act: str):
    """value, slope, and how far 32 bits of either may be off for the same a."""
    size = np.abs(a)
    if act == "relu":
        return np.where(a < 0, 0.0, a), np.where(a <= 0, 0.0, 1.0), np.zeros_like(a), np.zeros_like(a)
    if act == "silu":
        with np.errstate(over="ignore"):
            p = 1 / (1 + np.exp(-a))
        return a * p, p * (1 + a * (1 - p)), size * p * (2 * size + 8) * U, (10 + 14 * size) * U
    p, d = normal(a), np.exp(-a * a / 2) / np.sqrt(2 * np.pi)
    return a * p, p + a * d, size * p * 13 * U, (p + size * d) * 14 * U


def _projections(x, w, bias, n: int):
    k = x.shape[1]
    out = []
    for h in range(2):
        m = w[h * n:(h + 1) * n]
        b = 0.0 if bias is None else np.asarray(bias[h * n:(h + 1) * n], np.float64)
        out.append((x @ m.T + b, (k + 3) * U * (np.abs(x) @ np.abs(m.T) + np.abs(b))))
    return out


def forward(x, w, offsets, bias=None, act: str = "silu"):
    """x [rows][k], w [blocks][2 n][k] -> (y, bound), both [rows][n]; rows of no block are 0."""
    x, w = np.asarray(x, np.float64), np.asarray(w, np.float64)
    n = w.shape[1] // 2
    y, bound = np.zeros((x.shape[0], n)), np.zeros((x.shape[0], n))
    with np.errstate(invalid="ignore", over="ignore"):
        for g, (b, e) in enumerate(blocks_of(offsets, x.shape[0])):
            if b == e:
                continue
            (a, ea), (u, eu) = _projections(x[b:e], w[g], None if bias is None else bias[g], n)
            f, _, ef, _ = activation(a, act)
            y[b:e] = f * u
            bound[b:e] = np.abs(f) * eu + (np.abs(u) + eu) * (STEEP * ea + ef) + 2 * U * np.abs(f * u)
    return y, bound


def backward(dy, x, w, offsets, bias=None, act: str = "silu", half: bool = False):
    """-> (dx, dw, db) and their bounds."""
    dy, x, w = (np.asarray(v, np.float64) for v in (dy, x, w))
    n = w.shape[1] // 2
    dx, ex, dw, ew = np.zeros(x.shape), np.zeros(x.shape), np.zeros(w.shape), np.zeros(w.shape)
    db, eb = np.zeros(w.shape[:2]), np.zeros(w.shape[:2])
    with np.errstate(invalid="ignore", over="ignore"):
        for g, (b, e) in enumerate(blocks_of(offsets, x.shape[0])):
            if b == e:
                continue
            (a, ea), (u, eu) = _projections(x[b:e], w[g], None if bias is None else bias[g], n)
            f, slope, ef, es = activation(a, act)
            if act == "relu":
                es = np.where(np.abs(a) <= ea, 1.0, 0.0)
                bent = 0.0
            else:
                bent = BENT
            up, size = dy[b:e], np.abs(dy[b:e])
            d = np.concatenate([up * u * slope, up * f], axis=1)
            off = np.concatenate([size * (np.abs(slope) * eu + (np.abs(u) + eu) * (bent * ea + es)), size * (STEEP * ea + ef)], axis=1) + 3 * U * np.abs(d)
            rows = e - b
            db[g], eb[g] = d.sum(0), off.sum(0) + (rows + 2) * U * np.abs(d).sum(0)
            if half:
                off = off + 2.0 ** -8 * (np.abs(d) + off)
            dx[b:e] = d @ w[g]
            ex[b:e] = off @ np.abs(w[g]) + (2 * n + 2) * U * (np.abs(d) @ np.abs(w[g]))
            dw[g] = d.T @ x[b:e]
            ew[g] = off.T @ np.abs(x[b:e]) + (rows + 2) * U * (np.abs(d).T @ np.abs(x[b:e]))
    return (dx, dw, db), (ex, ew, eb)
