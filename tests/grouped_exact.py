"""Grouped layers on small whole numbers, where every order of 32-bit sums gives the same: results are compared for equality, so that a row
left out, taken twice or summed for another block shows, however many rows a block has.

x, dy, w and the bias are -2, -1, 1 or 2: a partial sum is a whole number below 4 m <= 2^24 in magnitude, which float32 holds, and one row
changes every element of its block's dw and db.  The 8-bit form of x is exact as well.  Results in bfloat16 are the sum, rounded once."""
import numpy as np

from oracle import grouped_ref as G

VALUES = np.array([-2.0, -1.0, 1.0, 2.0], np.float32)

# blocks' rows, inputs, outputs, types.  Long blocks beside short ones and empty ones: many sets of partial sums a block, joined in one part
# and in eight; slices that begin and end anywhere in the blocks; one run a block; matrices of whole tiles and not.
LONG = [
    ([30011, 0, 64, 65], 35, 96, ("f32",)), ([30011, 0, 64, 65], 32, 70, ("f32",)), ([30011, 0, 64, 65], 8, 8, ("f32", "bf16")),
    ([30011, 0, 64, 65], 64, 33, ("f32",)), ([0, 20011, 0, 3], 35, 96, ("f32", "bf16")), ([0, 20011, 0, 3], 128, 256, ("f32", "bf16")),
    ([29000, 0, 1003], 488, 504, ("f32", "bf16")), ([70001], 32, 32, ("f32",)), ([3, 40000, 257], 131, 257, ("bf16",)),
    ([9000, 1, 0, 7000], 5, 3, ("f32", "bf16")), ([64] * 40 + [2500], 64, 96, ("f32",)), ([1400, 100], 1024, 1032, ("f32", "bf16")),
]


class Numbers:
    """x, dy [rows][..], w [blocks][n][k], b [blocks][n]; `front` rows before the first block and `behind` after the last one are of no block."""

    def __init__(self, sizes, k, n, front=0, behind=0, seed=0):
        rng = np.random.default_rng(seed)
        self.sizes, self.k, self.n = sizes, k, n
        self.offsets = [front] + [front + int(s) for s in np.cumsum(sizes)]
        self.rows = self.offsets[-1] + behind
        draw = lambda *shape: VALUES[rng.integers(0, 4, size=shape)]
        self.x, self.dy = draw(self.rows, k), draw(self.rows, n)
        self.w, self.b = draw(len(sizes), n, k), draw(len(sizes), n)

    def forward(self, bias=True, relu=False):
        """y; sums of whole numbers below 2^24 are exact in float32 too."""
        y = np.zeros((self.rows, self.n), np.float32)
        for g, (a, b) in enumerate(G.blocks_of(self.offsets, self.rows)):
            y[a:b] = self.x[a:b] @ self.w[g].T + (self.b[g] if bias else 0)
        return np.maximum(y, 0) if relu else y

    def backward(self, gate=False, without=None):
        """dx, dw, db.  without: a row that the sums over rows leave out, the mistake that the comparison has to show."""
        dx, dw, db = np.zeros_like(self.x), np.zeros_like(self.w), np.zeros_like(self.b)
        for g, (a, b) in enumerate(G.blocks_of(self.offsets, self.rows)):
            dx[a:b] = self.dy[a:b] @ self.w[g]
            rows = [r for r in range(a, b) if r != without] if without is not None and a <= without < b else slice(a, b)
            dw[g], db[g] = self.dy[rows].T @ self.x[rows], self.dy[rows].sum(0)
        return np.where(self.x > 0, dx, np.float32(0)) if gate else dx, dw, db


def same(got, want, what):
    """Equality, of bits but for the sign of a zero."""
    bad = ~(got == want)
    assert not bad.any(), (what, int(bad.sum()), bad.size, got[bad][:4], want[bad][:4], np.argwhere(bad)[:4].tolist())
