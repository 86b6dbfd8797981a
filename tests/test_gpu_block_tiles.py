"""Gated layers and layers in 4 bits where a workgroup takes several tiles one after the other: the next one's loads and bias in front of this
one's results, whole and ragged tiles and rows of no block in turns, results through the caches and past them.  Inputs are small whole numbers,
so that every sum is exact and every element of every row is compared for equality, with products in 64 bits on the device; the activations
that are no whole numbers within the oracle's bounds."""
import numpy as np
import pytest
import torch

from oracle import gated_ref as G
from paper_2503_21364_amd import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
DEV = "cuda:0"
AT_ONCE = {256: 256, 128: 512}          # workgroups that run at once, by the rows of a tile


def _whole(shape, seed, most=2):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randint(-most, most + 1, shape, generator=g, device=DEV, dtype=torch.int32).float()


def _offsets(sizes, front):
    off = [front] + [front + int(v) for v in np.cumsum(sizes)]
    return off, torch.tensor(off, dtype=torch.int32, device=DEV)


def _tiles(sizes, front, behind, n, rows_of_tile, cols_of_tile):
    return sum((m + rows_of_tile - 1) // rows_of_tile for m in [front, *sizes, behind]) * ((n + cols_of_tile - 1) // cols_of_tile)


def _rounded(v, dtype):
    return v.to(DT[dtype]).double()         # of whole numbers below 2^24: through float32 or not is the same


def _blocks(off):
    return [(g, a, b) for g, (a, b) in enumerate(zip(off, off[1:])) if b > a]


# sizes of the blocks, rows in front of the first and behind the last, outputs, side of a tile
FOUR_BITS = [([30_000, 0, 129, 45_000, 77], 5000, 4000, 128, 128), ([70_001], 0, 0, 100, 128), ([140_000, 2000], 300, 0, 128, 128),
             ([33_000, 0, 25_600, 300], 4100, 1000, 512, 256), ([60_007], 0, 600, 450, 256), ([20_480] * 3, 0, 0, 512, 256)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k", [100, 256, 1024, 1100])
@pytest.mark.parametrize("sizes,front,behind,n,side", FOUR_BITS)
def test_layers_in_4_bits_tile_after_tile(sizes, front, behind, n, side, k, dtype):
    assert _tiles(sizes, front, behind, n, side, side) > AT_ONCE[side]
    off, offsets = _offsets(sizes, front)
    rows, blocks = off[-1] + behind, len(sizes)
    x, w, bias = _whole((rows, k), 1), _whole((blocks * n, k), 2), _whole((blocks, n), 3, 9)
    x4, w4 = B.Block4(rows, k), B.Block4(blocks * n, k)
    B.block4_pack(x, x4)
    B.block4_pack(w, w4)
    want = torch.zeros((rows, n), dtype=torch.float64, device=DEV)
    for g, a, b in _blocks(off):
        want[a:b] = x[a:b].double() @ w[g * n:(g + 1) * n].double().t().contiguous() + bias[g].double()
    del x
    for pad, relu in ((0, False), (8, True)):           # rows of whole lines where n allows, and not
        y = torch.full((rows, n + pad), 7.0, dtype=DT[dtype], device=DEV)
        for _ in range(2):
            B.grouped_linear4(x4, w4, offsets, y[:, :n], bias=bias, relu=relu)
        right = _rounded(want.clamp(min=0) if relu else want, dtype)
        assert torch.equal(y[:, :n].double(), right), (pad, (y[:, :n].double() != right).nonzero()[:4].tolist())
        assert (y[:, n:] == 7.0).all()


# the same, inputs, pad behind the rows of every operand (odd: none of them starts at a vector)
GATED = [([20_000, 0, 300, 20_480], 3000, 700, 512, 512, 0, 256), ([41_003], 0, 0, 512, 96, 0, 256), ([16_640, 25_600], 300, 0, 384, 520, 8, 256),
         ([100_000, 0, 200_000], 2000, 4000, 64, 32, 0, 128), ([76_000, 800], 130, 0, 64, 64, 0, 128), ([70_000, 5000, 33], 0, 999, 56, 264, 8, 128),
         ([40_000, 0, 129, 3000], 700, 300, 200, 77, 0, 128), ([36_000, 7000], 0, 0, 128, 128, 5, 128)]


class Gated:
    def __init__(self, sizes, front, behind, n, k, pad, in_major, seed):
        self.off, self.offsets = _offsets(sizes, front)
        self.rows, self.blocks, self.n, self.k, self.pad, self.in_major = self.off[-1] + behind, len(sizes), n, k, pad, in_major
        bf = torch.bfloat16
        self.x = self.wide(_whole((self.rows, k), seed, 1))
        self.w64 = _whole((self.blocks, 2 * n, k), seed + 1, 1).double()
        self.b = _whole((self.blocks, 2 * n), seed + 2, 3)
        self.y = torch.full((self.rows, n + pad), 7.0, dtype=bf, device=DEV)[:, :n]

    def wide(self, v):
        """In bfloat16, `pad` NaN behind every row."""
        t = torch.full((*v.shape[:-1], v.shape[-1] + self.pad), float("nan"), dtype=torch.bfloat16, device=DEV)
        t[..., :v.shape[-1]] = v.to(torch.bfloat16)
        return t[..., :v.shape[-1]]

    def weights(self):
        return self.wide((self.w64.transpose(1, 2) if self.in_major else self.w64).float())

    def projections(self, g, a, b):
        x, w = self.x[a:b].double(), self.w64[g]
        both = x @ w.t().contiguous() + self.b[g].double()
        return both[:, :self.n], both[:, self.n:]


@pytest.mark.parametrize("in_major", [False, True])
@pytest.mark.parametrize("sizes,front,behind,n,k,pad,side", GATED)
def test_gated_layers_tile_after_tile(sizes, front, behind, n, k, pad, side, in_major):
    assert _tiles(sizes, front, behind, n, side, side // 2) > AT_ONCE[side]
    t = Gated(sizes, front, behind, n, k, pad, in_major, 4)
    w = t.weights()
    for act in ("relu", "silu", "gelu"):
        for _ in range(2):
            B.grouped_gated(t.x, w, t.offsets, t.y, bias=t.b, act=act, in_major=in_major)
        got = t.y.double()
        assert (got[:front] == 0).all() and (got[t.off[-1]:] == 0).all()
        for g, a, b in _blocks(t.off):
            p, u = t.projections(g, a, b)
            if act == "relu":
                right = _rounded(p.clamp(min=0) * u, "bf16")
                assert torch.equal(got[a:b], right), (act, g, (got[a:b] != right).nonzero()[:4].tolist())
                continue
            # a and u are exact: the activation's own deviation, one product, one rounding; what the activation multiplies a with is held as 0
            # where it is below 2^-126 (a of -22: 1e-107), which a u 2^-126 is at least as much as
            f, off = _activation(p, act)
            right = f * u
            assert ((got[a:b] - right).abs() <= off * u.abs() + (2 * U + 2.0 ** -8) * right.abs() + 2.0 ** -126 * (p * u).abs()).all(), (act, g)
        if pad:
            assert (t.y.as_strided((t.rows, pad), t.y.stride(), n) == 7.0).all()


def _activation(a, act):
    """Value and what 32 bits may be off by, from the oracle at whole numbers."""
    low, high = int(a.min()), int(a.max())
    f, _, off, _ = G.activation(np.arange(low, high + 1, dtype=np.float64), act)
    at = (a - low).long()
    return torch.from_numpy(f).to(DEV)[at], torch.from_numpy(off).to(DEV)[at]


@pytest.mark.parametrize("in_major", [False, True])
@pytest.mark.parametrize("sizes,front,behind,n,k,pad,side", GATED)
def test_gradients_of_gated_layers_tile_after_tile(sizes, front, behind, n, k, pad, side, in_major):
    # u is 1 or -1, of one input, and 0 or 2 of its bias; a gradient of both projections is a whole number that bfloat16 holds
    t = Gated(sizes, front, behind, n, k, pad, in_major, 5)
    t.x[:, 0] = torch.where(t.x[:, 0] == 0, torch.ones_like(t.x[:, 0]), t.x[:, 0])
    t.w64[:, n:] = 0
    t.w64[:, n:, 0] = 1
    t.b[:, n:] = torch.where(t.b[:, n:] > 0, 2.0, 0.0)
    w = t.weights()
    dy = t.wide(_whole((t.rows, n), 6, 1))
    dx = torch.full((t.rows, k + pad), 7.0, dtype=torch.bfloat16, device=DEV)[:, :k]
    dw, db = torch.full((t.blocks, k, 2 * n) if in_major else (t.blocks, 2 * n, k), 7.0, dtype=torch.bfloat16, device=DEV), torch.full_like(t.b, 7.0)
    ws = torch.full((B.grouped_gated_backward_bytes(t.rows, t.blocks, n, k, torch.bfloat16),), 255, dtype=torch.uint8, device=DEV)
    B.grouped_gated_backward(dy, t.x, w, t.offsets, ws, bias=t.b, act="relu", dx=dx, dw=dw, db=db, in_major=in_major)
    assert (dx[:front] == 0).all() and (dx[t.off[-1]:] == 0).all()
    for g in range(t.blocks):
        a, b = t.off[g], t.off[g + 1]
        p, u = t.projections(g, a, b)
        up, f = dy[a:b].double(), p.clamp(min=0)
        d = torch.cat([up * u * (p > 0), up * f], dim=1)
        assert b == a or d.abs().max() <= 256
        dw64 = d.t().contiguous() @ t.x[a:b].double()
        assert b == a or max(dw64.abs().max(), d.sum(0).abs().max()) < 2 ** 24
        for got, right in ((db[g].double(), d.sum(0)), (dx[a:b].double(), _rounded(d @ t.w64[g], "bf16")),
                           (dw[g].double(), _rounded(dw64.t() if in_major else dw64, "bf16"))):
            assert torch.equal(got, right), (g, (got != right).nonzero()[:4].tolist())
    if pad:
        assert (dx.as_strided((t.rows, pad), dx.stride(), k) == 7.0).all()


@pytest.mark.parametrize("k", [512, 520, 1000])
def test_layers_in_tiles_of_192_rows(k):
    # a size whose tiles of 256 x 256 would leave a last round nearly empty, of 512 sums and more: forward, and the same product as dx
    n, (off, offsets) = 4096, _offsets([2999, 1, 0, 5289], 1)
    rows = off[-1] + 10
    x, w = _whole((rows, k), 7, 1).to(torch.bfloat16), _whole((4, n, k), 8, 1).to(torch.bfloat16)
    b = _whole((4, n), 9, 9)
    y, dx = (torch.full((rows, n), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    B.grouped_linear(x, w, offsets, y, bias=b, relu=True)
    ws = torch.empty(B.grouped_linear_backward_bytes(rows, 4, k, n, torch.bfloat16), dtype=torch.uint8, device=DEV)
    B.grouped_linear_backward(x, w.transpose(1, 2).contiguous(), offsets, ws, dx=dx)
    want, plain = (torch.zeros((rows, n), dtype=torch.float64, device=DEV) for _ in range(2))
    for g, s, e in _blocks(off):
        plain[s:e] = x[s:e].double() @ w[g].double().t().contiguous()
        want[s:e] = (plain[s:e] + b[g].double()).clamp(min=0)
    assert torch.equal(y.double(), _rounded(want, "bf16"))
    assert torch.equal(dx.double(), _rounded(plain, "bf16"))
