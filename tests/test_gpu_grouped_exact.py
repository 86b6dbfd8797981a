"""Grouped layers on small whole numbers: every result is equal to the oracle's, in long blocks too, where a bound on rounding
would let a row more or less pass.  And every instance of the kernels over small matrices, by the sizes that choose it."""
import numpy as np
import pytest
import torch

import grouped_exact as E
from paper_2503_21364_amd import binding as B

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
DEV = "cuda:0"


def _up(v, dtype="f32"):
    return torch.from_numpy(np.ascontiguousarray(v)).to(DT[dtype]).to(DEV)


class OnGpu:
    def __init__(self, t: E.Numbers, dtype="f32", in_major=False, pad=0):
        self.t, self.dtype, self.in_major = t, dtype, in_major
        wide = lambda v: _up(np.pad(v, ((0, 0), (0, pad)), constant_values=np.nan), dtype)[:, :v.shape[1]]
        x, dy = t.x.copy(), t.dy.copy()
        for v in (x, dy):                       # rows of no block reach nothing
            v[:t.offsets[0]] = np.nan
            v[t.offsets[-1]:] = np.nan
        self.x, self.dy = wide(x), wide(dy)
        self.w = _up(t.w.transpose(0, 2, 1) if in_major else t.w, dtype)
        self.b = _up(t.b)
        self.off = torch.tensor(t.offsets, dtype=torch.int32, device=DEV)
        self.keep = B.Checkpoint8(t.rows, t.k)
        self.keep.codes.fill_(99)
        self.keep.scale.fill_(99)

    def rounded(self, v):
        return torch.from_numpy(v).to(DT[self.dtype]).float().numpy()

    def forward(self, keep=False, bias=True, relu=False):
        t = self.t
        y = torch.full((t.rows, t.n + 1), 7.0, dtype=DT[self.dtype], device=DEV)
        B.grouped_linear(self.x, self.w, self.off, y[:, :t.n], bias=self.b if bias else None, relu=relu, in_major=self.in_major,
                         checkpoint=self.keep if keep else None)
        E.same(y[:, :t.n].float().cpu().numpy(), self.rounded(t.forward(bias, relu)), ("y", keep, bias, relu))
        assert (y[:, t.n] == 7.0).all()
        if keep:
            back = torch.empty((t.rows, t.k), device=DEV)
            B.checkpoint8_unpack(self.keep, back)
            inside = np.zeros_like(t.x)
            inside[t.offsets[0]:t.offsets[-1]] = t.x[t.offsets[0]:t.offsets[-1]]
            E.same(back.cpu().numpy(), inside, "8-bit form")

    def backward(self, codes=False, gate=False, which=("dx", "dw", "db")):
        t = self.t
        dx = torch.full((t.rows, t.k + 1), 7.0, dtype=DT[self.dtype], device=DEV)
        dw, db = torch.full(self.w.shape, 7.0, device=DEV), torch.full((len(t.sizes), t.n), 7.0, device=DEV)
        need = B.grouped_linear_backward_bytes(t.rows, len(t.sizes), t.n, t.k, DT[self.dtype])
        room = torch.full((need + 4096,), 255, dtype=torch.uint8, device=DEV)           # partial sums that nobody wrote are NaN
        out = dict(dx=dx[:, :t.k], dw=dw, db=db)
        B.grouped_linear_backward(self.dy, self.w, self.off, room[:need], x=None if codes else self.x, checkpoint=self.keep if codes else None,
                                  gate=gate, in_major=self.in_major, **{q: out[q] for q in which})
        want = dict(zip(("dx", "dw", "db"), t.backward(gate)))
        for q in which:
            got = out[q].float().cpu().numpy()
            got = got.transpose(0, 2, 1) if q == "dw" and self.in_major else got
            E.same(got, self.rounded(want[q]) if q == "dx" else want[q], (q, codes, gate, which))
        assert (dx[:, t.k] == 7.0).all() and (room[need:] == 255).all()


LONG = [(*s[:3], dtype) for s in E.LONG for dtype in s[3]]


@pytest.mark.parametrize("in_major", [False, True])
@pytest.mark.parametrize("sizes,k,n,dtype", LONG)
def test_long_blocks(sizes, k, n, dtype, in_major):
    g = OnGpu(E.Numbers(sizes, k, n, front=2, behind=3, seed=1), dtype, in_major)
    g.forward()
    g.forward(keep=True, relu=True)
    g.backward()
    g.backward(gate=True)
    g.backward(codes=True, gate=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k,n", [(35, 96), (136, 264), (257, 131), (9, 3)])
@pytest.mark.parametrize("rows", [1, 64, 1500])
def test_many_blocks_of_few_rows(rows, k, n, dtype):
    sizes = np.bincount(np.random.default_rng(rows).integers(0, 70, size=rows), minlength=70).tolist()
    g = OnGpu(E.Numbers(sizes, k, n, front=2, behind=1, seed=rows), dtype)
    g.forward(keep=True)
    g.backward(codes=True)
    g.backward(gate=True)


@pytest.mark.parametrize("in_major", [False, True])
def test_sums_in_large_tiles(in_major):
    """bfloat16 matrices and rows enough for the kernel's large tiles, in several slices."""
    g = OnGpu(E.Numbers([15000, 0, 1003], 2048, 2040, front=2, behind=3, seed=1), "bf16", in_major)
    g.t.dw = g.t.backward()
    g.t.backward = lambda gate: g.t.dw
    g.backward(which=("dw", "db"))
    B.checkpoint8_pack(torch.nan_to_num(g.x), g.keep)
    g.backward(codes=True, which=("dw", "db"))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("which", [("dw",), ("db",), ("dx", "db")])
@pytest.mark.parametrize("k,n", [(35, 96), (40, 72), (131, 257)])
def test_gradients_one_by_one(k, n, which, dtype):
    g = OnGpu(E.Numbers([1300, 0, 77], k, n, front=2, behind=3, seed=4), dtype)
    g.forward(keep=True)
    g.backward(which=which)
    g.backward(codes=True, which=which)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes,k,n", [([3, 0, 17, 1], 24, 16), ([3, 0, 17, 1], 23, 15), ([3, 0, 17, 1] * 20, 256, 32), ([3, 0, 17, 1] * 20, 257, 31)])
def test_few_rows(sizes, k, n, dtype):
    """16 and 64 columns a workgroup, whole runs of values and not, every gate."""
    for in_major in (False, True):
        for k_, n_ in ((k, n), (n, k)):
            g = OnGpu(E.Numbers(sizes, k_, n_, front=2, behind=3, seed=k), dtype, in_major)
            g.forward()
            g.forward(keep=True, relu=True)
            g.backward(which=("dx",))
            g.backward(gate=True, which=("dx",))
            g.backward(codes=True, gate=True, which=("dx",))


# ---- small matrices in float32.  790 rows in 4 blocks are more than few: 790 / 64 rows > 4 + 8 blocks.
SMALL = [500, 0, 290, 41]


@pytest.mark.parametrize("sums", [4, 35, 57, 100])                       # turns of a tile of the rows
@pytest.mark.parametrize("cols", [5, 31, 35, 64, 70, 96, 104, 120])      # tiles of 16 results: 1 .. 6 and 8
def test_products_of_small_matrices(cols, sums):
    for in_major in (False, True):
        g = OnGpu(E.Numbers(SMALL, sums, cols, front=2, behind=67, seed=cols), "f32", in_major, pad=in_major * 3)
        g.forward()
        g.forward(bias=False, relu=True)
        g.forward(keep=True)
        g = OnGpu(E.Numbers(SMALL, cols, sums, front=2, behind=67, seed=sums), "f32", in_major, pad=in_major * 3)
        g.backward(which=("dx",))
        g.backward(gate=True, which=("dx",))
        g.forward(keep=True)
        g.backward(codes=True, gate=True, which=("dx",))


@pytest.mark.parametrize("k", [5, 16, 24, 48, 50, 64])                   # 1 .. 4 tiles of 16 inputs
@pytest.mark.parametrize("n", [4, 10, 32, 40, 64, 70, 81, 96])           # 2, 4, 5 and 6 tiles of outputs
def test_gradients_of_small_matrices(n, k):
    for in_major in (False, True):
        g = OnGpu(E.Numbers(SMALL, k, n, front=2, behind=67, seed=n), "f32", in_major, pad=in_major * 3)
        g.backward()
        g.backward(gate=True)
        g.forward(keep=True)
        g.backward(codes=True)
        g.backward(codes=True, gate=True, which=("dx", "dw"))
