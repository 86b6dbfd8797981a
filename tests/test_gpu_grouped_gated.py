"""Gated layers of blocks and their gradients against the 64-bit oracle, element by element, within the oracle's bounds of 32-bit
arithmetic; results in bfloat16 are rounded once more, 2^-8 of their value."""
import numpy as np
import pytest
import torch

from oracle import gated_ref as G
from oracle.grouped_ref import blocks_of
from paper_2503_21364_amd import binding as B

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
DEV = "cuda:0"


def _np(t):
    return t.detach().double().cpu().numpy()


def _close(got, want, bound, dtype, what):
    got, tol = _np(got), bound * 1.0001 + (2.0 ** -8 * (np.abs(want) + bound) if dtype == "bf16" else 0.0) + 1e-36
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want), err_msg=what)
    with np.errstate(invalid="ignore"):
        bad = ~np.isnan(want) & ~(np.abs(got - want) <= tol)
    assert not bad.any(), (what, int(bad.sum()), got[bad][:4], want[bad][:4], tol[bad][:4], np.argwhere(bad)[:4].tolist())


class Layer:
    """Random layer; `pad` columns behind every row of x, dy and the results, and the rows of no block, hold NaN (results: 7)."""

    def __init__(self, sizes, k, n, dtype="f32", in_major=False, pad=0, front=0, behind=0, seed=0, act="silu", bias=True, wpad=0):
        g = torch.Generator().manual_seed(seed)
        self.sizes, self.k, self.n, self.dtype, self.in_major, self.act, self.pad = sizes, k, n, dtype, in_major, act, pad
        self.offsets = [front] + [front + int(v) for v in np.cumsum(sizes)]
        self.rows = self.offsets[-1] + behind
        blocks, dt = len(sizes), DT[dtype]

        def rows_of(width):
            t = torch.randn(self.rows, width + pad, generator=g).to(dt)
            t[:, width:] = float("nan")
            t[:front] = float("nan")
            t[self.offsets[-1]:] = float("nan")
            return t.to(DEV)[:, :width]

        self.x, self.dy = rows_of(k), rows_of(n)
        w = (torch.randn(blocks, 2 * n, k, generator=g) / k ** 0.5).to(dt)
        self.w64 = w.double().numpy()
        w = (w.transpose(1, 2) if in_major else w).contiguous()
        if wpad:                            # rows of the matrices further apart than they are long
            wide = torch.full((*w.shape[:2], w.shape[2] + wpad), float("nan"), dtype=dt)
            wide[..., :w.shape[2]] = w
            self.w = wide.to(DEV)[..., :w.shape[2]]
        else:
            self.w = w.to(DEV)
        self.b = torch.randn(blocks, 2 * n, generator=g).to(DEV) if bias else None
        self.off = torch.tensor(self.offsets, dtype=torch.int32, device=DEV)
        new = lambda width: torch.full((self.rows, width + pad), 7.0, dtype=dt, device=DEV)[:, :width]
        self.y, self.dx = new(n), new(k)
        self.dw = torch.full(w.shape, 7.0, dtype=dt, device=DEV)
        self.db = torch.full((blocks, 2 * n), 7.0, device=DEV)
        need = B.grouped_gated_backward_bytes(self.rows, blocks, n, k, dt)
        self.ws = torch.full((need + 256,), 255, dtype=torch.uint8, device=DEV)

    def forward(self, stream=None):
        B.grouped_gated(self.x, self.w, self.off, self.y, bias=self.b, act=self.act, in_major=self.in_major, stream=stream)

    def between(self, t, width):
        if self.pad and self.rows:
            assert (t.as_strided((self.rows, self.pad), t.stride(), width) == 7.0).all()

    def check_forward(self):
        _close(self.y, *G.forward(_np(self.x), self.w64, self.offsets, None if self.b is None else _np(self.b), self.act), self.dtype, "y")
        self.between(self.y, self.n)

    def backward(self, which=("dx", "dw", "db"), stream=None):
        B.grouped_gated_backward(self.dy, self.x, self.w, self.off, self.ws[:-256], bias=self.b, act=self.act, in_major=self.in_major, stream=stream,
                                 **{q: getattr(self, q) for q in which})

    def check_backward(self, which=("dx", "dw", "db")):
        want, bound = G.backward(_np(self.dy), _np(self.x), self.w64, self.offsets, None if self.b is None else _np(self.b), self.act, self.dtype == "bf16")
        for i, q in enumerate(("dx", "dw", "db")):
            got = getattr(self, q)
            if q not in which:
                assert (got == 7.0).all(), q
                continue
            got = got.transpose(1, 2) if q == "dw" and self.in_major else got
            _close(got, want[i], bound[i], "f32" if q == "db" else self.dtype, q)
        self.between(self.dx, self.k)
        assert (self.ws[-256:] == self.ws[-1]).all() and int(self.ws[-1]) in (1, 255)


# sizes of the blocks, inputs, outputs: single values, tiles that are just full or just not, every kernel in both its alignments, the anchor
# decoder's layers, many blocks of few rows, blocks without rows
SHAPES = [
    ([1], 1, 1), ([1], 35, 32), ([0, 1, 0], 32, 70), ([3, 0, 0, 5, 1], 7, 5), ([127, 128, 129], 31, 33), ([300], 64, 64), ([40, 0, 217, 64], 35, 32),
    ([500, 1, 2], 32, 70), ([255, 256, 257], 128, 128), ([700, 20], 131, 257), ([90, 300], 256, 192), ([16] * 70, 96, 40), ([2049, 511], 64, 320),
    ([33], 1000, 24), ([1, 1, 1, 1], 512, 512), ([900, 0, 130], 512, 264), ([1300, 1], 8, 1024), ([600], 1032, 136), ([5000], 9, 9), ([4200, 300], 72, 8),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("in_major", [False, True])
@pytest.mark.parametrize("sizes,k,n", SHAPES)
def test_forward(sizes, k, n, in_major, dtype):
    for act, bias in (("silu", True), ("gelu", False), ("relu", True)):
        t = Layer(sizes, k, n, dtype, in_major, seed=k + n, act=act, bias=bias)
        t.forward()
        t.check_forward()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("in_major", [False, True])
@pytest.mark.parametrize("sizes,k,n", SHAPES)
def test_backward(sizes, k, n, in_major, dtype):
    for act, bias in (("silu", True), ("gelu", False), ("relu", True)):
        t = Layer(sizes, k, n, dtype, in_major, seed=k + n + 1, act=act, bias=bias)
        t.backward()
        t.check_backward()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("in_major", [False, True])
@pytest.mark.parametrize("k,n", [(35, 32), (136, 200), (512, 256)])
def test_strides_rows_of_no_block_and_gradients_left_out(k, n, in_major, dtype):
    for pad in (8, 5):
        t = Layer([60, 0, 700, 1], k, n, dtype, in_major, pad=pad, front=5, behind=70, seed=pad, wpad=pad)
        t.forward()
        t.check_forward()
        for which in (("dx", "dw", "db"), ("dx",), ("dw",), ("db",), ("dw", "db")):
            for q in ("dx", "dw", "db"):
                getattr(t, q).fill_(7.0)
            t.ws.fill_(255)
            t.backward(which)
            t.check_backward(which)


@pytest.mark.parametrize("in_major", [False, True])
@pytest.mark.parametrize("sizes,k,n", [([6000, 0, 2500, 30], 256, 512), ([20_011, 0, 64], 72, 640), ([3000] * 8, 128, 256)])
def test_large_tiles(sizes, k, n, in_major):
    # enough rows for the 256 x 256 tiles of the bfloat16 kernel; the bias' sums are joined from many sets
    t = Layer(sizes, k, n, "bf16", in_major, front=3, behind=2, seed=1)
    t.forward()
    t.check_forward()
    t.backward()
    t.check_backward()
    first = [getattr(t, q).clone() for q in ("dx", "dw", "db")]
    t.ws.fill_(1)
    t.backward()
    assert all(torch.equal(a.nan_to_num(), getattr(t, q).nan_to_num()) for a, q in zip(first, ("dx", "dw", "db")))      # the same bits


# the one kernel that takes all gradients of small matrices, in all its shapes
@pytest.mark.parametrize("in_major", [False, True])
@pytest.mark.parametrize("k,n", [(4, 4), (5, 6), (16, 16), (35, 32), (33, 15), (48, 33), (64, 48), (63, 47), (20, 48), (64, 7), (65, 33), (40, 49), (100, 60)])
def test_many_rows_of_small_matrices(k, n, in_major):
    for act, pad in (("silu", 0), ("gelu", 3)):
        t = Layer([5011, 0, 64, 20_000, 1], k, n, "f32", in_major, pad=pad, front=2, behind=3, seed=2, act=act)
        t.forward()
        t.check_forward()
        t.backward()
        t.check_backward()
        for which in (("dx",), ("dw",), ("db",)):
            for q in ("dx", "dw", "db"):
                getattr(t, q).fill_(7.0)
            t.backward(which)
            t.check_backward(which)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k,n", [(16, 16), (64, 96), (256, 256)])
def test_whole_numbers_through_a_relu_are_exact(k, n, dtype):
    # x, w, dy of -2 .. 2: every sum, and every product of two sums, is a whole number that float32 holds; one row left out would show
    rng = np.random.default_rng(3)
    sizes = [1000, 0, 33, 1]
    t = Layer(sizes, k, n, dtype, seed=4, act="relu", bias=False)
    draw = lambda *shape: torch.from_numpy(rng.integers(-1, 2, size=shape).astype(np.float32)).to(DT[dtype])
    t.x.copy_(draw(*t.x.shape))
    t.dy.copy_(draw(*t.dy.shape))
    w = draw(*t.w.shape)
    w[:, n:] = 0                            # u: 1 or -1 alone, of one input, so that a product of gradients stays a whole number
    w[:, n:, 0] = 1
    t.x[:, 0] = torch.where(t.x[:, 0] == 0, torch.ones_like(t.x[:, 0]), t.x[:, 0])
    t.w.copy_(w)
    t.forward()
    t.backward()
    x, dy, w64 = _np(t.x), _np(t.dy), w.double().numpy()
    for g, (a, b) in enumerate(blocks_of(t.offsets, t.rows)):
        p, u = x[a:b] @ w64[g, :n].T, x[a:b] @ w64[g, n:].T
        f = np.maximum(p, 0)
        exact = lambda v: torch.from_numpy(v).to(DT[dtype]).double().numpy()
        assert np.array_equal(_np(t.y[a:b]), exact(f * u))
        d = np.concatenate([dy[a:b] * u * (p > 0), dy[a:b] * f], axis=1)
        if dtype == "bf16":
            assert np.abs(d).max(initial=0) <= 256          # held by bfloat16
        assert np.array_equal(_np(t.dx[a:b]), exact(d @ w64[g]))
        assert np.array_equal(_np(t.dw[g]), exact(d.T @ x[a:b]))
        assert np.array_equal(_np(t.db[g]), d.sum(0))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
def test_far_arguments_of_the_activation(act, dtype):
    # a from -200 to 200 by way of the bias; u = 1
    n, values = 64, torch.tensor(np.linspace(-200, 200, 64), dtype=torch.float32)
    t = Layer([3, 40], 16, n, dtype, act=act, seed=5)
    t.w.zero_()
    t.w64[:] = 0
    t.b[:, :n] = values.to(DEV)
    t.b[:, n:] = 1.0
    t.forward()
    t.check_forward()
    t.backward()
    t.check_backward()
    assert torch.isfinite(t.y).all() and torch.isfinite(t.db).all()


@pytest.mark.parametrize("dtype,k,n", [("f32", 35, 32), ("bf16", 128, 128), ("bf16", 131, 77)])
def test_rows_that_are_not_finite_touch_no_other(dtype, k, n):
    t = Layer([400, 300], k, n, dtype, seed=6)
    clean = Layer([400, 300], k, n, dtype, seed=6)
    t.x[7] = float("nan")
    t.x[650, 3] = float("inf")
    for q in (t, clean):
        q.forward()
        q.backward()
    keep = torch.ones(t.rows, dtype=torch.bool, device=DEV)
    keep[7] = keep[650] = False
    assert torch.isnan(t.y[7]).all() and torch.equal(t.y[keep], clean.y[keep])
    assert torch.isnan(t.dx[7]).all() and torch.equal(t.dx[keep], clean.dx[keep])
    assert torch.isnan(t.dw[0]).all() and torch.isnan(t.db[0]).all()


def test_gradient_is_that_of_differences():
    rng = np.random.default_rng(7)
    for act in ("silu", "gelu"):
        t = Layer([6, 0, 11], 20, 12, seed=8, act=act)
        t.backward()
        x, dy, b = (_np(v) for v in (t.x, t.dy, t.b))
        loss = lambda x_, w_, b_: (G.forward(x_, w_, t.offsets, b_, act)[0] * dy).sum()
        ex, ew, eb, h = rng.normal(size=x.shape), rng.normal(size=t.w64.shape), rng.normal(size=b.shape), 1e-5
        for f, got in ((lambda q: loss(x + q * ex, t.w64, b), (_np(t.dx) * ex).sum()), (lambda q: loss(x, t.w64 + q * ew, b), (_np(t.dw) * ew).sum()),
                       (lambda q: loss(x, t.w64, b + q * eb), (_np(t.db) * eb).sum())):
            assert abs((f(h) - f(-h)) / (2 * h) - got) < 1e-3


def test_offsets_that_go_beyond_the_rows_count_as_the_rows():
    t = Layer([10, 200], 64, 32, "bf16", seed=9)
    t.off = torch.tensor([0, 10, 999], dtype=torch.int32, device=DEV)
    t.forward()
    t.check_forward()
    t.backward()
    t.check_backward()


@pytest.mark.parametrize("dtype,k,n,sizes", [("f32", 35, 32, [5000, 300]), ("bf16", 256, 256, [700, 0, 333]), ("bf16", 96, 40, [1, 2])])
def test_on_a_stream_and_in_a_graph(dtype, k, n, sizes):
    t = Layer(sizes, k, n, dtype, seed=10)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    t.forward(stream=side)
    t.backward(stream=side)
    side.synchronize()
    t.check_forward()
    t.check_backward()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        t.forward()
        t.backward()
    for seed in (1, 2, 3):
        g = torch.Generator().manual_seed(seed)
        t.x.copy_(torch.randn(t.x.shape, generator=g))
        t.dy.copy_(torch.randn(t.dy.shape, generator=g))
        for q in (t.y, t.dx, t.dw, t.db):
            q.fill_(7.0)
        t.ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        t.check_forward()
        t.check_backward()


# ---- few rows: all gradients from those of both projections in 32 bits
FEW = [([1], 1, 1), ([2], 3, 1), ([1], 2, 2), ([3, 0, 1], 3, 2), ([2, 1], 4, 2), ([0, 1, 0], 5, 2), ([1], 1, 300), ([1, 2], 300, 1), ([5, 0, 9, 16, 17], 65, 33),
       ([1, 1], 259, 131), ([64], 66, 34), ([3] * 20, 129, 63), ([0] * 5 + [33], 600, 72), ([1] * 70, 12, 7), ([7, 12], 1030, 513), ([4] * 60, 257, 130),
       ([0, 0, 300] + [0] * 30, 70, 66)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("in_major", [False, True])
@pytest.mark.parametrize("sizes,k,n", FEW)
def test_few_rows(sizes, k, n, in_major, dtype):
    for pad, front, act in ((0, 0, "silu"), (3, 2, "gelu")):
        t = Layer(sizes, k, n, dtype, in_major, pad=pad, front=front, behind=front, seed=k, act=act, wpad=pad)
        t.forward()
        t.check_forward()
        t.backward()
        t.check_backward()
        first = [getattr(t, q).clone() for q in ("dx", "dw", "db")]
        for which in (("dx",), ("dw",), ("db",), ("dx", "db"), ("dw", "db")):
            for q in ("dx", "dw", "db"):
                getattr(t, q).fill_(7.0)
            t.ws.fill_(255)
            t.backward(which)
            t.check_backward(which)
            for q, was in zip(("dx", "dw", "db"), first):
                assert q not in which or torch.equal(getattr(t, q).nan_to_num(), was.nan_to_num())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("in_major", [False, True])
def test_few_rows_that_are_not_finite_touch_no_other_and_no_other_block(in_major, dtype):
    # widths that end inside the vectors: what is read twice, or behind the sums, must not be multiplied by what is not finite
    t, clean = (Layer([5, 7, 0, 2], 67, 37, dtype, in_major, seed=6) for _ in range(2))
    t.x[2] = float("nan")
    t.dy[7, 36] = float("inf")
    for q in (t, clean):
        q.backward()
    keep = torch.ones(t.rows, dtype=torch.bool, device=DEV)
    keep[2] = keep[7] = False
    assert torch.isnan(t.dx[2]).all() and not torch.isfinite(t.dx[7]).any() and torch.equal(t.dx[keep], clean.dx[keep])
    assert torch.isnan(t.dw[0]).all() and torch.isnan(t.db[0]).all()
    assert torch.equal(t.dw[2:], clean.dw[2:]) and torch.equal(t.db[2:], clean.db[2:])
    dw, own = (q.dw[1].transpose(0, 1) if in_major else q.dw[1] for q in (t, clean))
    touched = [36, 37 + 36]
    rest = [o for o in range(2 * 37) if o not in touched]
    assert torch.equal(dw[rest], own[rest]) and not torch.isfinite(dw[touched]).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_few_rows_in_a_graph(dtype):
    t = Layer([3, 0, 9, 1], 130, 70, dtype, seed=12)
    t.backward()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        t.backward()
    for i in range(3):
        t.x.copy_(torch.randn(t.x.shape, generator=torch.Generator().manual_seed(i)))
        for q in ("dx", "dw", "db", "ws"):
            getattr(t, q).fill_(7 if q != "ws" else 1)
        graph.replay()
        torch.cuda.synchronize()
        t.check_backward()


# rows, inputs and outputs of every kernel's own: few rows, small float32 matrices (both directions), the general one, bfloat16 tiles
@pytest.mark.parametrize("dtype,rows,k,n", [("f32", 40, 16, 64), ("f32", 5000, 16, 48), ("f32", 5000, 16, 64), ("f32", 5000, 80, 80), ("bf16", 40, 16, 64),
                                            ("bf16", 3000, 16, 64), ("bf16", 5000, 4, 64)])
def test_gelu_keeps_its_digits_far_below_zero(dtype, rows, k, n):
    # a from -0.4 to -12.8 by way of the bias, u = 1, both exact; the normal distribution goes down to 1e-37 there.  It and its density are off by 12
    # roundings, a product with a, u or dy by one more each; a result in bfloat16 is rounded once more
    t = Layer([rows], k, n, dtype, act="gelu", seed=21)
    t.w.zero_()
    t.dy.zero_()
    t.dy[0] = 1.0                               # the bias' gradients are those of one row
    t.b[0, :n] = -torch.linspace(0.4, 12.8, n).to(DEV)
    t.b[0, n:] = 1.0
    t.forward()
    t.backward()
    a, u24 = _np(t.b[0, :n]), 2.0 ** -24
    p, d = G.normal(a), np.exp(-a * a / 2) / np.sqrt(2 * np.pi)
    assert p.min() > 2.0 ** -125
    y = _np(t.y)
    assert (y == y[0]).all()
    assert (np.abs(y[0] - a * p) <= np.abs(a * p) * (14 * u24 + (2.0 ** -8 if dtype == "bf16" else 0))).all()
    db = _np(t.db[0])
    assert (np.abs(db[n:] - a * p) <= np.abs(a * p) * 14 * u24).all()
    assert (np.abs(db[:n] - (p + a * d)) <= (p + np.abs(a) * d) * 15 * u24).all()


# rows that end inside a vector, before the first one does, and in its last value; outputs likewise, by tiles of 16 and of 32; NaN behind every row
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("in_major", [False, True])
@pytest.mark.parametrize("sizes", [[1], [3, 0, 17], [2] * 170])
def test_few_rows_however_their_vectors_end(sizes, in_major, dtype):
    for k, n in ((1, 1), (2, 3), (3, 65), (5, 33), (7, 70), (9, 2), (15, 69), (17, 66), (31, 35), (47, 34), (49, 33), (66, 1), (127, 18), (130, 97), (515, 67)):
        t = Layer(sizes, k, n, dtype, in_major, pad=3, front=1, behind=2, seed=k + n, wpad=5)
        t.forward()
        t.check_forward()
        t.backward()
        t.check_backward()
