"""Layer norms of blocks and their gradients against the 64-bit oracle, element by element, within the oracle's bounds of
32-bit arithmetic; a result in bfloat16 is rounded once more, 2^-8 of its value."""
import numpy as np
import pytest
import torch

from oracle import norm_ref as N
from paper_2503_21364_amd import binding as B

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
DEV = "cuda:0"
U = 2.0 ** -24


def _np(t):
    return t.detach().double().cpu().numpy()


def _close(got, want, bound, dtype, what):
    got, tol = _np(got), bound * 1.0001 + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0.0) + 1e-38
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want), err_msg=what)
    with np.errstate(invalid="ignore"):
        bad = ~np.isnan(want) & ~(np.abs(got - want) <= tol)
    assert not bad.any(), (what, int(bad.sum()), got[bad][:4], want[bad][:4], tol[bad][:4], np.argwhere(bad)[:4].tolist())


class Case:
    """Random rows of the given blocks; `pad` columns behind every row and the rows of no block hold NaN."""

    def __init__(self, sizes, k, dtype="f32", pad=0, front=0, behind=0, seed=0, level=0.5, affine=True):
        g = torch.Generator().manual_seed(seed)
        self.sizes, self.k, self.dtype, self.pad = sizes, k, dtype, pad
        self.offsets = [front] + [front + int(v) for v in np.cumsum(sizes)]
        self.rows = self.offsets[-1] + behind

        def rows_of(scale, shift):
            t = (torch.randn(self.rows, k + pad, generator=g) * scale + shift).to(DT[dtype])
            t[:, k:] = float("nan")
            t[:front] = float("nan")
            t[self.offsets[-1]:] = float("nan")
            return t.to(DEV)[:, :k]

        self.x, self.dy = rows_of(1.5, level), rows_of(1.0, 0.1)
        blocks = len(sizes)
        self.gain = (1 + 0.3 * torch.randn(blocks, k, generator=g)).to(DEV) if affine else None
        self.shift = torch.randn(blocks, k, generator=g).to(DEV) if affine else None
        self.off = torch.tensor(self.offsets, dtype=torch.int32, device=DEV)
        new = lambda: torch.full((self.rows, k + pad), 7.0, dtype=DT[dtype], device=DEV)[:, :k]
        self.y, self.dx = new(), new()
        self.dgain, self.dshift = (torch.full((blocks, k), 7.0, device=DEV) for _ in range(2))
        self.ws = torch.full((B.grouped_norm_backward_bytes(self.rows, blocks, k, DT[dtype]),), 255, dtype=torch.uint8, device=DEV)

    def between(self, t):
        if self.pad and self.rows:
            assert (t.as_strided((self.rows, self.pad), t.stride(), self.k) == 7.0).all()

    def forward(self, eps=1e-5, stream=None):
        B.grouped_norm(self.x, self.off, self.y, gain=self.gain, shift=self.shift, eps=eps, stream=stream)

    def check_forward(self, eps=1e-5):
        opt = lambda t: None if t is None else _np(t)
        _close(self.y, *N.forward(_np(self.x), self.offsets, opt(self.gain), opt(self.shift), eps), self.dtype, "y")
        self.between(self.y)

    def backward(self, eps=1e-5, which=("dx", "dgain", "dshift"), stream=None):
        B.grouped_norm_backward(self.dy, self.x, self.off, self.ws, gain=self.gain, eps=eps, stream=stream, **{q: getattr(self, q) for q in which})

    def check_backward(self, eps=1e-5, which=("dx", "dgain", "dshift"), inputs=None):
        dy, x = inputs or (_np(self.dy), _np(self.x))
        want, bound = N.backward(dy, x, self.offsets, None if self.gain is None else _np(self.gain), eps)
        for i, q in enumerate(("dx", "dgain", "dshift")):
            if q in which:
                _close(getattr(self, q), want[i], bound[i], self.dtype if q == "dx" else "f32", q)
        self.between(self.dx)


# values of a row: one, a lane's vector and its neighbours, every arrangement of a row over lanes and its ends, rows longer than registers
WIDTHS = [1, 2, 7, 8, 9, 31, 33, 35, 64, 65, 96, 100, 128, 131, 255, 257, 512, 513, 1000, 1024, 1025, 2048, 2050, 4096, 4099, 8192, 8200, 16384,
          16390, 32768, 32800, 65536]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k", WIDTHS)
def test_widths(k, dtype):
    sizes = [5, 0, 1, 37, 2] if k > 4096 else [40, 0, 1, 217, 64, 3]
    t = Case(sizes, k, dtype, pad=3, front=2, behind=3, seed=k)
    t.forward()
    t.check_forward()
    t.backward()
    t.check_backward()
    for which in (("dx",), ("dgain",), ("dshift",), ("dx", "dshift")):
        for q in ("dx", "dgain", "dshift"):
            getattr(t, q).fill_(7.0)
        t.backward(which=which)
        t.check_backward(which=which)
        for q in {"dx", "dgain", "dshift"} - set(which):
            assert (getattr(t, q) == 7.0).all(), q


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes", [[1], [0], [0, 0, 3], [1] * 200, [300, 0, 2000], [5003], [7] * 70 + [900], [0] * 130 + [1, 0, 64]])
@pytest.mark.parametrize("k", [35, 96, 640])
def test_blocks(sizes, k, dtype):
    t = Case(sizes, k, dtype, seed=len(sizes) + k)
    t.forward()
    t.check_forward()
    t.backward()
    t.check_backward()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_rows_take_many_runs(dtype):
    t = Case([30_011, 0, 64, 20_000], 96, dtype, seed=3)
    t.forward()
    t.check_forward()
    t.backward()
    t.check_backward()
    one = [getattr(t, q).clone() for q in ("dx", "dgain", "dshift")]
    t.ws.random_(0, 255)
    t.backward()
    assert all(torch.equal(a, getattr(t, q)) for a, q in zip(one, ("dx", "dgain", "dshift")))          # the same bits


@pytest.mark.parametrize("k", [96, 20_000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_without_gain_and_shift_and_in_place(k, dtype):
    t = Case([9, 30], k, dtype, affine=False, seed=5)
    t.forward(eps=0.25)
    t.check_forward(eps=0.25)
    t.backward(eps=0.25)
    t.check_backward(eps=0.25)
    for place in ("dy", "x"):
        t = Case([9, 30, 70], k, dtype, seed=6)
        before = _np(t.dy), _np(t.x)
        t.dx = getattr(t, place)
        t.backward()
        t.check_backward(inputs=before)
    t = Case([9, 30, 70], k, dtype, seed=7)
    x = _np(t.x)
    t.y = t.x
    t.forward()
    _close(t.y, *N.forward(x, t.offsets, _np(t.gain), _np(t.shift)), dtype, "y in the place of x")


def test_rows_far_from_zero_keep_their_digits():
    # level 4096, spread 1: mean(x^2) - mean^2 would have nothing left of the variance's last digits
    g = torch.Generator().manual_seed(11)
    x = (4096 + torch.randn(50, 256, generator=g)).to(DEV)
    y, off = torch.empty_like(x), torch.tensor([0, 50], dtype=torch.int32, device=DEV)
    B.grouped_norm(x, off, y)
    want, _ = N.forward(_np(x), [0, 50])
    # the mean of numbers in [4090, 4103] is off by at most the 14 roundings of partial sums below 2^20 (half an ulp is 2^-5 there),
    # over 256 values, and its own: 14 * 2^-5 / 256 + 2^-12; the spread is 1
    assert np.abs(_np(y) - want).max() <= (14 * 2.0 ** -5 / 256 + 2.0 ** -12) * 1.2


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_one_value_and_rows_that_are_not_finite(dtype):
    t = Case([4, 6], 96, dtype, seed=9)
    t.x[1] = 3.0
    t.x[2] = 0.0
    t.x[5, 7] = float("nan")
    t.x[6, 95] = float("inf")
    t.x[7, 0] = float("-inf")
    t.forward()
    want, bound = N.forward(_np(t.x), t.offsets, _np(t.gain), _np(t.shift))
    got = _np(t.y)
    assert np.isnan(got[5:8]).all() and np.isfinite(np.delete(got, [5, 6, 7], axis=0)).all()
    # 1 / deviation is 1 / sqrt(eps) = 316 there, and a mean that is one rounding off shows as 316 * 3 * 2^-24: the oracle's bound has it
    _close(t.y[1:3], want[1:3], bound[1:3], dtype, "rows of one value")
    t.backward()
    assert torch.isnan(t.dx[5:8]).all() and torch.isfinite(t.dx[:5]).all() and torch.isfinite(t.dx[8:]).all()
    assert torch.isfinite(t.dgain[0]).all() and torch.isnan(t.dgain[1]).all() and torch.isfinite(t.dshift).all()


def test_gradient_is_that_of_differences():
    rng = np.random.default_rng(4)
    t = Case([6, 0, 11], 40, seed=12)
    t.backward(eps=0.1)
    x, dy, gain, shift = (_np(v) for v in (t.x, t.dy, t.gain, t.shift))
    loss = lambda x_, g_, s_: (N.forward(x_, t.offsets, g_, s_, eps=0.1)[0] * dy).sum()
    ex, eg, es, h = rng.normal(size=x.shape), rng.normal(size=gain.shape), rng.normal(size=shift.shape), 1e-5
    for f, got in ((lambda q: loss(x + q * ex, gain, shift), (_np(t.dx) * ex).sum()), (lambda q: loss(x, gain + q * eg, shift), (_np(t.dgain) * eg).sum()),
                   (lambda q: loss(x, gain, shift + q * es), (_np(t.dshift) * es).sum())):
        assert abs((f(h) - f(-h)) / (2 * h) - got) < 1e-3


def test_offsets_that_go_beyond_the_rows_count_as_the_rows():
    t = Case([10, 20], 64, seed=13)
    t.off = torch.tensor([0, 10, 99], dtype=torch.int32, device=DEV)
    t.forward()
    t.check_forward()
    t.backward()
    t.check_backward()


@pytest.mark.parametrize("k", [96, 1000])
def test_on_a_stream_and_in_a_graph(k):
    t = Case([70, 0, 333], k, "bf16", seed=14)
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
        for q in (t.y, t.dx, t.dgain, t.dshift):
            q.fill_(7.0)
        t.ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        t.check_forward()
        t.check_backward()


def _additions(k):
    """On a value's way into a sum over a row: those of a thread, over a wavefront and over wavefronts."""
    return min(k, max(16, (k + 1023) // 1024 + 3) + 6 + 4)


# every arrangement of a row: over 8, 16, 64, 256 and 1024 lanes, and longer than registers
FAR_WIDTHS = [1, 20, 96, 100, 500, 1000, 4000, 4100, 8190, 9000, 20_000]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k", FAR_WIDTHS)
def test_rows_of_one_value_give_their_shift(k, dtype):
    # d = x - mean is the mean's error, (M + 2) u of the value at most; its own mean is off by (M + 2) u of it, the difference rounded once; 1 / deviation
    # is 1 / sqrt(eps), or 2^8 / d, at most.  In bfloat16 sums of values that are alike are exact, and so is d
    t = Case([6, 2], k, dtype, seed=31)
    t.gain[1:].fill_(1.0)
    t.shift[1:].fill_(0.0)
    for i, v in enumerate((0.1, -1000.1, 1e6 + 0.5, 1e10, 3.3e38, -7.7e20, 0.0, 1e-30)):
        t.x[i] = v
    t.forward()
    m, value = _additions(k) + 4, np.abs(_np(t.x[:, :1]))
    h = 0.0 * value if dtype == "bf16" else np.minimum(m * m * U * U * value / 1e-5 ** 0.5, 2.0 ** 8 * m * U)
    gain, shift = (_np(v)[[0] * 6 + [1] * 2] for v in (t.gain, t.shift))
    assert (np.abs(_np(t.y) - shift) <= np.abs(gain) * h + (2 * U + (2.0 ** -8 if dtype == "bf16" else 0)) * (np.abs(shift) + np.abs(gain) * h)).all()
    # the gradients: h is 0, 1 / deviation 1 / sqrt(eps), but for d's square: of the first two rows alone, whose d is small beside it
    t.backward()
    assert torch.isfinite(t.dx).all()
    dy, dgain = _np(t.dy), _np(t.dgain)
    assert (np.abs(dgain[0]) <= (np.abs(dy[:6]) * h[:6]).sum(0) * (1 + 20 * U)).all() and (np.abs(dgain[1]) <= (np.abs(dy[6:]) * h[6:]).sum(0) * (1 + 20 * U)).all()
    d = dy[:2] * gain[:2]
    want = (d - d.mean(1, keepdims=True)) / 1e-5 ** 0.5
    near = (m * U * value[:2]) ** 2 * (2.0 ** -16 + 4 * m * U) / 1e-5 if dtype == "f32" else 0.0
    off = np.abs(d).mean(1, keepdims=True)
    tol = ((np.abs(d) + off) * (near + m * U + h[:2] ** 2) + off * h[:2] ** 2) / 1e-5 ** 0.5
    assert (np.abs(_np(t.dx[:2]) - want) <= tol * 1.01 + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0)).all()


@pytest.mark.parametrize("k", FAR_WIDTHS[3:])
def test_rows_far_from_zero_are_those_of_level_zero(k):
    # level 2^20, spread 1, float32: d is exact, its mean `off` the mean's error, (M + 2) u 2^20 at most and itself off by (M + 2) u of what it is summed
    # from; the mean of the squares is off by (M + 2) u of itself, which holds off^2, too
    g = torch.Generator().manual_seed(32)
    x = (2.0 ** 20 + torch.randn(40, k, generator=g)).to(DEV)
    y, off = torch.empty_like(x), torch.tensor([0, 40], dtype=torch.int32, device=DEV)
    B.grouped_norm(x, off, y)
    want, _ = N.forward(_np(x), [0, 40])
    m = _additions(k) + 4
    e = m * U * 2.0 ** 20
    tol = m * U * (1.2 + e) + np.abs(want) * (m * U * (1.2 + e * e) + 4 * U)
    assert (np.abs(_np(y) - want) <= tol).all(), np.abs(_np(y) - want).max()
    dy, dx, dgain = torch.randn(40, k, generator=g).to(DEV), torch.empty_like(x), torch.empty(1, k, device=DEV)
    ws = torch.empty(B.grouped_norm_backward_bytes(40, 1, k), dtype=torch.uint8, device=DEV)
    B.grouped_norm_backward(dy, x, off, ws, dx=dx, dgain=dgain)
    d = _np(dy)
    grads, _ = N.backward(d, _np(x), [0, 40])
    assert (np.abs(_np(dgain)[0] - grads[1][0]) <= (np.abs(d) * tol).sum(0) + 42 * U * np.abs(d * want).sum(0)).all()
    # s (dy - mean(dy) - h mean(dy h)): of the terms' magnitudes, 1.2 being more than 1 / deviation, the sum of w d has off times that of w beside it
    size = np.abs(d) + np.abs(d).mean(1, keepdims=True) + np.abs(want) * np.abs(d * want).mean(1, keepdims=True)
    along = (np.abs(d) * tol).mean(1, keepdims=True) + m * U * (np.abs(d * want).mean(1, keepdims=True) + 2.4 * e * np.abs(d).mean(1, keepdims=True))
    spread = m * U * (1.2 + e * e) + 8 * U
    assert (np.abs(_np(dx) - grads[0]) <= 1.2 * (size * (spread + m * U) + np.abs(want) * along + tol * np.abs(d * want).mean(1, keepdims=True))).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k", FAR_WIDTHS[1:])
def test_rows_of_large_values_keep_theirs(k, dtype):
    # squares, sums and differences that pass 2^128, in blocks with ordinary rows
    t = Case([9, 3], k, dtype, pad=3, seed=33)
    sign = torch.where(torch.arange(k) % 2 == 0, 1.0, -1.0).to(DEV)
    for i, v in ((1, 1e18), (2, 3e19), (4, 1e25), (5, 1e30), (7, 1e37)):
        t.x[i] *= v
    t.x[8] = 3.3e38 * sign
    t.x[9] = 3.3e38
    t.x[9, 0] = -3.3e38
    t.x[10] = 2.0 ** 100 * (1 + 2.0 ** -7 * (torch.arange(k) % 3).to(DEV))
    t.forward()
    t.check_forward()
    assert (t.y[8] != t.shift[0].to(t.y.dtype)).any() and torch.isfinite(t.y).all()
    t.backward()
    t.check_backward()
    assert torch.isfinite(t.dx).all() and torch.isfinite(t.dgain).all()


@pytest.mark.parametrize("k", [96, 1000, 20_000])
def test_rows_of_large_values_in_place(k):
    t = Case([5, 80], k, "f32", seed=34)
    t.x[3] *= 1e30
    t.x[70:] *= 1e22
    x, dy = _np(t.x), _np(t.dy)
    t.dx = t.dy
    t.backward()
    t.check_backward(inputs=(dy, x))
    t.y = t.x
    t.forward()
    _close(t.y, *N.forward(x, t.offsets, _np(t.gain), _np(t.shift)), "f32", "y in the place of x")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k", [9, 96, 1000, 5000, 20_000])
@pytest.mark.parametrize("eps", [1e-5, 1e6])
def test_rows_that_are_not_finite_are_nan_whatever_eps_is(eps, k, dtype):
    # of an eps that is left at the scale of large rows, too, where it is all there is beside what is no number
    t = Case([4, 2], k, dtype, seed=35)
    t.x[1, k // 2] = float("inf")
    t.x[2, 0] = float("-inf")
    t.x[4, k - 1] = float("nan")
    t.forward(eps=eps)
    t.backward(eps=eps)
    bad = torch.tensor([False, True, True, False, True, False], device=DEV)
    for got in (t.y, t.dx):
        assert torch.isnan(got[bad]).all() and torch.isfinite(got[~bad]).all()
