"""The 4-bit form, equal to the oracle's byte for byte, and layers of blocks in it: within (k + 2) 2^-24 of the sum of the magnitudes of
their products, which are exact; results in bfloat16 rounded once more, 2^-8 of their value."""
import numpy as np
import pytest
import torch

from oracle import block4_ref as Q
from oracle.grouped_ref import blocks_of
from paper_2503_21364_amd import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
DEV = "cuda:0"


def _np(t):
    return t.detach().double().cpu().numpy()


def _form(rows, k):
    f = B.Block4(rows, k)
    f.codes.fill_(0x99)
    f.scale.fill_(0x99)
    return f


def _bytes(f):
    return f.codes.cpu().numpy(), f.scale.cpu().numpy()


def _packed(x):
    """The form of a float tensor, by the library."""
    f = _form(*x.shape)
    B.block4_pack(x, f)
    return f


# ---- the form
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,k", [(1, 1), (3, 31), (2, 32), (5, 33), (7, 96), (1, 127), (4, 128), (3, 129), (2, 511), (9, 512), (5, 513), (300, 131), (2, 4100)])
@pytest.mark.parametrize("pad", [0, 3])
def test_form_there_and_back(rows, k, pad, dtype):
    rng = np.random.default_rng(rows * 1000 + k)
    v = rng.normal(size=(rows, k + pad)) * np.exp2(rng.integers(-30, 30, size=(rows, 1)))
    v[rng.random(v.shape) < 0.1] = 0
    x = torch.from_numpy(v.astype(np.float32)).to(DT[dtype])
    if pad:
        x[:, k:] = float("nan")
    x = x.to(DEV)[:, :k]
    f = _packed(x)
    codes, scale = Q.pack(_np(x))
    np.testing.assert_array_equal(_bytes(f)[1], scale)
    np.testing.assert_array_equal(_bytes(f)[0], codes)
    back = torch.full((rows, k + pad), 7.0, dtype=DT[dtype], device=DEV)
    B.block4_unpack(f, back[:, :k])
    np.testing.assert_array_equal(_np(back[:, :k]), Q.unpack(codes, scale, k))
    assert (back[:, k:] == 7.0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_form_of_every_bfloat16(dtype):
    # all 65536 of them, sorted and in random company, negative zeros, denormals, infinities and NaN
    rng = np.random.default_rng(2)
    bits = np.concatenate([np.arange(65536), rng.permutation(65536)]).astype(np.uint16)
    x = torch.from_numpy((bits.astype(np.uint32) << 16).view(np.float32).reshape(-1, 256).copy()).to(DT[dtype]).to(DEV)
    f = _packed(x)
    codes, scale = Q.pack(_np(x))
    np.testing.assert_array_equal(_bytes(f)[1], scale)
    np.testing.assert_array_equal(_bytes(f)[0], codes)
    back = torch.empty_like(x)
    B.block4_unpack(f, back)
    got, want = _np(back), Q.unpack(codes, scale, 256)
    np.testing.assert_array_equal(got, want)
    assert (np.signbit(got) == np.signbit(want))[np.isfinite(want)].all()


def test_form_at_ties_and_next_to_them():
    # every border between two codes, and the float32 on either side of it, at several steps
    border = np.array([0.25, 0.5, 0.75, 1.0, 1.25, 1.5, 1.75, 2.0, 2.5, 3.0, 3.5, 4.0, 5.0, 6.0, 6.9999995], np.float32)
    near = np.concatenate([border, np.nextafter(border, np.float32(0)), np.nextafter(border[:-1], np.float32(9))])
    rows = []
    for e in (-100, -1, 0, 3, 100):
        for sign in (1, -1):
            for at in range(0, len(near), 31):
                v = np.zeros(32, np.float32)
                v[:len(near[at:at + 31])] = sign * near[at:at + 31]
                v[31] = 6.0                                     # the step is 1
                rows.append(v * np.float32(2.0) ** e)
    x = np.stack(rows)
    f = _packed(torch.from_numpy(x).to(DEV))
    codes, scale = Q.pack(x)
    np.testing.assert_array_equal(_bytes(f)[1], scale)
    np.testing.assert_array_equal(_bytes(f)[0], codes)


# ---- layers
class Layer:
    def __init__(self, sizes, k, n, dtype="f32", pad=0, front=0, behind=0, seed=0, whole=False):
        g = torch.Generator().manual_seed(seed)
        self.sizes, self.k, self.n, self.dtype, self.pad = sizes, k, n, dtype, pad
        self.offsets = [front] + [front + int(v) for v in np.cumsum(sizes)]
        self.rows, blocks = self.offsets[-1] + behind, len(sizes)
        draw = (lambda *s: torch.randint(-2, 3, s, generator=g).float()) if whole else (lambda *s: torch.randn(s, generator=g))
        x = draw(self.rows, k)
        x[:front] = float("nan")
        x[self.offsets[-1]:] = float("nan")
        self.x4, self.w4 = _packed(x.to(DEV)), _packed(draw(blocks * n, k).to(DEV))
        self.b = draw(blocks, n).to(DEV)
        self.off = torch.tensor(self.offsets, dtype=torch.int32, device=DEV)
        self.y = torch.full((self.rows, n + pad), 7.0, dtype=DT[dtype], device=DEV)[:, :n]

    def run(self, bias=True, relu=False, stream=None):
        B.grouped_linear4(self.x4, self.w4, self.off, self.y, bias=self.b if bias else None, relu=relu, stream=stream)

    def check(self, bias=True, relu=False, exact=False):
        want, mag = Q.forward(_bytes(self.x4), _bytes(self.w4), self.offsets, self.k, _np(self.b) if bias else None, relu)
        got = _np(self.y)
        tol = (self.k + 3) * U * mag + (2.0 ** -8 * np.abs(want) if self.dtype == "bf16" else 0) + 1e-38
        if exact:
            want, tol = torch.from_numpy(want).to(DT[self.dtype]).double().numpy(), 0.0
        # where the magnitudes add up to 2^128 and more, a sum in 32 bits may pass through infinity, whatever its value is
        fits = ~(mag >= 2.0 ** 127)
        np.testing.assert_array_equal(np.isnan(got[fits]), np.isnan(want[fits]))
        with np.errstate(invalid="ignore"):
            bad = fits & ~np.isnan(want) & ~(np.abs(got - want) <= tol)
        assert not bad.any(), (int(bad.sum()), got[bad][:4], want[bad][:4], np.argwhere(bad)[:4].tolist())
        if self.pad and self.rows:
            assert (self.y.as_strided((self.rows, self.pad), self.y.stride(), self.n) == 7.0).all()


SHAPES = [
    ([1], 1, 1), ([1], 35, 96), ([0, 1, 0], 32, 70), ([3, 0, 0, 5, 1], 7, 5), ([127, 128, 129], 31, 33), ([300], 64, 64), ([40, 0, 217, 64], 35, 96),
    ([500, 1, 2], 129, 70), ([255, 256, 257], 128, 128), ([700, 20], 131, 257), ([90, 300], 256, 192), ([16] * 70, 96, 40), ([2049, 511], 640, 320),
    ([33], 1000, 24), ([1, 1, 1, 1], 512, 512), ([900, 0, 130], 513, 264), ([1300, 1], 8, 1024), ([600], 1032, 136), ([1], 4096, 333), ([17, 2], 4224, 65),
    ([6000, 0, 2500, 30], 384, 512), ([20_011, 0, 64], 200, 640),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes,k,n", SHAPES)
def test_layer(sizes, k, n, dtype):
    t = Layer(sizes, k, n, dtype, seed=k + n)
    t.run()
    t.check()
    t.run(bias=False, relu=True)
    t.check(bias=False, relu=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes,k,n", SHAPES)
def test_layer_of_whole_numbers_is_exact(sizes, k, n, dtype):
    # -2 .. 2 are codes of some step whatever 32 of them share it, and sums of their products whole numbers below 2^24
    t = Layer(sizes, k, n, dtype, seed=k + n + 1, whole=True)
    t.run()
    t.check(exact=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes,k,n", [([60, 0, 700, 1], 136, 200), ([4, 3], 600, 40), ([3000, 900], 256, 384)])
def test_strides_and_rows_of_no_block(sizes, k, n, dtype):
    for pad in (8, 5):
        t = Layer(sizes, k, n, dtype, pad=pad, front=5, behind=70, seed=pad)
        t.run(relu=True)
        t.check(relu=True)


@pytest.mark.parametrize("dtype,sizes,k,n", [("f32", [20], 256, 64), ("bf16", [900, 200], 640, 256)])
def test_what_is_not_finite_and_what_is_far_apart(dtype, sizes, k, n):
    t = Layer(sizes, k, n, dtype, seed=3)
    clean = Layer(sizes, k, n, dtype, seed=3)
    t.x4.scale[5, 1] = 255                      # what pack makes of an infinity or a NaN
    t.x4.codes[5, 16:32] = 0
    t.w4.scale[7, 0] = 255
    t.w4.codes[7, :16] = 0
    t.run()
    clean.run()
    keep = torch.ones_like(t.y, dtype=torch.bool)
    keep[5] = False
    keep[:sizes[0], 7] = False
    assert torch.isnan(t.y[5]).all() and torch.isnan(t.y[:sizes[0], 7]).all()
    assert torch.equal(t.y[keep], clean.y[keep])
    # powers of two from the least to the greatest
    t = Layer(sizes, k, n, dtype, seed=4)
    t.x4.scale[1, :k // 32] = 1
    t.w4.scale[3, :k // 32] = 252
    t.x4.scale[2, :k // 32] = 0
    t.x4.codes[2] = 0
    t.run()
    t.check()


def test_offsets_that_go_beyond_the_rows_count_as_the_rows():
    t = Layer([10, 200], 64, 32, "bf16", seed=9)
    t.off = torch.tensor([0, 10, 999], dtype=torch.int32, device=DEV)
    t.run()
    t.check()


@pytest.mark.parametrize("dtype,sizes,k,n", [("f32", [3, 0, 1], 1024, 200), ("bf16", [3000, 0, 333], 512, 512)])
def test_on_a_stream_and_in_a_graph(dtype, sizes, k, n):
    t = Layer(sizes, k, n, dtype, seed=10)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    t.run(stream=side)
    side.synchronize()
    t.check()
    x = torch.randn(t.rows, k, device=DEV)
    back = torch.empty_like(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.block4_pack(x, t.x4)
        B.block4_unpack(t.x4, back)
        t.run()
    for seed in (1, 2, 3):
        x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(seed)))
        t.y.fill_(7.0)
        t.x4.codes.fill_(0x99)
        t.x4.scale.fill_(0x99)
        graph.replay()
        torch.cuda.synchronize()
        codes, scale = Q.pack(_np(x[:40]))
        np.testing.assert_array_equal(t.x4.codes[:40].cpu().numpy(), codes)
        np.testing.assert_array_equal(_np(back[:40]), Q.unpack(codes, scale, k))
        t.check()


def test_rows_of_a_layer_in_bfloat16_are_those_of_its_4_bit_operands():
    # the same product through grouped_linear, whose operands are the values that the codes stand for
    t = Layer([200, 56], 256, 128, "bf16", seed=11)
    x, w = torch.empty(t.rows, 256, dtype=torch.bfloat16, device=DEV), torch.empty(2 * 128, 256, dtype=torch.bfloat16, device=DEV)
    B.block4_unpack(t.x4, x)
    B.block4_unpack(t.w4, w)
    other = torch.empty_like(t.y)
    B.grouped_linear(x, w.reshape(2, 128, 256), t.off, other, bias=t.b)
    t.run()
    want, mag = Q.forward(_bytes(t.x4), _bytes(t.w4), t.offsets, 256, _np(t.b))
    assert (np.abs(_np(other) - _np(t.y)) <= 2 * ((256 + 3) * U * mag + 2.0 ** -8 * np.abs(want))).all()
    assert [b - a for a, b in blocks_of(t.offsets, t.rows)] == [200, 56]
