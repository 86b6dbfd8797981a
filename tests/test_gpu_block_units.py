"""The operators of blocks one after the other, as a block's decoder uses them: norm, gated layer, linear layer and the gradients all the way
back; and the same layers answered from 4-bit weights.  Every operator is held to its own oracle and bound on what it was given, so that a
buffer that another one still needed, or had not finished, shows.  Also: rows whose offsets pass 32 bits, blocks without rows in the kernels for few
rows, a thousand blocks, no rows at all."""
import numpy as np
import pytest
import torch

from oracle import block4_ref as Q
from oracle import gated_ref as G
from oracle import grouped_ref as L
from oracle import norm_ref as N
from paper_2503_21364_amd import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
DEV = "cuda:0"


def _np(t):
    return t.detach().double().cpu().numpy()


def _close(got, want, bound, rounded, what):
    got = _np(got)
    tol = bound * 1.0001 + (2.0 ** -8 * (np.abs(want) + bound) if rounded else 0.0) + 1e-36
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (what, int(bad.sum()), got[bad][:4], want[bad][:4], tol[bad][:4])


class Unit:
    """h = norm(x), y = gated(h), z = linear(y); dz to dy to dh to dx, and the gradients of all weights.  One workspace for all three."""

    def __init__(self, sizes, k, n, dtype, seed=0, act="silu"):
        g = torch.Generator().manual_seed(seed)
        self.k, self.n, self.dtype, self.act, self.blocks = k, n, dtype, act, len(sizes)
        self.offsets = [0] + [int(v) for v in np.cumsum(sizes)]
        rows, dt = self.offsets[-1], DT[dtype]
        self.off = torch.tensor(self.offsets, dtype=torch.int32, device=DEV)
        draw = lambda *s: torch.randn(s, generator=g)
        self.x, self.dz = draw(rows, k).to(dt).to(DEV), draw(rows, k).to(dt).to(DEV)
        self.gain, self.shift = (1 + 0.2 * draw(self.blocks, k)).to(DEV), (0.2 * draw(self.blocks, k)).to(DEV)
        self.w = (draw(self.blocks, 2 * n, k) / k ** 0.5).to(dt).to(DEV)
        self.b = draw(self.blocks, 2 * n).to(DEV)
        self.v = (draw(self.blocks, k, n) / n ** 0.5).to(dt).to(DEV)
        e = lambda *s, t=dt: torch.empty(s, dtype=t, device=DEV)
        self.h, self.y, self.z = e(rows, k), e(rows, n), e(rows, k)
        self.dy, self.dh, self.dx = e(rows, n), e(rows, k), e(rows, k)
        self.dv, self.dw, self.db = e(self.blocks, k, n, t=torch.float32), e(self.blocks, 2 * n, k), e(self.blocks, 2 * n, t=torch.float32)
        self.dgain, self.dshift = e(self.blocks, k, t=torch.float32), e(self.blocks, k, t=torch.float32)
        need = (B.grouped_linear_backward_bytes(rows, self.blocks, k, n, dt), B.grouped_gated_backward_bytes(rows, self.blocks, n, k, dt),
                B.grouped_norm_backward_bytes(rows, self.blocks, k, dt))
        self.ws = torch.empty(max(need), dtype=torch.uint8, device=DEV)

    def step(self):
        B.grouped_norm(self.x, self.off, self.h, gain=self.gain, shift=self.shift)
        B.grouped_gated(self.h, self.w, self.off, self.y, bias=self.b, act=self.act)
        B.grouped_linear(self.y, self.v, self.off, self.z)
        B.grouped_linear_backward(self.dz, self.v, self.off, self.ws, x=self.y, dx=self.dy, dw=self.dv)
        B.grouped_gated_backward(self.dy, self.h, self.w, self.off, self.ws, bias=self.b, act=self.act, dx=self.dh, dw=self.dw, db=self.db)
        B.grouped_norm_backward(self.dh, self.x, self.off, self.ws, gain=self.gain, dx=self.dx, dgain=self.dgain, dshift=self.dshift)

    def check(self):
        half, m = self.dtype == "bf16", max(np.diff(self.offsets))
        x, h, y, dy, dh, w, v = (_np(t) for t in (self.x, self.h, self.y, self.dy, self.dh, self.w, self.v))
        _close(self.h, *N.forward(x, self.offsets, _np(self.gain), _np(self.shift)), half, "h")
        _close(self.y, *G.forward(h, w, self.offsets, _np(self.b), self.act), half, "y")
        want, mag = L.forward(y, v, self.offsets)
        _close(self.z, want, (self.n + 2) * U * mag, half, "z")
        (want, dv, _), (mag, mv, _) = L.backward(_np(self.dz), y, v, self.offsets)
        _close(self.dy, want, (self.k + 2) * U * mag, half, "dy")
        _close(self.dv, dv, (m + 2) * U * mv, False, "dv")
        want, bound = G.backward(dy, h, w, self.offsets, _np(self.b), self.act, half)
        for i, (got, rounded) in enumerate(((self.dh, half), (self.dw, half), (self.db, False))):
            _close(got, want[i], bound[i], rounded, ("dh", "dw", "db")[i])
        want, bound = N.backward(dh, x, self.offsets, _np(self.gain))
        for i, (got, rounded) in enumerate(((self.dx, half), (self.dgain, False), (self.dshift, False))):
            _close(got, want[i], bound[i], rounded, ("dx", "dgain", "dshift")[i])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes,k,n,act", [([300, 0, 77], 35, 32, "gelu"), ([700, 130], 256, 192, "silu"), ([3, 0, 1, 2], 96, 40, "silu"), ([900], 131, 77, "gelu")])
def test_training_unit(sizes, k, n, act, dtype):
    t = Unit(sizes, k, n, dtype, act=act)
    t.step()
    t.check()


def test_gradients_of_a_unit_are_those_of_its_composition():
    """dx of the whole unit in float32 against torch's own gradients of the formulas in 64 bits.  The unit's bound is that of its parts: every stage's
    result is off by a relative 2^-24 times the terms of its sums (at most 2 n = 64, and the conditioning of sums of random signs, 2-norms), six stages,
    so that 6 * 64 * 2^-24 = 2.3e-5 of the gradient's 2-norm covers it."""
    t = Unit([40, 0, 23], 35, 32, "f32", seed=3)
    t.step()
    x = t.x.double().cpu().requires_grad_(True)
    z = []
    for g, (a, b) in enumerate(L.blocks_of(t.offsets, x.shape[0])):
        if a == b:
            continue
        c = x[a:b] - x[a:b].mean(1, keepdim=True)
        h = c / torch.sqrt((c * c).mean(1, keepdim=True) + 1e-5) * t.gain[g].double().cpu() + t.shift[g].double().cpu()
        p = h @ t.w[g].double().cpu().T + t.b[g].double().cpu()
        z.append((torch.nn.functional.silu(p[:, :t.n]) * p[:, t.n:]) @ t.v[g].double().cpu().T)
    want, = torch.autograd.grad((torch.cat(z) * t.dz.double().cpu()).sum(), x)
    assert (t.dx.double().cpu() - want).norm() <= 2.3e-5 * want.norm()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_two_graphs_share_a_workspace(dtype):
    a, b = Unit([200, 0, 64], 64, 96, dtype, seed=1), Unit([90, 300], 96, 64, dtype, seed=2)
    ws = a.ws if a.ws.numel() >= b.ws.numel() else b.ws
    a.ws = b.ws = ws
    for t in (a, b):
        t.step()
    torch.cuda.synchronize()
    graphs = []
    for t in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            t.step()
        graphs.append(g)
    for i in range(3):
        for t in (a, b):
            t.x.copy_(torch.randn(t.x.shape, generator=torch.Generator().manual_seed(10 + i)))
        ws.fill_(255)
        for g in graphs:
            g.replay()
        ws.fill_(1)                              # eager work between the replays
        torch.cuda.synchronize()
        a.check()
        b.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes,k,n", [([1], 256, 192), ([400, 0, 130], 256, 192), ([5, 2, 0, 9], 600, 70)])
def test_answering_unit_from_4_bit_weights(sizes, k, n, dtype):
    """norm, its output to 4 bits, a layer with a ReLU, to 4 bits again, a second layer; weights packed once."""
    t = Unit(sizes, k, n, dtype, seed=4)
    rows, w4, v4, h4, y4 = t.x.shape[0], B.Block4(t.blocks * n, k), B.Block4(t.blocks * k, n), B.Block4(t.x.shape[0], k), B.Block4(t.x.shape[0], n)
    b = torch.randn(t.blocks, n, device=DEV)
    B.block4_pack(t.w[:, :n].reshape(-1, k), w4)
    B.block4_pack(t.v.reshape(-1, n), v4)

    def answer():
        B.grouped_norm(t.x, t.off, t.h, gain=t.gain, shift=t.shift)
        B.block4_pack(t.h, h4)
        B.grouped_linear4(h4, w4, t.off, t.y, bias=b, relu=True)
        B.block4_pack(t.y, y4)
        B.grouped_linear4(y4, v4, t.off, t.z)

    def check():
        data = lambda f: (f.codes.cpu().numpy(), f.scale.cpu().numpy())
        _close(t.h, *N.forward(_np(t.x), t.offsets, _np(t.gain), _np(t.shift)), dtype == "bf16", "h")
        for form, of in ((h4, t.h), (y4, t.y), (w4, t.w[:, :n].reshape(-1, k)), (v4, t.v.reshape(-1, n))):
            codes, scale = Q.pack(_np(of))
            assert np.array_equal(data(form)[0], codes) and np.array_equal(data(form)[1], scale)
        want, mag = Q.forward(data(h4), data(w4), t.offsets, k, _np(b), True)
        _close(t.y, want, (k + 3) * U * mag, dtype == "bf16", "y")
        want, mag = Q.forward(data(y4), data(v4), t.offsets, n)
        _close(t.z, want, (n + 3) * U * mag, dtype == "bf16", "z")

    answer()
    check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        answer()
    for i in range(2):
        t.x.copy_(torch.randn(rows, k, generator=torch.Generator().manual_seed(20 + i)))
        t.z.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        check()


# ---- where it can go wrong by size
ROWS = (1 << 31) // 1024 + 3000           # of 1024 values: more than 2^31 of them


def _last(t, count=300):
    return _np(t[-count:])


def test_norm_of_more_than_2_31_values():
    x = torch.empty(ROWS, 1024, dtype=torch.bfloat16, device=DEV)
    for part in x.split(1 << 18):
        part.normal_()
    off = torch.tensor([0, ROWS - 1000, ROWS], dtype=torch.int32, device=DEV)
    gain, shift = torch.randn(2, 1024, device=DEV), torch.randn(2, 1024, device=DEV)
    y = torch.empty_like(x)
    B.grouped_norm(x, off, y, gain=gain, shift=shift)
    _close(y[-300:], *N.forward(_last(x), [0, 300], _np(gain[1:]), _np(shift[1:])), True, "y")
    dgain, dshift = torch.empty(2, 1024, device=DEV), torch.empty(2, 1024, device=DEV)
    ws = torch.empty(B.grouped_norm_backward_bytes(ROWS, 2, 1024, torch.bfloat16), dtype=torch.uint8, device=DEV)
    dy = y                                  # as good as any; dx takes its place
    last = _np(dy[-1000:])
    B.grouped_norm_backward(dy, x, off, ws, gain=gain, dx=dy, dgain=dgain, dshift=dshift)
    want, bound = N.backward(last, _last(x, 1000), [0, 1000], _np(gain[1:]))
    _close(dy[-1000:], want[0], bound[0], True, "dx")
    _close(dgain[1:], want[1], bound[1], False, "dgain")
    _close(dshift[1:], want[2], bound[2], False, "dshift")


def test_gated_layer_of_more_than_2_31_results():
    k, n = 16, 1024
    x = torch.randn(ROWS, k, device=DEV).to(torch.bfloat16)
    w = torch.randn(2, 2 * n, k, device=DEV).to(torch.bfloat16)
    off = torch.tensor([0, ROWS - 1000, ROWS], dtype=torch.int32, device=DEV)
    y = torch.empty(ROWS, n, dtype=torch.bfloat16, device=DEV)
    B.grouped_gated(x, w, off, y)
    _close(y[-300:], *G.forward(_last(x), _np(w[1:]), [0, 300]), True, "y")
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty(2, 2 * n, device=DEV)
    ws = torch.empty(B.grouped_gated_backward_bytes(ROWS, 2, n, k, torch.bfloat16), dtype=torch.uint8, device=DEV)
    B.grouped_gated_backward(y, x, w, off, ws, dx=dx, dw=dw, db=db)
    want, bound = G.backward(_last(y, 1000), _last(x, 1000), _np(w[1:]), [0, 1000], half=True)
    _close(dx[-1000:], want[0], bound[0], True, "dx")
    _close(dw[1:], want[1], bound[1], True, "dw")
    _close(db[1:], want[2], bound[2], False, "db")


def test_forms_and_layer_of_more_than_2_31_values():
    x = torch.empty(ROWS, 1024, dtype=torch.bfloat16, device=DEV)
    for part in x.split(1 << 18):
        part.normal_()
    f = B.Block4(ROWS, 1024)
    B.block4_pack(x, f)
    codes, scale = Q.pack(_last(x, 40))
    assert np.array_equal(f.codes[-40:].cpu().numpy(), codes) and np.array_equal(f.scale[-40:].cpu().numpy(), scale)
    B.block4_unpack(f, x)
    assert np.array_equal(_last(x, 40), Q.unpack(codes, scale, 1024))
    w4 = B.Block4(2 * 1024, 1024)
    w = torch.randn(2 * 1024, 1024, device=DEV)
    B.block4_pack(w, w4)
    off = torch.tensor([0, ROWS - 1000, ROWS], dtype=torch.int32, device=DEV)
    B.grouped_linear4(f, w4, off, x)
    want, mag = Q.forward((codes, scale), (w4.codes[1024:].cpu().numpy(), w4.scale[1024:].cpu().numpy()), [0, 40], 1024)
    _close(x[-40:], want, 1027 * U * mag, True, "y")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_thousand_blocks_of_few_rows_some_of_none(dtype):
    rng = np.random.default_rng(6)
    sizes = [int(v) for v in rng.integers(0, 4, 1000)]
    t = Unit(sizes, 24, 12, dtype, seed=5)
    t.step()
    t.check()
    first = [q.clone() for q in (t.dx, t.dw, t.db, t.dgain, t.dshift, t.z)]
    t.step()
    assert all(torch.equal(p, q) for p, q in zip(first, (t.dx, t.dw, t.db, t.dgain, t.dshift, t.z)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_rows_at_all(dtype):
    dt = DT[dtype]
    e = lambda *s, t=dt: torch.full(s, 7.0, dtype=t, device=DEV)
    off = torch.zeros(4, dtype=torch.int32, device=DEV)
    x, dy, w = e(0, 40), e(0, 24), e(3, 48, 40)
    dw, db, dgain, dshift = e(3, 48, 40), e(3, 48, t=torch.float32), e(3, 40, t=torch.float32), e(3, 40, t=torch.float32)
    B.grouped_norm(x, off, e(0, 40))
    B.grouped_gated(x, w, off, e(0, 24))
    ws = torch.empty(max(B.grouped_gated_backward_bytes(0, 3, 24, 40, dt), B.grouped_norm_backward_bytes(0, 3, 40, dt)), dtype=torch.uint8, device=DEV)
    B.grouped_gated_backward(dy, x, w, off, ws, dx=e(0, 40), dw=dw, db=db)
    B.grouped_norm_backward(x, x, off, ws, dx=e(0, 40), dgain=dgain, dshift=dshift)
    for t in (dw, db, dgain, dshift):
        assert (t == 0).all()
    f = B.Block4(0, 40)
    B.block4_pack(x, f)
    B.block4_unpack(f, x)
    B.grouped_linear4(f, B.Block4(3 * 24, 40), off, e(0, 24))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_no_block_where_rows_are_few(dtype):
    dt = DT[dtype]
    rows, k, n = 20, 256, 160
    x, dy = torch.randn(rows, k, device=DEV).to(dt), torch.randn(rows, n, device=DEV).to(dt)
    x[:3] = float("nan")
    x[15:] = float("nan")
    dy[:3] = float("nan")
    off = torch.tensor([3, 7, 7, 15], dtype=torch.int32, device=DEV)
    w = (torch.randn(3, 2 * n, k, device=DEV) / 16).to(dt)
    y, dx, dw, db = torch.full((rows, n), 7.0, dtype=dt, device=DEV), torch.full((rows, k), 7.0, dtype=dt, device=DEV), torch.empty_like(w), torch.empty(3, 2 * n, device=DEV)
    B.grouped_gated(x, w, off, y)
    _close(y, *G.forward(np.nan_to_num(_np(x)), _np(w), [3, 7, 7, 15]), dtype == "bf16", "y")
    ws = torch.empty(B.grouped_gated_backward_bytes(rows, 3, n, k, dt), dtype=torch.uint8, device=DEV)
    B.grouped_gated_backward(dy, x, w, off, ws, dx=dx, dw=dw, db=db)
    want, bound = G.backward(np.nan_to_num(_np(dy)), np.nan_to_num(_np(x)), _np(w), [3, 7, 7, 15], half=dtype == "bf16")
    for i, (got, rounded) in enumerate(((dx, dtype == "bf16"), (dw, dtype == "bf16"), (db, False))):
        _close(got, want[i], bound[i], rounded, ("dx", "dw", "db")[i])
    f, w4 = B.Block4(rows, k), B.Block4(3 * n, k)
    B.block4_pack(x, f)
    B.block4_pack(w[:, :n].reshape(-1, k), w4)
    B.grouped_linear4(f, w4, off, y)
    data = lambda q: (q.codes.cpu().numpy(), q.scale.cpu().numpy())
    xs = data(f)
    xs[1][:3] = xs[1][15:] = 0
    want, mag = Q.forward(xs, data(w4), [3, 7, 7, 15], k)
    _close(y, want, (k + 3) * U * mag, dtype == "bf16", "y of 4 bits")


def test_tiles_of_192_rows():
    """A size whose tiles of 256 x 256 would leave a last round nearly empty: forward (n = 4096) and dx (k = 4096) of 8300 rows in ragged blocks."""
    rows, offsets, many, few = 8300, [1, 3000, 3001, 8290], 4096, 72
    g = torch.Generator().manual_seed(12)
    off = torch.tensor(offsets, dtype=torch.int32, device=DEV)
    a = torch.randn(rows, few, generator=g).to(torch.bfloat16).to(DEV)
    w = (torch.randn(3, many, few, generator=g) / 8).to(torch.bfloat16).to(DEV)
    out = torch.full((rows, many), 7.0, dtype=torch.bfloat16, device=DEV)
    want, mag = L.forward(_np(a), _np(w), offsets)
    B.grouped_linear(a, w, off, out)
    _close(out, want, (few + 2) * U * mag, True, "y")
    # the same product as dx of a layer of 4096 inputs and 72 outputs
    v = w.transpose(1, 2).contiguous()
    ws = torch.empty(B.grouped_linear_backward_bytes(rows, 3, few, many, torch.bfloat16), dtype=torch.uint8, device=DEV)
    first = out.clone()
    B.grouped_linear_backward(a, v, off, ws, dx=out)
    _close(out, want, (few + 2) * U * mag, True, "dx")
    assert torch.equal(first, out)          # the same sums in the same order


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k", [4101, 8191, 8193, 16385, 20011])
def test_norms_of_long_rows_in_place(k, dtype):
    """Rows whose last vector begins in front of the one before it ends, results in the place of x and of dy, many rows a run."""
    dt, half, rows, offsets = DT[dtype], dtype == "bf16", 600, [2, 2, 30, 597]
    g = torch.Generator().manual_seed(k)
    x0, dy0 = (torch.randn(rows, k, generator=g).to(dt).to(DEV) for _ in range(2))
    gain, shift = torch.randn(3, k, generator=g).to(DEV), torch.randn(3, k, generator=g).to(DEV)
    off = torch.tensor(offsets, dtype=torch.int32, device=DEV)
    y = x0.clone()
    B.grouped_norm(y, off, y, gain=gain, shift=shift)
    _close(y, *N.forward(_np(x0), offsets, _np(gain), _np(shift)), half, "y")
    want, bound = N.backward(_np(dy0), _np(x0), offsets, _np(gain))
    ws = torch.empty(B.grouped_norm_backward_bytes(rows, 3, k, dt), dtype=torch.uint8, device=DEV)
    for place in ("x", "dy"):
        x, dy, dgain, dshift = x0.clone(), dy0.clone(), torch.full((3, k), 7.0, device=DEV), torch.full((3, k), 7.0, device=DEV)
        dx = x if place == "x" else dy
        B.grouped_norm_backward(dy, x, off, ws, gain=gain, dx=dx, dgain=dgain, dshift=dshift)
        _close(dx, want[0], bound[0], half, "dx")
        _close(dgain, want[1], bound[1], False, "dgain")
        _close(dshift, want[2], bound[2], False, "dshift")
