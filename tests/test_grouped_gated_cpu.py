"""Gated layers of blocks without a GPU: the oracle against differences and closed forms, and the calls' checks of their arguments."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import gated_ref as G
from paper_2503_21364_amd import binding as B


@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
def test_gradients_of_the_oracle_are_differences(act):
    rng = np.random.default_rng(5)
    offsets, rows, n, k = [1, 4, 4, 9], 10, 4, 6
    x, w, b, up = rng.normal(size=(rows, k)), rng.normal(size=(3, 2 * n, k)), rng.normal(size=(3, 2 * n)), rng.normal(size=(rows, n))
    (dx, dw, db), _ = G.backward(up, x, w, offsets, b, act)
    loss = lambda x_, w_, b_: (G.forward(x_, w_, offsets, b_, act)[0] * up).sum()
    h = 1e-6
    for _ in range(4):
        ex, ew, eb = rng.normal(size=x.shape), rng.normal(size=w.shape), rng.normal(size=b.shape)
        diff = lambda f: (f(h) - f(-h)) / (2 * h)
        assert abs(diff(lambda t: loss(x + t * ex, w, b)) - (dx * ex).sum()) < 1e-6
        assert abs(diff(lambda t: loss(x, w + t * ew, b)) - (dw * ew).sum()) < 1e-6
        assert abs(diff(lambda t: loss(x, w, b + t * eb)) - (db * eb).sum()) < 1e-6


def test_activations_of_the_oracle():
    a = np.array([-30.0, -1.0, 0.0, 1.0, 30.0])
    np.testing.assert_allclose(G.activation(a, "silu")[0], a / (1 + np.exp(-a)), rtol=1e-15)
    np.testing.assert_allclose(G.activation(a, "gelu")[0], [0, -0.15865525393145707, 0, 0.8413447460685429, 30], atol=1e-15)
    assert G.activation(a, "relu")[0].tolist() == [0, 0, 0, 1, 30] and G.activation(a, "relu")[1].tolist() == [0, 0, 0, 1, 1]
    t = torch.linspace(-9, 9, 4001, dtype=torch.float64, requires_grad=True)
    for act, f in (("silu", torch.nn.functional.silu), ("gelu", torch.nn.functional.gelu)):
        slope, = torch.autograd.grad(f(t).sum(), t)
        np.testing.assert_allclose(G.activation(t.detach().numpy(), act)[1], slope.numpy(), atol=1e-14)
        assert np.abs(slope.numpy()).max() <= G.STEEP and np.abs(np.diff(slope.numpy())).max() / (18 / 4000) <= G.BENT


def test_rows_of_no_block_and_empty_blocks_of_the_oracle():
    x, w = np.ones((6, 2)), np.ones((3, 6, 2))
    y, _ = G.forward(x, w, [1, 3, 3, 5], act="relu")
    assert (y[[0, 5]] == 0).all() and (y[1:5] == 4).all()
    (dx, dw, db), _ = G.backward(np.ones((6, 3)), x, w, [1, 3, 3, 5], act="relu")
    assert (dx[[0, 5]] == 0).all() and (dw[1] == 0).all() and (db[1] == 0).all() and (db[0] == 4).all()


# ---- refusals (fake pointers: every call below has to be refused before it reaches them)
def _layer(**kw):
    d = dict(w=0x10000, offsets=0x20000, ldw=16, w_block=16 * 16, blocks=3, rows=100, n=8, k=16, dtype=0, in_major=0)
    d.update(kw)
    return B.LinearC(*[d[f] for f, _ in B.LinearC._fields_])


BAD_LAYERS = [
    (dict(dtype=2), B.ERR_UNSUPPORTED), (dict(in_major=2), B.ERR_INVALID), (dict(blocks=0), B.ERR_INVALID), (dict(blocks=65537), B.ERR_INVALID),
    (dict(rows=1 << 31), B.ERR_INVALID), (dict(n=0), B.ERR_INVALID), (dict(k=0), B.ERR_INVALID), (dict(n=32769, w_block=1 << 30), B.ERR_INVALID),
    (dict(n=(1 << 31) + 1, w_block=1 << 40), B.ERR_INVALID), (dict(k=65537, ldw=65537, w_block=1 << 30), B.ERR_INVALID), (dict(ldw=15), B.ERR_INVALID),
    (dict(in_major=1, ldw=15), B.ERR_INVALID), (dict(w_block=255), B.ERR_INVALID), (dict(w=None), B.ERR_INVALID), (dict(w=0x10002), B.ERR_INVALID),
    (dict(offsets=None), B.ERR_INVALID), (dict(offsets=0x20002), B.ERR_INVALID), (dict(rows=(1 << 31) - 1, n=32768, w_block=1 << 21), B.ERR_UNSUPPORTED),
]


@pytest.mark.parametrize("bad,code", BAD_LAYERS)
def test_layers_are_refused(bad, code):
    lib, layer, p = B.lib(), _layer(**bad), C.c_void_p(0x40000)
    out = C.c_size_t(0)
    assert lib.lmk_gs_grouped_gated(C.byref(layer), p, 1 << 20, None, 0, p, 1 << 20, None) == code
    assert lib.lmk_gs_grouped_gated_backward_bytes(C.byref(layer), C.byref(out)) == code
    grads = B.GatedGrads(0x40000, 1 << 20, None, None)
    assert lib.lmk_gs_grouped_gated_backward(C.byref(layer), p, 1 << 20, p, 1 << 20, None, 0, C.byref(grads), p, 1 << 60, None) == code


def test_arguments_are_refused():
    lib, layer, p = B.lib(), _layer(), C.c_void_p(0x40000)
    call = lambda l=layer, x=p, ldx=16, b=None, act=0, y=p, ldy=8: lib.lmk_gs_grouped_gated(None if l is None else C.byref(l), x, ldx, b, act, y, ldy, None)
    for bad in (dict(l=None), dict(x=None), dict(x=C.c_void_p(0x40002)), dict(ldx=15), dict(ldx=(1 << 28) + 1), dict(y=None), dict(ldy=7), dict(act=3),
                dict(b=C.c_void_p(0x40002))):
        assert call(**bad) == B.ERR_INVALID, bad
    assert call(l=_layer(rows=0), x=None, y=None) == B.OK
    need = C.c_size_t(0)
    assert lib.lmk_gs_grouped_gated_backward_bytes(C.byref(layer), C.byref(need)) == B.OK and need.value > 0
    assert lib.lmk_gs_grouped_gated_backward_bytes(C.byref(layer), None) == B.ERR_INVALID
    full = dict(dx=0x70000, lddx=16, dw=0x80000, db=0x90000)

    def back(dy=p, lddy=8, x=p, ldx=16, b=None, act=0, out=full, ws=C.c_void_p(0x100000), size=need.value):
        g = None if out is None else C.byref(B.GatedGrads(out["dx"], out["lddx"], out["dw"], out["db"]))
        return lib.lmk_gs_grouped_gated_backward(C.byref(layer), dy, lddy, x, ldx, b, act, g, ws, size, None)

    for bad in (dict(dy=None), dict(lddy=7), dict(x=None), dict(ldx=15), dict(b=C.c_void_p(0x40001)), dict(act=3), dict(out=None),
                dict(out=dict(full, lddx=15)), dict(out=dict(full, dx=0x70001)), dict(out=dict(full, dw=0x80002)), dict(out=dict(full, db=0x90001)),
                dict(ws=None), dict(ws=C.c_void_p(0x100010))):
        assert back(**bad) == B.ERR_INVALID, bad
    assert back(size=need.value - 1) == B.ERR_CAPACITY
    assert back(out=dict(dx=None, lddx=0, dw=None, db=None)) == B.OK           # nothing to do


def test_binding_refuses_tensors_of_other_shapes():
    x, w, off, y = torch.zeros(10, 16), torch.zeros(3, 16, 16), torch.zeros(4, dtype=torch.int32), torch.zeros(10, 8)
    bad = [dict(x=torch.zeros(10, 17)), dict(x=x.double()), dict(w=torch.zeros(3, 15, 16)), dict(w=torch.zeros(3, 16, 32)[..., ::2]), dict(w=w.half()),
           dict(offsets=off.long()), dict(offsets=off[:3]), dict(out=torch.zeros(10, 16)), dict(out=torch.zeros(9, 8)), dict(out=y.bfloat16()),
           dict(bias=torch.zeros(3, 8)), dict(bias=torch.zeros(3, 16, dtype=torch.bfloat16)), dict(act="tanh"), dict()]
    for b in bad:                       # the last one for want of a GPU
        kw = dict(dict(x=x, w=w, offsets=off, out=y), **b)
        with pytest.raises(ValueError):
            B.grouped_gated(kw.pop("x"), kw.pop("w"), kw.pop("offsets"), kw.pop("out"), **kw)
    for b in (dict(dw=torch.zeros(3, 16, 15)), dict(dw=torch.zeros(3, 16, 16).bfloat16()), dict(db=torch.zeros(3, 8)), dict(dx=torch.zeros(10, 15)),
              dict(workspace=torch.zeros(10)), dict(bias=torch.zeros(2, 16)), dict(act="")):
        kw = dict(dict(workspace=None), **b)
        with pytest.raises(ValueError):
            B.grouped_gated_backward(y, x, w, off, kw.pop("workspace"), **kw)


def test_workspace_bytes_and_sizes_beyond_32_bits():
    a, b = B.grouped_gated_backward_bytes(1000, 4, 32, 35), B.grouped_gated_backward_bytes(300_000, 24, 32, 35, torch.bfloat16)
    assert 0 < a < b < 1 << 28 and b >= 300_000 * 64 * 2
    with pytest.raises(B.LmkGsError):
        B.grouped_gated_backward_bytes(1000, 0, 32, 35)
    for bad in ((1 << 32, 4, 32, 35), (1000, 1 << 32, 32, 35), (1000, 4, 1 << 31, 35), (1000, 4, 32, 1 << 32), (-1, 4, 32, 35)):
        with pytest.raises(ValueError):
            B.grouped_gated_backward_bytes(*bad)
