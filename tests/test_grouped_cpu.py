"""Grouped perceptron layers without a GPU: the oracle against its own definition (differences, closed forms), and the
calls' checks of their arguments, which refuse before anything is launched."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import grouped_ref as G
from paper_2503_21364_amd import binding as B


def test_gradients_of_the_oracle_are_those_of_its_forward_pass():
    # loss = sum(y * up): bilinear in (x, w), so central differences are exact up to rounding
    rng = np.random.default_rng(5)
    offsets, rows, n, k = [1, 4, 4, 9], 10, 5, 7
    x, w, b = rng.normal(size=(rows, k)), rng.normal(size=(3, n, k)), rng.normal(size=(3, n))
    up = rng.normal(size=(rows, n))
    (dx, dw, db), _ = G.backward(up, x, w, offsets)
    loss = lambda x_, w_, b_: (G.forward(x_, w_, offsets, b_)[0] * up).sum()
    for _ in range(4):
        ex, ew, eb = rng.normal(size=x.shape), rng.normal(size=w.shape), rng.normal(size=b.shape)
        h = 1e-3
        diff = lambda f: (f(h) - f(-h)) / (2 * h)
        assert abs(diff(lambda t: loss(x + t * ex, w, b)) - (dx * ex).sum()) < 1e-9
        assert abs(diff(lambda t: loss(x, w + t * ew, b)) - (dw * ew).sum()) < 1e-9
        assert abs(diff(lambda t: loss(x, w, b + t * eb)) - (db * eb).sum()) < 1e-9


def test_gate_of_the_oracle_is_the_gradient_through_a_relu():
    rng = np.random.default_rng(6)
    offsets, w = [0, 6], rng.normal(size=(1, 4, 5))
    pre, up = rng.normal(size=(6, 5)), rng.normal(size=(6, 4))
    x = np.maximum(pre, 0)
    (dx, _, _), _ = G.backward(up, x, w, offsets, gate=True)
    e, h = rng.normal(size=pre.shape), 1e-7
    loss = lambda t: (G.forward(np.maximum(pre + t * e, 0), w, offsets)[0] * up).sum()
    assert abs((loss(h) - loss(-h)) / (2 * h) - (dx * e).sum()) < 1e-6


def test_rows_of_no_block_and_empty_blocks_of_the_oracle():
    x, w = np.ones((6, 2)), np.ones((3, 3, 2))
    y, _ = G.forward(x, w, [1, 3, 3, 5], bias=np.ones((3, 3)))
    assert (y[[0, 5]] == 0).all() and (y[1:5] == 3).all()
    (dx, dw, db), _ = G.backward(np.ones((6, 3)), x, w, [1, 3, 3, 5])
    assert (dx[[0, 5]] == 0).all() and (dw[1] == 0).all() and (db[1] == 0).all() and (db[0] == 2).all()


@pytest.mark.parametrize("top,code,e", [(1.0, 64, -6), (127.0, 127, 0), (127.5, 64, 1), (127.25, 127, 0), (0.75, 96, -7)])
def test_scale_of_the_oracle(top, code, e):
    codes, scale = G.pack(np.array([[top, -top, 0.0, 1e-30, -1e-30]]))
    assert codes[0, :5].tolist() == [code, -code, 0, 1, -1] and scale[0, 0] == e + 127


def test_codes_of_the_oracle_are_within_half_a_step_and_keep_signs():
    rng = np.random.default_rng(7)
    x = (rng.normal(size=(50, 70)) * np.exp2(rng.integers(-60, 60, size=(50, 1)))).astype(np.float32)
    codes, scale = G.pack(x)
    back = G.unpack(codes, scale, 70)
    step = np.repeat(np.exp2(scale.astype(np.float64) - 127), 32, axis=1)[:, :70]
    assert (np.sign(back) == np.sign(x)).all()
    assert (np.abs(back - x) <= np.where(np.abs(x) < step / 2, step, step / 2)).all()
    top = np.abs(np.pad(x, ((0, 0), (0, 26)))).reshape(50, 3, 32).max(-1).astype(np.float64)
    assert (np.exp2(scale.astype(np.float64) - 127) <= top / 63.75).all()


# ---- refusals (fake pointers: every call below has to be refused before it reaches them)
def _layer(**kw):
    d = dict(w=0x10000, offsets=0x20000, ldw=16, w_block=8 * 16, blocks=3, rows=100, n=8, k=16, dtype=0, in_major=0)
    d.update(kw)
    return B.LinearC(*[d[f] for f, _ in B.LinearC._fields_])


BAD_LAYERS = [
    (dict(dtype=2), B.ERR_UNSUPPORTED), (dict(in_major=2), B.ERR_INVALID), (dict(blocks=0), B.ERR_INVALID),
    (dict(blocks=65537), B.ERR_INVALID), (dict(rows=1 << 31), B.ERR_INVALID), (dict(n=0), B.ERR_INVALID), (dict(k=0), B.ERR_INVALID),
    (dict(n=65537), B.ERR_INVALID), (dict(k=65537, ldw=65537, w_block=1 << 30), B.ERR_INVALID), (dict(ldw=15), B.ERR_INVALID),
    (dict(in_major=1, ldw=7), B.ERR_INVALID), (dict(ldw=(1 << 28) + 1, w_block=1 << 40), B.ERR_INVALID), (dict(w_block=127), B.ERR_INVALID),
    (dict(w_block=(1 << 40) + 1), B.ERR_INVALID), (dict(w=None), B.ERR_INVALID), (dict(w=0x10002), B.ERR_INVALID),
    (dict(offsets=None), B.ERR_INVALID), (dict(offsets=0x20002), B.ERR_INVALID),
    (dict(rows=(1 << 31) - 1, n=65536, w_block=1 << 20), B.ERR_UNSUPPORTED),
]


@pytest.mark.parametrize("bad,code", BAD_LAYERS)
def test_layers_are_refused(bad, code):
    lib, layer, p = B.lib(), _layer(**bad), C.c_void_p(0x40000)
    out = C.c_size_t(0)
    assert lib.lmk_gs_grouped_linear(C.byref(layer), p, 1 << 20, None, 0, p, 1 << 20, None, None) == code
    assert lib.lmk_gs_grouped_linear_backward_bytes(C.byref(layer), C.byref(out)) == code
    grads = B.LinearGrads(0x40000, 1 << 20, None, None)
    assert lib.lmk_gs_grouped_linear_backward(C.byref(layer), p, 1 << 20, p, 1 << 20, None, 0, C.byref(grads), None, 0, None) == code


def test_forward_arguments_are_refused():
    lib, layer, p = B.lib(), _layer(), C.c_void_p(0x40000)
    kept = B.Checkpoint8C(0x50000, 0x60000)
    call = lambda l=layer, x=p, ldx=16, b=None, relu=0, y=p, ldy=8, keep=None: lib.lmk_gs_grouped_linear(
        None if l is None else C.byref(l), x, ldx, b, relu, y, ldy, None if keep is None else C.byref(keep), None)
    for bad in (dict(l=None), dict(x=None), dict(x=C.c_void_p(0x40002)), dict(ldx=15), dict(ldx=(1 << 28) + 1), dict(y=None),
                dict(ldy=7), dict(relu=2), dict(b=C.c_void_p(0x40002)), dict(keep=B.Checkpoint8C(None, 0x60000)),
                dict(keep=B.Checkpoint8C(0x50000, None)), dict(keep=B.Checkpoint8C(0x50008, 0x60000))):
        assert call(**bad) == B.ERR_INVALID, bad
    empty = _layer(rows=0)
    assert call(l=empty, x=None, y=None, keep=kept) == B.OK          # nothing to do


def test_backward_arguments_are_refused():
    lib, layer, p = B.lib(), _layer(), C.c_void_p(0x40000)
    kept = B.Checkpoint8C(0x50000, 0x60000)
    need = C.c_size_t(0)
    assert lib.lmk_gs_grouped_linear_backward_bytes(C.byref(layer), C.byref(need)) == B.OK and need.value > 0
    assert lib.lmk_gs_grouped_linear_backward_bytes(C.byref(layer), None) == B.ERR_INVALID
    full = dict(dx=0x70000, lddx=16, dw=0x80000, db=0x90000)

    def call(dy=p, lddy=8, x=None, ldx=0, kept_=kept, gate=0, out=full, ws=C.c_void_p(0x100000), size=need.value):
        g = None if out is None else C.byref(B.LinearGrads(out["dx"], out["lddx"], out["dw"], out["db"]))
        return lib.lmk_gs_grouped_linear_backward(C.byref(layer), dy, lddy, x, ldx, None if kept_ is None else C.byref(kept_), gate, g,
                                                  ws, size, None)

    for bad in (dict(dy=None), dict(lddy=7), dict(out=None), dict(gate=2), dict(x=p, ldx=16), dict(kept_=None),
                dict(kept_=None, x=p, ldx=15), dict(kept_=B.Checkpoint8C(0x50000, None)), dict(out=dict(full, lddx=15)),
                dict(out=dict(full, dw=0x80002)), dict(out=dict(full, db=0x90001)), dict(ws=None), dict(ws=C.c_void_p(0x100010)),
                dict(kept_=None, gate=1, out=dict(full, dw=None, db=None))):
        assert call(**bad) == B.ERR_INVALID, bad
    assert call(size=need.value - 1) == B.ERR_CAPACITY


def test_checkpoint_arguments_are_refused():
    lib, p = B.lib(), C.c_void_p(0x40000)
    c = B.Checkpoint8C(0x50000, 0x60000)
    pack = lambda x=p, ldx=16, rows=4, k=16, dtype=0, out=c: lib.lmk_gs_checkpoint8_pack(
        x, ldx, rows, k, dtype, None if out is None else C.byref(out), None)
    unpack = lambda x=p, ldx=16, rows=4, k=16, dtype=0, out=c: lib.lmk_gs_checkpoint8_unpack(
        None if out is None else C.byref(out), rows, k, dtype, x, ldx, None)
    for f in (pack, unpack):
        for bad in (dict(x=None), dict(x=C.c_void_p(0x40001)), dict(ldx=15), dict(rows=1 << 31), dict(k=0), dict(k=65537, ldx=1 << 20),
                    dict(out=None), dict(out=B.Checkpoint8C(None, 1)), dict(out=B.Checkpoint8C(0x50004, 0x60000))):
            assert f(**bad) == B.ERR_INVALID, bad
        assert f(dtype=2) == B.ERR_UNSUPPORTED
        assert f(rows=(1 << 31) - 1, k=65536, ldx=65536) == B.ERR_UNSUPPORTED
        assert f(rows=0, x=None) == B.OK


def test_binding_refuses_tensors_of_other_shapes():
    x, w, off, y = torch.zeros(10, 16), torch.zeros(3, 8, 16), torch.zeros(4, dtype=torch.int32), torch.zeros(10, 8)
    bad = [
        dict(x=torch.zeros(10, 17)), dict(x=x.double()), dict(x=x.t().contiguous().t()), dict(w=torch.zeros(8, 16)),
        dict(w=torch.zeros(3, 16, 8).transpose(1, 2)), dict(w=w.half()), dict(offsets=off.long()), dict(offsets=off[:3]),
        dict(out=torch.zeros(10, 9)), dict(out=torch.zeros(9, 8)), dict(out=y.bfloat16()), dict(bias=torch.zeros(3, 9)),
        dict(bias=torch.zeros(3, 8, dtype=torch.bfloat16)), dict(checkpoint=B.Checkpoint8(10, 15, "cpu")),
    ]
    for b in bad:
        kw = dict(dict(x=x, w=w, offsets=off, out=y), **b)
        with pytest.raises(ValueError):
            B.grouped_linear(kw.pop("x"), kw.pop("w"), kw.pop("offsets"), kw.pop("out"), **kw)
    dy = torch.zeros(10, 8)
    for b in (dict(dw=torch.zeros(3, 16, 8)), dict(db=torch.zeros(3, 16)), dict(dx=torch.zeros(10, 15)), dict(x=torch.zeros(9, 16)),
              dict(workspace=torch.zeros(10)), dict(dw=torch.zeros(3, 8, 32)[..., ::2]), dict(checkpoint=B.Checkpoint8(9, 16, "cpu"))):
        with pytest.raises(ValueError):
            B.grouped_linear_backward(dy, w, off, **b)
    with pytest.raises(ValueError):
        B.Checkpoint8(4, 16, codes=torch.zeros(4, 16, dtype=torch.int8), scale=torch.zeros(4, 1, dtype=torch.uint8))
    with pytest.raises(ValueError):
        B.checkpoint8_pack(torch.zeros(4, 17), B.Checkpoint8(4, 16, "cpu"))


def test_workspace_bytes_cover_the_sizes():
    a = B.grouped_linear_backward_bytes(1000, 4, 96, 35)
    b = B.grouped_linear_backward_bytes(300_000, 24, 96, 35)
    assert 0 < a < b < 1 << 28
    with pytest.raises(B.LmkGsError):
        B.grouped_linear_backward_bytes(1000, 0, 96, 35)
