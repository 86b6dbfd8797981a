"""The 4-bit form and its layers without a GPU: the oracle against its definition, and
the calls' checks of their arguments."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import block4_ref as Q
from paper_2503_21364_amd import binding as B


def _values():
    rng = np.random.default_rng(1)
    x = (rng.normal(size=(60, 131)) * np.exp2(rng.integers(-120, 120, size=(60, 1)))).astype(np.float32)
    x[0] = 0
    x[1, ::2] = 0
    x[2, 0], x[3, 40], x[4, 130] = np.inf, -np.inf, np.nan
    x[5] = 1e-45                                                        # the least there is, below every step
    x[6], x[7] = np.float32(2.0 ** -126), np.float32(3.4e38)
    ties = np.concatenate([np.arange(0, 7.01, 0.25), [6.99, 5.01, 4.99]]).astype(np.float32)
    x[8, :32], x[9, :32] = np.resize(ties[ties < 7], 32), -np.resize(ties[ties < 7], 32)
    x[10, :32] = np.resize(np.array([7.0, 6.999999, 0.1, -0.0], np.float32), 32)
    return x


def test_forms_of_the_oracle_are_nearest_and_steps_least():
    x = _values()
    codes, scale = Q.pack(x)
    back = Q.unpack(codes, scale, 131)
    assert codes.shape == (60, 128) and scale.shape == (60, 16)
    fine = np.repeat(np.pad(scale, ((0, 0), (0, 0)))[:, :5], 32, axis=1)[:, :131] != 255
    assert np.isnan(back[~fine]).all() and (~fine).sum() == 32 + 32 + 3
    step = np.repeat(np.exp2(scale[:, :5].astype(np.float64) - 127), 32, axis=1)[:, :131]
    # no value is further off than half the distance to its neighbours: half a step up to 2, a whole one above (or to 7 from 6)
    q = np.abs(np.where(fine, x, 0).astype(np.float64)) / step
    off = np.abs(np.where(fine, back, 0) / step - np.where(fine, x, 0) / step)
    far = q >= 7                                                        # 3.4e38: the largest step there is, and 6 of it
    assert (off[~far] <= np.where(q <= 2, 0.25, np.where(q <= 4, 0.5, 1.0))[~far]).all()
    assert far.sum() == 131 and far[7].all() and (back[7] == 6 * 2.0 ** 125).all()
    top = np.abs(np.pad(np.where(fine, x, 0), ((0, 0), (0, 29)))).reshape(60, 5, 32).max(-1).astype(np.float64)
    least = (scale[:, :5] <= 1) | (scale[:, :5] >= 252)
    assert (least | (top / np.exp2(scale[:, :5].astype(np.float64) - 128) >= 7)).all()
    assert (np.signbit(back[fine]) == np.signbit(x[fine])).all()


@pytest.mark.parametrize("q,n", [(0.25, 0), (0.2500001, 1), (0.75, 2), (1.25, 2), (1.75, 4), (2.5, 4), (3.5, 6), (5.0, 6), (5.0001, 7), (6.99, 7)])
def test_ties_go_to_the_even_code(q, n):
    assert Q.number(q) == n


# ---- refusals (fake pointers: every call below has to be refused before it reaches them)
def test_form_arguments_are_refused():
    lib, p = B.lib(), C.c_void_p(0x40000)
    c = B.Block4C(0x50000, 0x60000)
    pack = lambda x=p, ldx=16, rows=4, k=16, dtype=0, out=c: lib.lmk_gs_block4_pack(x, ldx, rows, k, dtype, None if out is None else C.byref(out), None)
    unpack = lambda x=p, ldx=16, rows=4, k=16, dtype=0, out=c: lib.lmk_gs_block4_unpack(None if out is None else C.byref(out), rows, k, dtype, x, ldx, None)
    for f in (pack, unpack):
        for bad in (dict(x=None), dict(x=C.c_void_p(0x40001)), dict(ldx=15), dict(ldx=(1 << 28) + 1), dict(rows=1 << 31), dict(k=0), dict(k=65537, ldx=1 << 20),
                    dict(out=None), dict(out=B.Block4C(None, 0x60000)), dict(out=B.Block4C(0x50000, None)), dict(out=B.Block4C(0x50008, 0x60000)),
                    dict(out=B.Block4C(0x50000, 0x60008))):
            assert f(**bad) == B.ERR_INVALID, bad
        assert f(dtype=2) == B.ERR_UNSUPPORTED
        assert f(rows=(1 << 31) - 1, k=65536, ldx=65536) == B.ERR_UNSUPPORTED
        assert f(rows=0, x=None) == B.OK


def test_layer_arguments_are_refused():
    lib, p = B.lib(), C.c_void_p(0x40000)
    form = B.Block4C(0x50000, 0x60000)

    def call(x=form, b=None, relu=0, y=p, ldy=8, layer=True, **kw):
        d = dict(w=B.Block4C(0x10000, 0x20000), offsets=0x30000, blocks=3, rows=100, n=8, k=16, dtype=0)
        d.update(kw)
        l = B.Linear4C(*[d[f] for f, _ in B.Linear4C._fields_])
        return lib.lmk_gs_grouped_linear4(C.byref(l) if layer else None, None if x is None else C.byref(x), b, relu, y, ldy, None)

    for bad in (dict(layer=False), dict(blocks=0), dict(blocks=65537), dict(rows=1 << 31), dict(n=0), dict(n=65537), dict(k=0), dict(k=65537),
                dict(w=B.Block4C(None, 0x20000)), dict(w=B.Block4C(0x10000, None)), dict(w=B.Block4C(0x10008, 0x20000)), dict(w=B.Block4C(0x10000, 0x20004)),
                dict(offsets=None), dict(offsets=0x30002), dict(x=None), dict(x=B.Block4C(0x50004, 0x60000)), dict(x=B.Block4C(0x50000, 0x60002)),
                dict(b=C.c_void_p(0x40002)), dict(relu=2), dict(y=None), dict(y=C.c_void_p(0x40002)), dict(ldy=7), dict(ldy=(1 << 28) + 1)):
        assert call(**bad) == B.ERR_INVALID, bad
    assert call(dtype=2) == B.ERR_UNSUPPORTED
    assert call(rows=(1 << 31) - 1, n=65536, ldy=65536) == B.ERR_UNSUPPORTED
    assert call(rows=0, x=None, y=None) == B.OK


def test_binding_refuses_tensors_of_other_shapes():
    form = lambda rows, k: B.Block4(rows, k, "cpu")
    x, w, off, y = form(10, 16), form(24, 16), torch.zeros(4, dtype=torch.int32), torch.zeros(10, 8)
    for b in (dict(x=form(9, 16)), dict(x=form(10, 17)), dict(w=form(23, 16)), dict(w=form(24, 15)), dict(offsets=off.long()), dict(offsets=off[:3]),
              dict(out=torch.zeros(10, 9)), dict(out=y.double()), dict(out=torch.zeros(80)), dict(bias=torch.zeros(3, 9)), dict(bias=torch.zeros(24)), dict()):
        kw = dict(dict(x=x, w=w, offsets=off, out=y), **b)
        with pytest.raises(ValueError):
            B.grouped_linear4(kw.pop("x"), kw.pop("w"), kw.pop("offsets"), kw.pop("out"), **kw)
    for codes, scale in ((torch.zeros(4, 64, dtype=torch.int8), None), (torch.zeros(4, 63, dtype=torch.uint8), None),
                         (torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 1, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            B.Block4(4, 16, codes=codes, scale=scale)
    for f in (lambda t: B.block4_pack(t, form(4, 16)), lambda t: B.block4_unpack(form(4, 16), t)):
        for t in (torch.zeros(4, 17), torch.zeros(4, 16).half(), torch.zeros(4, 16)):
            with pytest.raises(ValueError):
                f(t)
    with pytest.raises(ValueError, match="2\\^32"):
        B.Block4(1 << 32, 16, "meta")
