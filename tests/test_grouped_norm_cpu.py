"""Layer norms of blocks without a GPU: the oracle against its definition, and the calls' checks of their arguments, which refuse
before anything is launched."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import norm_ref as N
from paper_2503_21364_amd import binding as B


def test_rows_of_the_oracle_have_level_and_spread_of_shift_and_gain():
    rng = np.random.default_rng(1)
    x = 5 + 3 * rng.normal(size=(7, 50))
    y, _ = N.forward(x, [1, 3, 3, 6], gain=np.full((3, 50), 2.0), shift=np.full((3, 50), -1.0), eps=1e-12)
    assert (y[[0, 6]] == 0).all()
    np.testing.assert_allclose(y[1:6].mean(1), -1, atol=1e-12)
    np.testing.assert_allclose(y[1:6].std(1), 2, rtol=1e-9)


def test_gradients_of_the_oracle_are_differences():
    rng = np.random.default_rng(2)
    offsets, rows, k = [1, 4, 4, 9], 10, 6
    x, gain, shift, up = rng.normal(size=(rows, k)), rng.normal(size=(3, k)), rng.normal(size=(3, k)), rng.normal(size=(rows, k))
    (dx, dgain, dshift), _ = N.backward(up, x, offsets, gain, eps=0.1)
    loss = lambda x_, g_, s_: (N.forward(x_, offsets, g_, s_, eps=0.1)[0] * up).sum()
    h = 1e-5
    for _ in range(5):
        ex, eg, es = rng.normal(size=x.shape), rng.normal(size=gain.shape), rng.normal(size=shift.shape)
        diff = lambda f: (f(h) - f(-h)) / (2 * h)
        assert abs(diff(lambda t: loss(x + t * ex, gain, shift)) - (dx * ex).sum()) < 1e-8
        assert abs(diff(lambda t: loss(x, gain + t * eg, shift)) - (dgain * eg).sum()) < 1e-8
        assert abs(diff(lambda t: loss(x, gain, shift + t * es)) - (dshift * es).sum()) < 1e-8


def test_bounds_of_the_oracle_hold_for_32_bits_in_numpy():
    rng = np.random.default_rng(3)
    for level in (0.0, 100.0):
        x, dy = (level + rng.normal(size=(20, 96))).astype(np.float32), rng.normal(size=(20, 96)).astype(np.float32)
        y, bound = N.forward(x, [0, 20], eps=1e-5)
        c = x - x.mean(1, keepdims=True, dtype=np.float32)
        s = 1 / np.sqrt((c * c).mean(1, keepdims=True, dtype=np.float32) + np.float32(1e-5))
        assert (np.abs(c * s - y) <= bound).all()
        (dx, _, _), (ex, _, _) = N.backward(dy, x, [0, 20], eps=1e-5)
        h = c * s
        got = s * (dy - dy.mean(1, keepdims=True) - h * (dy * h).mean(1, keepdims=True))
        assert (np.abs(got - dx) <= ex).all()


# ---- refusals (fake pointers: every call below has to be refused before it reaches them)
def _norm(**kw):
    d = dict(gain=0x10000, shift=0x20000, offsets=0x30000, blocks=3, rows=100, k=16, dtype=0, eps=1e-5)
    d.update(kw)
    return B.NormC(*[d[f] for f, _ in B.NormC._fields_])


BAD = [(dict(dtype=2), B.ERR_UNSUPPORTED), (dict(blocks=0), B.ERR_INVALID), (dict(blocks=65537), B.ERR_INVALID), (dict(rows=1 << 31), B.ERR_INVALID),
       (dict(k=0), B.ERR_INVALID), (dict(k=65537), B.ERR_INVALID), (dict(offsets=None), B.ERR_INVALID), (dict(offsets=0x30002), B.ERR_INVALID),
       (dict(gain=0x10002), B.ERR_INVALID), (dict(shift=0x20001), B.ERR_INVALID), (dict(eps=0.0), B.ERR_INVALID), (dict(eps=-1.0), B.ERR_INVALID),
       (dict(eps=float("nan")), B.ERR_INVALID), (dict(eps=float("inf")), B.ERR_INVALID), (dict(rows=(1 << 31) - 1, k=65536), B.ERR_UNSUPPORTED)]


@pytest.mark.parametrize("bad,code", BAD)
def test_norms_are_refused(bad, code):
    lib, norm, p = B.lib(), _norm(**bad), C.c_void_p(0x40000)
    out, grads = C.c_size_t(0), B.NormGrads(0x50000, 1 << 20, None, None)
    assert lib.lmk_gs_grouped_norm(C.byref(norm), p, 1 << 20, p, 1 << 20, None) == code
    assert lib.lmk_gs_grouped_norm_backward_bytes(C.byref(norm), C.byref(out)) == code
    assert lib.lmk_gs_grouped_norm_backward(C.byref(norm), p, 1 << 20, p, 1 << 20, C.byref(grads), None, 0, None) == code


def test_arguments_are_refused():
    lib, norm, p = B.lib(), _norm(), C.c_void_p(0x40000)
    call = lambda n=norm, x=p, ldx=16, y=p, ldy=16: lib.lmk_gs_grouped_norm(None if n is None else C.byref(n), x, ldx, y, ldy, None)
    for bad in (dict(n=None), dict(x=None), dict(x=C.c_void_p(0x40002)), dict(ldx=15), dict(ldx=(1 << 28) + 1), dict(y=None),
                dict(y=C.c_void_p(0x40001)), dict(ldy=15)):
        assert call(**bad) == B.ERR_INVALID, bad
    assert call(n=_norm(rows=0), x=None, y=None) == B.OK
    need = C.c_size_t(0)
    assert lib.lmk_gs_grouped_norm_backward_bytes(C.byref(norm), C.byref(need)) == B.OK and need.value > 0
    assert lib.lmk_gs_grouped_norm_backward_bytes(C.byref(norm), None) == B.ERR_INVALID
    full = dict(dx=0x70000, lddx=16, dgain=0x80000, dshift=0x90000)

    def back(n=norm, dy=p, lddy=16, x=p, ldx=16, out=full, ws=C.c_void_p(0x100000), size=need.value):
        g = None if out is None else C.byref(B.NormGrads(out["dx"], out["lddx"], out["dgain"], out["dshift"]))
        return lib.lmk_gs_grouped_norm_backward(None if n is None else C.byref(n), dy, lddy, x, ldx, g, ws, size, None)

    for bad in (dict(n=None), dict(dy=None), dict(lddy=15), dict(x=None), dict(ldx=15), dict(out=None), dict(out=dict(full, lddx=15)),
                dict(out=dict(full, dx=0x70002)), dict(out=dict(full, dgain=0x80002)), dict(out=dict(full, dshift=0x90001)), dict(ws=None),
                dict(ws=C.c_void_p(0x100080))):
        assert back(**bad) == B.ERR_INVALID, bad
    assert back(size=need.value - 1) == B.ERR_CAPACITY
    assert back(out=dict(dx=None, lddx=0, dgain=None, dshift=None), ws=None, size=0) == B.OK          # nothing to do
    assert back(n=_norm(rows=0), out=dict(full, dgain=None, dshift=None), dy=None, x=None, ws=None, size=0) == B.OK


def test_binding_refuses_tensors_of_other_shapes():
    x, off = torch.zeros(10, 16), torch.zeros(4, dtype=torch.int32)
    good = dict(x=x, offsets=off, out=torch.zeros(10, 16))
    bad = [dict(x=x.double()), dict(x=x[0]), dict(x=x.t().contiguous().t()), dict(offsets=off.long()), dict(offsets=off[:1]),
           dict(offsets=off[::2]), dict(out=torch.zeros(10, 17)), dict(out=torch.zeros(10, 16).bfloat16()), dict(gain=torch.zeros(3, 15)),
           dict(gain=torch.zeros(2, 16)), dict(shift=torch.zeros(3, 16).bfloat16()), dict(shift=torch.zeros(3, 32)[:, ::2]), dict()]
    for b in bad:                       # the last one for want of a GPU
        kw = dict(good, **b)
        with pytest.raises(ValueError):
            B.grouped_norm(kw.pop("x"), kw.pop("offsets"), kw.pop("out"), **kw)
    for b in (dict(dx=torch.zeros(10, 15)), dict(dgain=torch.zeros(3, 15)), dict(dshift=torch.zeros(4, 16)), dict(workspace=torch.zeros(10)),
              dict(gain=torch.zeros(3, 17))):
        with pytest.raises(ValueError):
            B.grouped_norm_backward(x, x, off, **b)
    with pytest.raises(ValueError):
        B.grouped_norm_backward(torch.zeros(9, 16), x, off)


def test_workspace_bytes_and_sizes_beyond_32_bits():
    a, b = B.grouped_norm_backward_bytes(1000, 4, 96), B.grouped_norm_backward_bytes(300_000, 24, 96, torch.bfloat16)
    assert 0 < a < b < 1 << 26
    with pytest.raises(B.LmkGsError):
        B.grouped_norm_backward_bytes(1000, 0, 96)
    for bad in ((1 << 32, 4, 96), (1000, 1 << 32, 96), (1000, 4, (1 << 32) + 1), (-1, 4, 96)):
        with pytest.raises(ValueError):
            B.grouped_norm_backward_bytes(*bad)


def test_in_every_size_the_sets_of_partial_sums_fit_the_workspace():
    # set g + (first row of g) / per + run: at most rows / per + blocks of them, whatever `per` is
    for rows in (0, 1, 7, 300, 4097, 300_000):
        for k in (1, 96, 1024, 5000, 20_000, 65_536):
            for blocks in (1, 3, 300):
                assert B.grouped_norm_backward_bytes(rows, blocks, k) >= (blocks + 1) * 2 * k * 4


def test_tensors_of_another_device_than_the_current_one_are_refused(monkeypatch):
    class Somewhere:                    # a tensor on the second GPU, as far as the check looks
        device = torch.device("cuda", 1)
        get_device = lambda self: 1

    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    with pytest.raises(ValueError, match="current device"):
        B._stream_on(Somewhere(), None)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1, raising=False)

    class Other:
        device = torch.device("cuda", 0)
        cuda_stream = 1

    with pytest.raises(ValueError, match="stream"):
        B._stream_on(Somewhere(), Other())


@pytest.mark.parametrize("bytes_of", [lambda t: B.grouped_linear_backward_bytes(10, 2, 8, 8, t), lambda t: B.grouped_norm_backward_bytes(10, 2, 8, t),
                                      lambda t: B.grouped_gated_backward_bytes(10, 2, 8, 8, t)])
def test_a_workspace_of_another_type_is_refused_as_the_calls_refuse_it(bytes_of):
    assert bytes_of(torch.float32) > 0 and bytes_of(torch.bfloat16) > 0
    for dtype in (torch.float16, torch.float64, None):
        with pytest.raises(ValueError, match="float32 or bfloat16"):
            bytes_of(dtype)
