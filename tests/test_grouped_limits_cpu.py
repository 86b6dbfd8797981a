"""Which sizes the grouped layers' calls refuse because they do not fit a launch, without a GPU: every call below is refused, or
has no rows and so nothing to launch."""
import ctypes as C

import pytest
import torch

from paper_2503_21364_amd import binding as B

P = C.c_void_p(0x40000)
KEPT = B.Checkpoint8C(0x50000, 0x60000)


def _layer(rows, blocks, k, n, dtype=0, w_block=None):
    return B.LinearC(0x10000, 0x20000, k, k * n if w_block is None else w_block, blocks, rows, n, k, dtype, 0)


def _forward(layer, keep=False):
    return B.lib().lmk_gs_grouped_linear(C.byref(layer), P, layer.k, None, 0, P, layer.n, C.byref(KEPT) if keep else None, None)


def _backward(layer, dx=True, sums=False, kept=True):
    grads = B.LinearGrads(0x70000 if dx else None, layer.k, 0x80000 if sums else None, 0x90000 if sums else None)
    return B.lib().lmk_gs_grouped_linear_backward(C.byref(layer), P, layer.n, None, 0, C.byref(KEPT) if kept else None, 0, C.byref(grads),
                                                  C.c_void_p(0x100000), C.c_size_t((1 << 64) - 1), None)


def _bytes(layer):
    out = C.c_size_t(0)
    return B.lib().lmk_gs_grouped_linear_backward_bytes(C.byref(layer), C.byref(out))


def test_a_product_of_rows_is_not_refused_for_the_sums_that_it_does_not_take():
    # 256 matrices of 65536 x 65536 are too many sums to join; y and dx are not summed over rows
    layer = _layer(0, 256, 65536, 65536, dtype=1)
    assert _bytes(layer) == B.ERR_UNSUPPORTED and _backward(layer, sums=True) == B.ERR_UNSUPPORTED
    assert _forward(layer) == B.OK and _backward(layer) == B.OK


# ---- a launch holds fewer than 2^32 threads in a dimension
ROWS = (1 << 31) - 1


def test_products_of_more_rows_than_a_launch_holds():
    small = dict(blocks=1, k=1, n=1)                            # tiles of 64 rows, 256 threads each
    for layer in (_layer((1 << 30) + 1, **small), _layer(ROWS, **small), _layer(ROWS, 3, 8, 8, dtype=1), _layer(ROWS, 1, 256, 136)):
        assert _forward(layer) == B.ERR_UNSUPPORTED
        assert _backward(layer) == B.ERR_UNSUPPORTED
        assert _bytes(layer) == B.ERR_UNSUPPORTED


def test_an_8_bit_form_of_more_values_than_a_launch_holds():
    # the general kernel does not write it on the way: 2^32 values of four a thread, and the product itself would fit
    rows = 1 << 29
    assert _forward(_layer(rows, 1, 129, 1), keep=True) == B.ERR_UNSUPPORTED
    lib = B.lib()
    assert lib.lmk_gs_checkpoint8_pack(P, 32, ROWS, 32, 0, C.byref(KEPT), None) == B.ERR_UNSUPPORTED
    assert lib.lmk_gs_checkpoint8_unpack(C.byref(KEPT), ROWS, 32, 0, P, 32, None) == B.ERR_UNSUPPORTED


def test_more_sums_to_join_than_a_launch_holds():
    # 2^34 of them, 1024 a workgroup; refused before dx is queued
    layer = _layer(0, 257, 8192, 8192, dtype=1)
    assert _bytes(layer) == B.ERR_UNSUPPORTED
    assert _backward(layer, sums=True) == B.ERR_UNSUPPORTED
    assert _forward(layer) == B.OK and _backward(layer) == B.OK
    assert _bytes(_layer(0, 255, 8192, 8192, dtype=1)) == B.OK


# ---- sizes that 32-bit fields would cut off
def test_sizes_beyond_32_bits_are_refused_and_not_cut_off():
    big = (1 << 32) + 5
    for bad in ((big, 4, 96, 35), (1000, big, 96, 35), (1000, 4, big, 35), (1000, 4, 96, big), (-1, 4, 96, 35)):
        with pytest.raises((ValueError, B.LmkGsError)):
            B.grouped_linear_backward_bytes(*bad)
    with pytest.raises(ValueError, match="2\\^32"):
        B.Checkpoint8(big, 16, "meta")
    meta = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device="meta")
    with pytest.raises(ValueError, match="2\\^32"):
        B.grouped_linear(meta(big, 16), meta(3, 8, 16), meta(4, dtype=torch.int32), meta(big, 8))
    with pytest.raises(ValueError, match="2\\^32"):
        B.grouped_linear_backward(meta(big, 8), meta(3, 8, 16), meta(4, dtype=torch.int32), dx=meta(big, 16))
    with pytest.raises(ValueError, match="2\\^32"):
        B.grouped_linear(meta(10, 16), meta(big, 8, 16), meta(big + 1, dtype=torch.int32), meta(10, 8))
