"""Which sizes the grouped layers' calls refuse because they do not fit a launch, without a GPU: every call below is refused, or
has no rows and so nothing to launch."""
import ctypes as C

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
