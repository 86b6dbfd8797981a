"""Grouped layers with an infinity or a NaN among the weights: it reaches the results that are summed over it and no others, whichever
kernel the sizes choose.  Bounds as in test_gpu_grouped.py; what is not finite is equal."""
import numpy as np
import pytest
import torch

from oracle import grouped_ref as G
from test_gpu_grouped import Layer, _np

pytestmark = pytest.mark.gpu


def _plant(t, block, out, inp, value):
    t.w64[block, out, inp] = value
    t.w[(block, inp, out) if t.in_major else (block, out, inp)] = value


# Sums of every length modulo the four and the sixteen indices that the kernels take at a time, in small matrices; then
# the bfloat16 kernels' aligned and unaligned sizes, and one that only the general kernel takes.  The infinities are among the last indices of a sum,
# where the kernels go past its end.
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("in_major", [False, True])
@pytest.mark.parametrize("k,n", [(32, 70), (35, 96), (33, 4), (64, 5), (18, 9), (7, 23), (50, 66), (13, 81), (64, 64), (136, 264), (131, 257), (6, 300)])
def test_weights_that_are_not_finite(k, n, in_major, dtype):
    t = Layer([650, 130, 40], k, n, dtype, in_major, seed=n)
    _plant(t, 0, n - 1, 1, np.inf)
    _plant(t, 0, n - 2, k - 1, -np.inf)
    _plant(t, 1, n - 1, 0, -np.inf)
    _plant(t, 1, 0, k - 1, np.inf)
    _plant(t, 1, n - 1, k - 2, np.nan)
    assert np.isinf(G.backward(_np(t.dy), _np(t.x), t.w64, t.offsets)[0][0]).sum() == 2 * 650 + 2 * 130
    for keep in (None, t.kept()):
        t.forward(keep=keep)
        t.check_forward()
        t.forward(relu=True, keep=keep)
        t.check_forward(relu=True)
    for which in (("dx", "dw", "db"), ("dx",)):
        t.backward(which=which)
        t.check_backward(which=which)
        t.backward(gate=True, which=which)
        t.check_backward(gate=True, which=which)
    x64 = G.unpack(keep.codes.cpu().numpy(), keep.scale.cpu().numpy(), k)
    t.backward(keep, gate=True)
    t.check_backward(x64, gate=True)
    assert torch.isfinite(t.dw).all() and torch.isfinite(t.dx[780:]).all()
