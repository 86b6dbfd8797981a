"""The comparison on whole numbers, without a GPU: it is exact in 32 bits, agrees with the oracle, and shows one row too few."""
import numpy as np
import pytest

import grouped_exact as E
from oracle import grouped_ref as G


@pytest.mark.parametrize("sizes,k,n", [s[:3] for s in E.LONG])
def test_one_row_left_out_shows_in_every_long_block(sizes, k, n):
    t = E.Numbers(sizes, k, n, front=2, behind=3, seed=1)
    assert max(sizes) * 4 < 1 << 24
    _, dw, db = t.backward()
    rng = np.random.default_rng(2)
    for a, b in zip(t.offsets, t.offsets[1:]):
        if a == b:
            continue
        _, dw1, db1 = t.backward(without=int(rng.integers(a, b)))
        with pytest.raises(AssertionError):
            E.same(dw1, dw, "dw")
        with pytest.raises(AssertionError):
            E.same(db1, db, "db")
        if len(sizes) > 8:
            break


@pytest.mark.parametrize("sizes,k,n", [([3, 0, 40], 35, 70), ([500, 1], 8, 5)])
def test_whole_numbers_agree_with_the_oracle(sizes, k, n):
    t = E.Numbers(sizes, k, n, front=2, behind=3)
    E.same(t.forward(), G.forward(t.x, t.w, t.offsets, t.b)[0], "y")
    E.same(t.forward(relu=True), G.forward(t.x, t.w, t.offsets, t.b, relu=True)[0], "y")
    for gate in (False, True):
        for got, want in zip(t.backward(gate), G.backward(t.dy, t.x, t.w, t.offsets, gate)[0]):
            E.same(got, want, "gradient")
    codes, scale = G.pack(t.x)
    E.same(G.unpack(codes, scale, k), t.x, "8-bit form")
