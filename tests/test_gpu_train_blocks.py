"""The example that trains an anchor decoder in blocks: its gradients against torch's for the same step, and that the error falls.

The example's backward pass reads the layers' inputs from 8 bits: their values are off by 1/127.5 of the largest of 32, at
most, and a gradient of a weight is a sum over anchors of products with them; a gradient's relative error in the 2-norm is
therefore bounded by about 1/127.5 times sqrt(32) (where one of 32 values is large and the others are not), 0.045, and is
far below for values of like size."""
import os
import sys

import pytest
import torch

from paper_2503_21364_amd import binding as B

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def _trainer(**kw):
    import train_blocks
    return train_blocks, train_blocks.Trainer(**kw)


def test_gradients_of_a_step_are_those_of_the_same_step_in_torch():
    T, t = _trainer(anchors=3000, blocks=5, k=4, width=160, height=96)
    before = [p.clone() for p in t.net.tensors()]
    t.step(0)
    torch.cuda.synchronize()
    D, status = B.read_status(t.frame)
    assert status == B.OK and D > 1000
    w1, b1, *rest = [p.double().requires_grad_(True) for p in before]
    w2, b2 = rest[:3], rest[3:]
    d = t.position - t.eyes[0][:, None]
    x = torch.cat([t.feature, (d / d.norm(dim=0, keepdim=True)).T], dim=1).double()
    edge = t.blocks.tolist()
    y = [[], [], []]
    for g, (a, b) in enumerate(zip(edge, edge[1:])):
        h = torch.relu(x[a:b] @ w1[g].T + b1[g])
        for m in range(3):
            y[m].append(h[:, m * T.F:(m + 1) * T.F] @ w2[m][g] + b2[m][g])
    attributes = t._combine(*[torch.cat(v) for v in y])
    torch.autograd.backward(list(attributes.values()), [getattr(t.scene_grads, n).double() for n in attributes])
    for name, want, got in zip(["w1", "b1", "w2", "w2", "w2", "b2", "b2", "b2"], [w1, b1, *w2, *b2], t.grads):
        off = float((got.double() - want.grad).norm() / want.grad.norm())
        assert off < 0.045, (name, off)


def test_error_falls():
    _, t = _trainer(anchors=4000, blocks=6, k=4, width=160, height=96)
    errors = [float(t.step(i % 4)) for i in range(24)]
    assert sum(errors[-4:]) < 0.7 * sum(errors[:4]), errors
