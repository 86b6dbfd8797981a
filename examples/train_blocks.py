"""Trains the anchor decoder of a scene in blocks, every block with perceptrons of its own.

    python examples/train_blocks.py [--anchors 20000] [--blocks 8] [--steps 20]

The anchors are put into voxel order and cut into blocks of consecutive anchors.  A step decodes them for one
viewpoint, renders, and takes the gradient of the squared error against a target image (the scene as one
decoder shared by all blocks renders it) back to the weights of every block:

    x = [feature, direction]        grouped_linear, 35 -> 3 x 32, ReLU; x is kept in 8 bits
    h = three times 32 units        grouped_linear for each perceptron's third of the columns; h is kept in 8 bits,
                                    and is not needed any more
    activations, combination        a few tensor operations (their gradients are torch's)
    image                           preprocess, bin_sort, render
    gradients                       render_backward, preprocess_backward, those of the activations, then
                                    grouped_linear_backward of the second layers (through the ReLU, from the kept
                                    form of h) and of the first ones (from the kept form of x)
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2503_21364_amd import binding as B  # noqa: E402
from paper_2503_21364_amd import scenes  # noqa: E402

F = scenes.ANCHOR_FEAT
NETS = ("opacity", "colour", "cov")
Y00 = 0.5 / np.sqrt(np.pi)
DEV = "cuda:0"


class BlockDecoder:
    """Weights of the three perceptrons for every block: first layers side by side ([blocks][3 F][F + 3]), second layers
    as the decoder has them ([blocks][F][outputs])."""

    def __init__(self, blocks: int, k: int, seed: int = 7001):
        nets = [scenes.make_decoder(seed + g, k) for g in range(blocks)]
        stack = lambda f: torch.from_numpy(np.stack([f(m) for m in nets])).to(DEV)
        self.w1 = stack(lambda m: np.concatenate([m[n]["w1"] for n in NETS]))
        self.b1 = stack(lambda m: np.concatenate([m[n]["b1"] for n in NETS]))
        self.w2 = [stack(lambda m, n=n: m[n]["w2t"]) for n in NETS]
        self.b2 = [stack(lambda m, n=n: m[n]["b2"]) for n in NETS]

    def tensors(self):
        return [self.w1, self.b1, *self.w2, *self.b2]


class Trainer:
    def __init__(self, anchors: int, blocks: int, k: int = 4, width: int = 640, height: int = 360, lr: float = 2e-3):
        scene = scenes.make_anchor_scene(anchors, k=k, layout="clusters")
        scene = B.reorder_anchors(scene, 2.0)
        self.a, self.k = anchors, k
        cams = scenes.make_cameras(2, width, height)[:4]
        self.cams = [B.make_camera(c) for c in cams]
        self.eyes = [torch.tensor(np.asarray(c["cam_pos"]), dtype=torch.float32, device=DEV) for c in cams]
        f = lambda t: torch.from_numpy(np.ascontiguousarray(t, dtype=np.float32)).to(DEV)
        self.position, self.feature = f(scene["position"]), f(scene["feature"])
        self.extent, self.offsets = f(scene["extent"]), f(scene["offsets"])
        edges = np.linspace(0, anchors, blocks + 1).astype(np.int32)
        self.blocks = torch.from_numpy(edges).to(DEV)

        # the targets: one decoder for the whole scene
        shared, out = B.AnchorScene(scene, scenes.make_decoder(7000, k)), B.DecodedScene(anchors, k)
        self.frame, self.targets = B.Frame(anchors * k, width, height, 60 * anchors * k), []
        for cam, c in zip(self.cams, cams):
            B.anchor_decode(shared, c["cam_pos"], out)
            B.render_frame(out.scene(), cam, self.frame)
            self.targets.append(self.frame.out_rgb.clone())

        # what a step writes and keeps
        self.net = BlockDecoder(blocks, k)
        self.grads = [torch.empty_like(t) for t in self.net.tensors()]
        for p, g in zip(self.net.tensors(), self.grads):
            p.grad = g
        self.optimiser = torch.optim.Adam(self.net.tensors(), lr=lr)
        e = lambda *shape: torch.empty(shape, dtype=torch.float32, device=DEV)
        self.h, self.dh = e(anchors, 3 * F), e(anchors, 3 * F)
        self.y = [e(anchors, per * k) for per in scenes.ANCHOR_OUTS.values()]
        self.kept_x, self.kept_h = B.Checkpoint8(anchors, F + 3), [B.Checkpoint8(anchors, F) for _ in NETS]
        need = [B.grouped_linear_backward_bytes(anchors, blocks, 3 * F, F + 3)]
        need += [B.grouped_linear_backward_bytes(anchors, blocks, per * k, F) for per in scenes.ANCHOR_OUTS.values()]
        self.work = torch.empty(max(need), dtype=torch.uint8, device=DEV)
        self.decoded = B.DecodedScene(anchors, k)
        self.scene = self.decoded.scene()
        self.scene_grads = B.SceneGrads(self.scene)
        self.grad_feat = e(anchors * k, B.FEAT_STRIDE)

    def _combine(self, y_op, y_col, y_cov):
        """Outputs of the perceptrons to the attributes of the primitives, as lmk_gs_anchor_decode defines them."""
        a, k = self.a, self.k
        opacity = torch.tanh(y_op).clamp(min=0).reshape(-1)
        sh = torch.nn.functional.pad((torch.sigmoid(y_col.reshape(a * k, 3)) - 0.5) / Y00, (0, 1))
        cov = y_cov.reshape(a, k, 7)
        scale = (torch.sigmoid(cov[..., :3]) * self.extent[3:].T[:, None]).reshape(a * k, 3).T
        rot = cov[..., 3:].reshape(a * k, 4).T
        return dict(opacity=opacity, sh=sh, scale=scale, rot=rot)

    def step(self, view: int) -> torch.Tensor:
        """One optimisation step on viewpoint `view`; the squared error in front of it, on the GPU."""
        net, cam = self.net, self.cams[view]
        d = self.position - self.eyes[view][:, None]
        x = torch.cat([self.feature, (d / d.norm(dim=0, keepdim=True)).T], dim=1)

        # ---- forward
        B.grouped_linear(x, net.w1, self.blocks, self.h, bias=net.b1, relu=True, checkpoint=self.kept_x)
        for m in range(3):
            B.grouped_linear(self.h[:, m * F:(m + 1) * F], net.w2[m], self.blocks, self.y[m], bias=net.b2[m], in_major=True,
                             checkpoint=self.kept_h[m])
        y = [t.detach().requires_grad_(True) for t in self.y]
        attributes = self._combine(*y)
        centre = self.position.T[:, None] + self.offsets * self.extent[:3].T[:, None]
        self.decoded.mean.copy_(centre.reshape(-1, 3).T)
        for name, t in attributes.items():
            getattr(self.decoded, name).copy_(t.detach())
        B.render_frame(self.scene, cam, self.frame)

        # ---- backward
        off = self.frame.out_rgb - self.targets[view]
        B.render_backward(cam, self.frame, 2 * off / off.numel(), None, self.grad_feat)
        B.preprocess_backward(self.scene, cam, self.frame, self.grad_feat, self.scene_grads)
        torch.autograd.backward(list(attributes.values()), [getattr(self.scene_grads, name) for name in attributes])
        dw1, db1, dw2, db2 = self.grads[0], self.grads[1], self.grads[2:5], self.grads[5:8]
        for m in range(3):
            B.grouped_linear_backward(y[m].grad, net.w2[m], self.blocks, self.work, checkpoint=self.kept_h[m], gate=True, in_major=True,
                                      dx=self.dh[:, m * F:(m + 1) * F], dw=dw2[m], db=db2[m])
        B.grouped_linear_backward(self.dh, net.w1, self.blocks, self.work, checkpoint=self.kept_x, dw=dw1, db=db1)
        self.optimiser.step()
        return off.square().mean()


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--anchors", type=int, default=20_000)
    ap.add_argument("--blocks", type=int, default=8)
    ap.add_argument("--steps", type=int, default=20)
    args = ap.parse_args()
    t = Trainer(args.anchors, args.blocks)
    for i in range(args.steps):
        print(f"step {i}: squared error {float(t.step(i % len(t.cams))):.6f}", flush=True)


if __name__ == "__main__":
    main()
