"""A feed-forward block trained by several simulated ranks on one GPU, every step through the library:

  each rank    forward and backward of two linear layers (GELU between them, a residual around them); the
               weights' and biases' gradients go straight into the rank's flat gradient
  exchange     the weights' gradients are sparsified with error feedback, compressed, summed and
               decoded (TagcBucket); the biases', too small to be worth it, are just summed
  optimizer    norm of all gradients, clipping, AdamW with 8-bit moments on fp32 weights, whose bf16
               copies the layers use

    python examples/train_block.py [--steps 60] [--ranks 4] [--width 512]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2504_05638_amd import binding as B  # noqa: E402
from paper_2504_05638_amd.bucket import TagcBucket  # noqa: E402
from paper_2504_05638_amd.train import AdamW, dense_views, linear, linear_backward  # noqa: E402


class Block:
    """x + w2 gelu(w1 x + b1) + b2, its fp32 parameters and their bf16 copies."""

    def __init__(self, width, gen):
        shapes = [(4 * width, width), (4 * width,), (width, 4 * width), (width,)]
        self.params = [torch.randn(s, generator=gen, device="cuda") * (s[1] ** -0.5 if len(s) == 2 else 0.0) for s in shapes]
        self.copies = [p.to(torch.bfloat16) for p in self.params]
        # the flat gradient that a communication hook would see: the weights are compressed
        self.segments, at = [], 0
        for s in shapes:
            n = torch.Size(s).numel()
            self.segments.append((at, n, 100_000, B.TAGC_SEG_COMPRESS if len(s) == 2 else 0))
            at += n
        self.size = at

    def views(self, flat):
        return [flat[at:at + n].view(p.shape) for (at, n, _, _), p in zip(self.segments, self.params)]

    def step(self, x, target, grad):
        """The loss of one rank's batch; its gradient is written into `grad`."""
        w1, b1, w2, b2 = self.copies
        g1, gb1, g2, gb2 = self.views(grad)
        h, pre = linear(x, w1, b1, activation="gelu", save=True)
        y, _ = linear(h, w2, b2, residual=x)
        off = y.float() - target.float()
        dy = (off * (2.0 / off.numel())).to(torch.bfloat16)
        dh = linear_backward(dy, h, w2, dw=g2, db=gb2)
        linear_backward(dh, x, w1, pre, activation="gelu", dw=g1, db=gb1, need_dx=False)
        return off.square().mean()


def train(steps=60, ranks=4, width=512, rows=256, seed=0, tell=lambda *a: None):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    block, teacher = Block(width, gen), Block(width, gen)
    grads = [torch.zeros(block.size, dtype=torch.bfloat16, device="cuda") for _ in range(ranks)]
    bucket = TagcBucket(block.segments, B.TAGC_BF16, ranks, sizing_milli=1500, seed=seed, dense=True, error_feedback=True)
    # what the optimizer reads: the decoded sums of the weights' gradients, the plain sums of the biases'
    summed = dense_views(bucket)
    for i, (_, n, _, compressed) in enumerate(block.segments):
        if not compressed:
            summed[i] = torch.zeros(n, device="cuda")
    opt = AdamW(params=block.params, grads=summed, copies=block.copies, groups=[(2e-3, 0.01), (2e-3, 0.0)],
                group_of=[0 if s[3] else 1 for s in block.segments], bits=8, grad_scale=1.0 / ranks, max_norm=1.0, seed=seed)
    losses = []
    for _ in range(steps):
        loss = 0.0
        for r in range(ranks):
            x = torch.randn(rows, width, generator=gen, device="cuda").to(torch.bfloat16)
            h, _ = linear(x, teacher.copies[0], teacher.copies[1], activation="gelu")
            target, _ = linear(h, teacher.copies[2], teacher.copies[3], residual=x)
            loss = loss + block.step(x, target, grads[r])
        bucket.run(grads, fused=True)
        for i, (at, n, _, compressed) in enumerate(block.segments):
            if not compressed:
                summed[i].copy_(torch.stack([g[at:at + n] for g in grads]).float().sum(0))
        norm, _ = opt.grad_norm()
        opt.step()
        losses.append(loss / ranks)
        if len(losses) % 10 == 0:
            tell("step %d: loss %.4f, gradient norm %.4f, %d entries of the gradient sent" % (
                len(losses), float(losses[-1]), float(norm), bucket.header()["U"]))
    bucket.close()
    return [float(x) for x in losses]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--ranks", type=int, default=4)
    ap.add_argument("--width", type=int, default=512)
    a = ap.parse_args()
    train(a.steps, a.ranks, a.width, tell=lambda *x: print(*x, flush=True))
