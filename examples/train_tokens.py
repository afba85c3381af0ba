"""A small language model trained by several simulated ranks on one GPU, every step through the library: tokens' vectors and positions from
tables, a block of linear layers between two norms, the loss over the vocabulary; the linear layers' gradients go through
the exchange (sparsified with error feedback, compressed, summed, decoded), tables', norms' and biases' are just summed; AdamW
over all of them.

The tokens are a chain in which each has a few that may follow it, so that the loss falls from log(vocab) towards the chain's own.
With --teacher every other rank's loss is the divergence from the chain's distribution, as a teacher's largest scores tell it.

    python examples/train_tokens.py [--steps 100] [--ranks 2] [--width 256] [--vocab 1000] [--teacher]
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2504_05638_amd import binding as B  # noqa: E402
from paper_2504_05638_amd.bucket import TagcBucket  # noqa: E402
from paper_2504_05638_amd.train import (AdamW, cross_entropy, cross_entropy_backward, dense_views, distill, distill_backward,  # noqa: E402
                                        embedding, embedding_backward, linear, linear_backward, norm, norm_backward)


class Model:
    """head(norm2(h + w2 gelu(w1 norm1(h) + b1) + b2)), h = table[token] + positions[place]; fp32 parameters and their bf16 copies."""

    NAMES = ["table", "positions", "gain1", "shift1", "w1", "b1", "w2", "b2", "gain2", "head"]

    def __init__(self, vocab, places, width, gen):
        d = width
        shapes = [(vocab, d), (places, d), (d,), (d,), (4 * d, d), (4 * d,), (d, 4 * d), (d,), (d,), (vocab, d)]
        scale = {"table": 0.02, "positions": 0.02, "w1": d ** -0.5, "w2": 0.5 * d ** -0.5, "head": d ** -0.5}
        self.params = [torch.randn(s, generator=gen, device="cuda").mul_(scale.get(n, 0.0)).add_(1.0 if n.startswith("gain") else 0.0)
                       for n, s in zip(self.NAMES, shapes)]
        self.copies = [p.to(torch.bfloat16) for p in self.params]
        self.segments, at = [], 0
        for n, p in zip(self.NAMES, self.params):
            self.segments.append((at, p.numel(), 100_000, B.TAGC_SEG_COMPRESS if n in ("w1", "w2") else 0))
            at += p.numel()
        self.size = at

    def views(self, flat):
        return [flat[at:at + n].view(p.shape) for (at, n, _, _), p in zip(self.segments, self.params)]

    def step(self, tokens, targets, grad, teacher=None):
        """The mean loss of one rank's tokens [batch, length]; its gradient is written into `grad`.  `teacher`: (ids, logits) of every
        place, in targets' stead."""
        table, positions, gain1, shift1, w1, b1, w2, b2, gain2, head = self.copies
        g = dict(zip(self.NAMES, self.views(grad)))
        places = torch.arange(tokens.shape[1], device="cuda").expand_as(tokens).contiguous()
        h = embedding(tokens, table, residual=embedding(places, positions))
        a, stats1 = norm(h, gain1, shift1, save=True)
        u, pre = linear(a, w1, b1, activation="gelu", save=True)
        y, _ = linear(u, w2, b2, residual=h)
        z, stats2 = norm(y, gain2, kind="rms", save=True)
        each = torch.full((1,), 1.0 / tokens.numel(), device="cuda")
        if teacher is None:
            loss, saved = cross_entropy(z, head, targets, save=True)
            dz = cross_entropy_backward(each, z, head, targets, saved, dw=g["head"])
        else:
            loss, saved = distill(z, head, *teacher, save=True)
            dz = distill_backward(each, z, head, *teacher, saved, dw=g["head"])
        dy = norm_backward(dz, y, gain2, stats2, kind="rms", dw=g["gain2"])
        du = linear_backward(dy, u, w2, dw=g["w2"], db=g["b2"])
        da = linear_backward(du, a, w1, pre, activation="gelu", dw=g["w1"], db=g["b1"])
        dh = norm_backward(da, h, gain1, stats1, residual=dy, dw=g["gain1"], db=g["shift1"])
        embedding_backward(dh, tokens, g["table"])
        embedding_backward(dh, places, g["positions"])
        return loss.mean()


class Chain:
    """Tokens of which each may be followed by four, the first of them mostly."""

    def __init__(self, vocab, gen):
        self.vocab, self.gen = vocab, gen
        self.follow = torch.randint(0, vocab, (vocab, 4), generator=gen, device="cuda")
        self.share = torch.tensor([0.7, 0.15, 0.1, 0.05], device="cuda")

    def sample(self, batch, length):
        out = torch.empty((batch, length + 1), dtype=torch.int64, device="cuda")
        out[:, 0] = torch.randint(0, self.vocab, (batch,), generator=self.gen, device="cuda")
        for i in range(length):
            which = torch.multinomial(self.share, batch, replacement=True, generator=self.gen)
            out[:, i + 1] = self.follow[out[:, i], which]
        return out[:, :-1].contiguous(), out[:, 1:].contiguous()

    def teacher(self, tokens):
        return self.follow[tokens].contiguous(), self.share.log().expand(*tokens.shape, 4).contiguous()


def train(steps=100, ranks=2, width=256, vocab=1000, batch=8, length=64, teacher=False, seed=0, tell=lambda *a: None):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    model, chain = Model(vocab, length, width, gen), Chain(vocab, gen)
    grads = [torch.zeros(model.size, dtype=torch.bfloat16, device="cuda") for _ in range(ranks)]
    bucket = TagcBucket(model.segments, B.TAGC_BF16, ranks, sizing_milli=1500, seed=seed, dense=True, error_feedback=True)
    summed = dense_views(bucket)
    for i, (_, n, _, compressed) in enumerate(model.segments):
        if not compressed:
            summed[i] = torch.zeros(n, device="cuda")
    opt = AdamW(params=model.params, grads=summed, copies=model.copies, groups=[(2e-3, 0.01), (2e-3, 0.0)],
                group_of=[0 if p.dim() == 2 else 1 for p in model.params], bits=8, grad_scale=1.0 / ranks, max_norm=1.0, seed=seed)
    losses = []
    for _ in range(steps):
        loss = 0.0
        for r in range(ranks):
            tokens, targets = chain.sample(batch, length)
            loss = loss + model.step(tokens, targets, grads[r], chain.teacher(tokens) if teacher and r % 2 else None)
        bucket.run(grads, fused=True)
        for i, (at, n, _, compressed) in enumerate(model.segments):
            if not compressed:
                summed[i].copy_(torch.stack([g[at:at + n] for g in grads]).float().sum(0))
        norm_, _ = opt.grad_norm()
        opt.step()
        losses.append(loss / ranks)
        if len(losses) % 10 == 0:
            tell("step %d: loss %.4f (log vocab %.2f), gradient norm %.4f" % (len(losses), float(losses[-1]), math.log(vocab), float(norm_)))
    bucket.close()
    return [float(x) for x in losses]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--ranks", type=int, default=2)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--vocab", type=int, default=1000)
    ap.add_argument("--teacher", action="store_true")
    a = ap.parse_args()
    train(a.steps, a.ranks, a.width, a.vocab, teacher=a.teacher, tell=lambda *x: print(*x, flush=True))
