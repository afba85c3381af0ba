"""The layers together, as a model's step has them: vectors from tables, norms, linear layers, a loss over the vocabulary, and back into one flat
gradient; eager, captured in a graph, and in the example.

Gradients are compared with float64's as 2-norms.  A step rounds some 20 times between a weight and its gradient, each by half a step at
most (2^-8 of the value in bfloat16); what a rounding changes reaches the gradient through norms, slopes and shares, none of which
makes more than twice of it: 20 * 2 * 2^-8 = 0.16.  In float32 sums of some hundred terms add to it: 20 * 2 * 128 * 2^-24 = 3e-4."""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BOUND = {torch.bfloat16: 0.16, torch.float32: 3e-4}
NAMES = ["table", "positions", "gain1", "shift1", "w1", "b1", "w2", "b2", "gain2", "head"]


def _example():
    spec = importlib.util.spec_from_file_location("train_tokens", os.path.join(ROOT, "examples", "train_tokens.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _reference(weights, tokens, targets, teacher, scale):
    """Loss of every row and gradients, from the definitions in float64."""
    p = [w.detach().double().requires_grad_() for w in weights]
    table, positions, gain1, shift1, w1, b1, w2, b2, gain2, head = p
    h = table[tokens] + positions[torch.arange(tokens.shape[1], device="cuda")]
    z = h - h.mean(-1, keepdim=True)
    a = z / (z.square().mean(-1, keepdim=True) + 1e-5).sqrt() * gain1 + shift1
    u = a @ w1.t() + b1
    u = 0.5 * u * torch.erfc(-u / math.sqrt(2))
    y = h + u @ w2.t() + b2
    z = y / (y.square().mean(-1, keepdim=True) + 1e-5).sqrt() * gain2
    log_p = torch.log_softmax(z @ head.t(), -1)
    if teacher is None:
        there = targets >= 0
        loss = torch.where(there, -log_p.gather(-1, targets.clamp(min=0)[..., None])[..., 0], 0.0)
    else:
        log_q = torch.log_softmax(teacher[1].double(), -1)
        loss = (log_q.exp() * (log_q - log_p.gather(-1, teacher[0]))).sum(-1)
    return loss, torch.autograd.grad(loss.sum() * scale, p)


class _Step:
    """The example's step, for both types."""

    def __init__(self, dtype, vocab, length, width, batch, seed=0):
        self.model = _example().Model(vocab, length, width, torch.Generator(device="cuda").manual_seed(seed))
        for p, n in zip(self.model.params, NAMES):
            if p.dim() == 1:        # (nothing of which is 0 or 1)
                p.add_(torch.linspace(-0.3, 0.4, p.numel(), device="cuda"))
            if n in ("table", "positions"):
                p.mul_(20)
        self.model.copies = [p.to(dtype) for p in self.model.params]
        self.gen = torch.Generator(device="cuda").manual_seed(seed + 1)
        self.vocab, self.shape = vocab, (batch, length)
        self.tokens, self.targets = (torch.zeros(self.shape, dtype=torch.int64, device="cuda") for _ in range(2))
        self.grad = torch.empty(self.model.size, dtype=dtype, device="cuda")
        self.fill()

    def fill(self):
        t = torch.randint(0, self.vocab, (self.shape[0], self.shape[1] + 1), generator=self.gen, device="cuda")
        self.tokens.copy_(t[:, :-1])
        self.targets.copy_(torch.where(torch.rand(self.shape, generator=self.gen, device="cuda") < 0.2, -100, t[:, 1:]))

    def run(self, teacher=None):
        return self.model.step(self.tokens, self.targets, self.grad, teacher)

    def check(self, loss, teacher=None):
        dtype = self.grad.dtype
        want, grads = _reference(self.model.copies, self.tokens, self.targets, teacher, 1.0 / self.tokens.numel())
        assert abs(float(loss) - float(want.mean())) < BOUND[dtype] * float(want.mean())
        for n, g, r in zip(NAMES, self.model.views(self.grad), grads):
            off = float((g.double() - r).norm() / r.norm())
            assert off < BOUND[dtype], (n, off)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sizes", [(300, 16, 96, 4), (1003, 33, 130, 7), (97, 1, 64, 1)], ids=str)
def test_step(sizes, dtype):
    s = _Step(dtype, *sizes)
    s.check(s.run())
    ids = torch.randint(0, sizes[0], (*s.shape, 5), generator=s.gen, device="cuda")
    logits = torch.randn((*s.shape, 5), generator=s.gen, device="cuda")
    s.check(s.run((ids, logits)), (ids, logits))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_step_replayed_from_a_graph(dtype):
    """Replays with other tokens, eager steps and synchronizations between them, give what eager steps give, bit for bit."""
    s = _Step(dtype, 500, 40, 128, 6)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        loss = s.run()
    for _ in range(4):
        s.fill()
        want = s.run().clone()
        grad = s.grad.clone()
        torch.cuda.synchronize()
        s.grad.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, want) and torch.equal(s.grad, grad)


def test_two_graphs_of_losses_side_by_side():
    """Two captured losses, each with its own workspace, replayed on two streams at once."""
    from paper_2504_05638_amd.train import cross_entropy, cross_entropy_backward
    made = []
    for k in range(2):
        gen = torch.Generator(device="cuda").manual_seed(k)
        x, w = torch.randn(1500, 256, generator=gen, device="cuda").bfloat16(), (torch.randn(9000, 256, generator=gen, device="cuda") / 16).bfloat16()
        t, one = torch.randint(-100, 9000, (1500,), generator=gen, device="cuda"), torch.ones(1, device="cuda")
        dw = torch.empty_like(w)
        loss, saved = cross_entropy(x, w, t, save=True)
        want = (loss, cross_entropy_backward(one, x, w, t, saved, dw=dw), dw.clone())
        torch.cuda.synchronize()
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=stream):
            loss, saved = cross_entropy(x, w, t, save=True)
            dx = cross_entropy_backward(one, x, w, t, saved, dw=dw)
        made.append((stream, graph, want, (loss, dx, dw), (x, w, t, one)))
    torch.cuda.synchronize()
    for _ in range(3):
        for stream, graph, _, got, _ in made:
            with torch.cuda.stream(stream):
                got[2].zero_()
                graph.replay()
        torch.cuda.synchronize()
        for _, _, want, got, _ in made:
            assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("teacher", [False, True])
def test_the_example_runs(teacher):
    losses = _example().train(steps=4, ranks=2, width=64, vocab=200, batch=4, length=24, teacher=teacher)
    assert len(losses) == 4 and all(math.isfinite(x) for x in losses)
