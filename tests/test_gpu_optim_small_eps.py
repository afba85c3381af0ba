"""AdamW where eps is nothing against the roots of second moments that float32 holds as subnormal numbers."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
LR, BETAS = 0.25, (0.9, 0.95)


def _grads(n, seed):
    """Signs and sizes from 2e-21 to 2e-18: their squares times 0.05 are 2e-43 to 2e-37, subnormal and normal."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    size = 10 ** (torch.rand(n, generator=gen, device="cuda") * 3 - 20.7)
    return size * torch.sign(torch.randn(n, generator=gen, device="cuda"))


@pytest.mark.parametrize("eps", [0.0, 1e-20])
@pytest.mark.parametrize("begun", [True, False])
def test_32_bit_moments(eps, begun):
    """Bounds: g g and v are subnormal, rounded to multiples of q = 2^-149 once each (twice half a q), m to 4 e; the root halves
    v's relative error; quotient, products and differences 8 e more."""
    from paper_2504_05638_amd.train import AdamW
    g = _grads(20_011, 1)
    p = torch.zeros_like(g)
    opt = AdamW(params=[p], grads=[g], betas=BETAS, eps=eps, groups=[(LR, 0.0)])
    for step in (1, 2):
        m0, v0 = (t[0].double().clone() for t in (opt.m, opt.v))
        was = p.double().clone()
        if begun:
            opt.grad_norm()
            opt.step()
        else:
            opt.step(step)
        d = g.double()
        m, v = BETAS[0] * m0 + (1 - BETAS[0]) * d, BETAS[1] * v0 + (1 - BETAS[1]) * d * d
        root = (v / (1 - BETAS[1] ** step)).sqrt()
        update = LR / (1 - BETAS[0] ** step) * m / (root + eps)
        v_rel = (2 * 2.0 ** -149 + 6 * E * v) / v
        assert torch.isfinite(p).all()
        assert torch.all((p.double() - (was - update)).abs() <= (v_rel + 16 * E) * update.abs() + 2 * E * was.abs())


def test_8_bit_moments():
    """From moments of nothing the first step goes by the gradient's sign alone, whatever its size; later ones stay near it, since a
    code is within an eighth."""
    from paper_2504_05638_amd.train import AdamW
    g = _grads(20_011, 2)
    p = torch.zeros_like(g)
    opt = AdamW(params=[p], grads=[g], betas=BETAS, eps=0.0, bits=8, groups=[(LR, 0.0)])
    opt.step(1)
    # v's own rounding, to 2^-149, is a fiftieth of the smallest; the root halves it
    assert torch.all((p + LR * torch.sign(g)).abs() <= 0.01 * LR)
    opt.step(2)
    assert torch.isfinite(p).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_nothing_else_changes(bits):
    """A step with an eps of 1e-8 and one with an eps just small enough for the other form: the moments are the same bits, the updates
    within their roundings."""
    from paper_2504_05638_amd.train import AdamW
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    g = torch.randn(9001, generator=gen, device="cuda") * 1e-3
    out = []
    for eps in (1e-8, 1e-12):
        opt = AdamW(params=[torch.zeros_like(g)], grads=[g], betas=BETAS, eps=eps, bits=bits, groups=[(LR, 0.0)])
        for step in range(1, 4):
            opt.step(step)
        out.append(opt)
    a, b = out
    assert torch.equal(a.m[0], b.m[0]) and torch.equal(a.v[0], b.v[0])
    big = g.abs() > 1e-4   # (three updates of at most LR, changed by eps / |g| < 1e-4 of it and, in 8 bits, 4 times that where v was rounded down)
    assert torch.all((a.params[0] - b.params[0]).abs()[big] <= 3 * LR * 4e-4)
    assert np.isfinite(a.params[0].cpu().numpy()).all()
