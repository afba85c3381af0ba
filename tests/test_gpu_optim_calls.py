"""How the optimizer's calls go together: what would change nothing, or something else than was meant, is refused."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _adamw(**kw):
    from paper_2504_05638_amd.train import AdamW
    return AdamW(params=[torch.ones(1000, device="cuda")], grads=[torch.ones(1000, device="cuda")], groups=[(0.5, 0.0)], **kw)


@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_that_nothing_began(bits):
    opt = _adamw(bits=bits)
    with pytest.raises(RuntimeError, match="grad_norm"):
        opt.step()
    opt.grad_norm()
    opt.step()
    assert torch.allclose(opt.params[0], torch.full_like(opt.params[0], 0.5))
    assert opt.control[0].item() == 1


def test_a_given_step_of_an_optimizer_that_clips():
    opt = _adamw(max_norm=1.0)
    with pytest.raises(ValueError, match="max_norm"):
        opt.step(1)
    assert torch.equal(opt.params[0], torch.ones_like(opt.params[0]))
    opt.grad_norm()
    opt.step()      # clipped from 31.6 to 1: each gradient is 1 / sqrt(1000), m a tenth of that
    assert torch.allclose(opt.m[0], torch.full_like(opt.m[0], 0.1 * 1000 ** -0.5))


@pytest.mark.parametrize("step", [-1, 1 << 32, (1 << 32) + 1])
def test_a_step_that_does_not_fit_its_word(step):
    """(cut to 32 bits they would be step 4294967295, the one that grad_norm() began, and step 1)"""
    opt = _adamw()
    opt.grad_norm()
    with pytest.raises(ValueError, match="2\\^32"):
        opt.step(step)
    assert torch.equal(opt.params[0], torch.ones_like(opt.params[0]))
