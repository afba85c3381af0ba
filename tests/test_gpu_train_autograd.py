"""What torch's autograd gets to know of calls that write past it."""
import warnings

import pytest
import torch

pytestmark = pytest.mark.gpu


def _layer():
    return torch.randn(40, 64, device="cuda"), torch.randn(32, 64, device="cuda"), torch.randn(32, device="cuda"), torch.randn(40, 32, device="cuda")


def test_a_graph_that_is_not_recorded_is_told():
    from paper_2504_05638_amd.train import linear
    for which in range(4):
        args = list(_layer())
        args[which].requires_grad_()
        with pytest.warns(UserWarning, match="autograd"):
            y, _ = linear(*args)
        assert not y.requires_grad
        with warnings.catch_warnings():
            warnings.simplefilter("error")
            with torch.no_grad():
                again, _ = linear(*args)
            linear(*(t.detach() for t in args))
        assert torch.equal(y, again)


def test_written_tensors_count_a_version():
    from paper_2504_05638_amd.train import AdamW, linear, linear_backward
    x, w, b, dy = _layer()
    out, pre = torch.empty_like(dy), torch.empty_like(dy)
    flat = torch.zeros(w.numel() + 32, device="cuda")
    dw, db, dx = flat[:w.numel()].view_as(w), flat[w.numel():], torch.empty_like(x)

    def versions():
        return [t._version for t in (x, w, b, dy, out, pre, flat, dx)]

    was = versions()
    linear(x, w, b, activation="silu", save=True, out=out, pre=pre)
    assert [n > o for n, o in zip(versions(), was)] == [False] * 4 + [True, True, False, False]
    was = versions()
    linear_backward(dy, x, w, pre, activation="silu", dx=dx, dw=dw, db=db)
    assert [n > o for n, o in zip(versions(), was)] == [False] * 6 + [True, True]
    with torch.inference_mode():    # (tensors that have no version)
        linear(x, w, out=torch.empty_like(dy))
        y, _ = linear(x, w)
    copy = torch.zeros(32, device="cuda", dtype=torch.bfloat16)
    opt = AdamW(params=[w, b], grads=[dw, db], copies=[None, copy])
    was = versions() + [copy._version]
    opt.step(1)
    assert [n > o for n, o in zip(versions() + [copy._version], was)] == [False, True, True, False, False, False, False, False, True]


def test_a_stale_graph_raises():
    """loss.backward() through parameters that a step has changed since: torch's optimizers make it raise."""
    from paper_2504_05638_amd.train import AdamW
    x, w = _layer()[:2]
    w.requires_grad_()
    x.requires_grad_()
    loss = (x @ w.t()).square().sum()
    grad = torch.ones_like(w)
    AdamW(params=[w], grads=[grad]).step(1)
    with pytest.raises(RuntimeError, match="inplace"):
        loss.backward()
    with torch.inference_mode():
        p, g = torch.zeros(5, device="cuda"), torch.ones(5, device="cuda")
    AdamW(params=[p], grads=[g]).step(1)
