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
