"""Losses over a vocabulary: what a teacher that is not finite leaves."""
import math

import pytest
import torch

from .test_gpu_loss import T, _randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M", [40, 1100])
@pytest.mark.parametrize("K", [1, 2, 6])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("score", [math.nan, math.inf], ids=str)
def test_a_teacher_that_is_not_finite(score, dtype, K, M):
    """softmax of NaN or of +infinity is NaN: so are that row's loss, its dx, and dw of its terms; no other row's."""
    from paper_2504_05638_amd.train import distill, distill_backward
    D, V, row = 64, 300, 7
    x, w = _randn((M, D), 1, T[dtype]), _randn((V, D), 2, T[dtype], D ** -0.5)
    ids = torch.arange(M * K, device="cuda").view(M, K) * 7 % (V - K)
    ids[row] = V - K + torch.arange(K, device="cuda")          # (tokens that no other row has)
    logits = torch.randn((M, K), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    one, dwant, dw = torch.ones((), device="cuda"), torch.empty_like(w), torch.empty_like(w)
    want, saved = distill(x, w, ids, logits, save=True)
    dx_want = distill_backward(one, x, w, ids, logits, saved, dw=dwant)
    logits[row, 0] = score
    loss, saved = distill(x, w, ids, logits, save=True)
    dx = distill_backward(one, x, w, ids, logits, saved, dw=dw)
    keep = torch.arange(M, device="cuda") != row
    assert torch.isnan(loss[row]) and torch.equal(loss[keep], want[keep])
    assert torch.isnan(dx[row]).all() and torch.equal(dx[keep], dx_want[keep])
    assert torch.isnan(dw[V - K:]).all() and torch.equal(dw[:V - K], dwant[:V - K])
