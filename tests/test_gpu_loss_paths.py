"""Losses over a vocabulary where they take the ways that few rows do not: several terms a row over several pieces of the vocabulary, forward of more than 1024
rows without terms, with scores far apart, with rows that are not finite; and what a teacher that is not finite leaves.

Bounds are those of test_gpu_loss.py."""
import math

import pytest
import torch

from . import test_gpu_loss as plain
from .test_gpu_loss import E, Ref, T, _check, _near, _randn, _terms

pytestmark = pytest.mark.gpu


@pytest.fixture
def edges(monkeypatch):
    """Terms at multiples of 256 and in front of them, the first and the last token: on both sides of wherever a piece of the vocabulary, a tile or a strip
    ends; some of them twice in their row."""
    def terms(M, V, K, seed, empty, long=True):
        ids, logits = _terms(M, V, K, seed, empty, long)
        gen = torch.Generator(device="cuda").manual_seed(seed + 99)
        edge = 256 * torch.randint(0, V // 256 + 1, (M, K), generator=gen, device="cuda") - torch.randint(0, 2, (M, K), generator=gen, device="cuda")
        edge = torch.where(torch.rand((M, K), generator=gen, device="cuda") < 0.1, V - 1, edge % V)
        there = (ids >= 0) & (ids < V) & (torch.rand((M, K), generator=gen, device="cuda") < 0.6)
        ids = torch.where(there, edge.to(ids.dtype), ids)
        if K > 2:
            ids[:, 2] = torch.where((torch.rand(M, generator=gen, device="cuda") < 0.3) & there[:, 0] & there[:, 2], ids[:, 0], ids[:, 2])
        return ids, logits

    monkeypatch.setattr(plain, "_terms", terms)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K", [1, 3, 5, 17])
def test_terms_in_pieces_of_the_vocabulary_backward(K, dtype, edges):
    """ds of 65536 rows: 4096 tokens at a time in bfloat16, 1280 in float32."""
    print("[case] terms, pieces, backward", K, dtype, flush=True)
    _check((65536, 40, 5003), T[dtype], K, 2.0, True, K == 5, 11, 0, repeat=K == 3)


@pytest.mark.parametrize("K", [3, 5, 33, 300])
@pytest.mark.parametrize("shape,dtype", [((1400, 2001, 60_001), "f32"), ((300, 4001, 70_001), "bf16")], ids=str)
def test_terms_in_pieces_of_the_vocabulary_both_ways(shape, dtype, K, edges):
    """Two pieces forward and two and more backward; terms looked for (3) and listed by strips, a workgroup's terms of many rows (3 to 33) and of one (300)."""
    print("[case] terms, pieces, both ways", shape, dtype, K, flush=True)
    _check(shape, T[dtype], K, 1.0, True, K == 33, 21, 0, repeat=K == 5)


@pytest.mark.parametrize("V", [300, 7700])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_rows_without_any_term(dtype, V):
    """No row of more than are held counts, with a target, looked-for and listed terms: losses 0, dx 0, dw 0 or as it was."""
    from paper_2504_05638_amd import train
    for M in (1100, 4100):
        x, w = torch.full((M, 64), float("nan"), device="cuda", dtype=T[dtype]), _randn((V, 64), 1, T[dtype])
        dloss = torch.ones(M, device="cuda")
        for K in (0, 3, 6):
            print("[case] nothing counts", M, V, dtype, K, flush=True)
            t = torch.full((M, K) if K else (M,), -100, device="cuda")
            if K:
                t[::2], more = 5, (torch.where(torch.arange(M, device="cuda")[:, None] % 2 == 0, -math.inf, torch.randn((M, K), device="cuda")),)
                forward, backward = train.distill, train.distill_backward
            else:
                more, forward, backward = (), train.cross_entropy, train.cross_entropy_backward
            loss, saved = forward(x, w, t, *more, save=True)
            assert loss.shape == (M,) and not loss.any() and not saved.any()
            dw = torch.ones_like(w)
            assert not backward(dloss, x, w, t, *more, saved, dw=dw, accumulate=True).any() and torch.equal(dw, torch.ones_like(w))
            assert not backward(dloss, x, w, t, *more, saved, dw=dw).any() and not dw.any()


@pytest.mark.parametrize("V", [300, 7700])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_far_apart_of_many_rows(dtype, V):
    from paper_2504_05638_amd.train import cross_entropy, cross_entropy_backward
    x, w = _randn((1100, 64), 1, T[dtype], 40.0), _randn((V, 64), 2, T[dtype], 20.0)
    s = x.double() @ w.double().t()
    t = s.argmax(1)
    t[::3] = torch.arange(0, 1100, 3, device="cuda") % V      # (tokens that are out of the question, too)
    loss, saved = cross_entropy(x, w, t, save=True)
    ref = Ref(x, w, t, None, 1.0)
    _near(loss, *ref.loss(), torch.float32, "loss")
    _near(saved[:, :1], ref.lse, ref.lse_err, torch.float32, "lse")
    assert float(s.abs().max()) > 5000
    dx = cross_entropy_backward(torch.ones((), device="cuda"), x, w, t, saved)
    top = s.topk(2, dim=1).values
    sure = (top[:, 0] - top[:, 1] > 120) & (t == s.argmax(1))      # the others' share is under float32's numbers
    assert sure.any() and float(dx[sure].abs().max()) <= 2 * 70 * float(w.abs().max()) * float(ref.lse_err.max() + ref.s_err.max())


@pytest.mark.parametrize("V", [300, 7700])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_not_finite_rows_of_many_stay_where_they_are(dtype, V):
    """A score of -infinity is a token that the row cannot have (in float32 an infinity's products are NaN), one of +infinity or NaN leaves no loss."""
    from paper_2504_05638_amd.train import cross_entropy
    M, D = 1100, 64
    x, w, t = _randn((M, D), 1, T[dtype]), _randn((V, D), 2, T[dtype]), torch.arange(M, device="cuda") % V
    good, _ = cross_entropy(x, w, t)
    x[3, 5], x[30, 63], x[1099, 0] = float("nan"), float("inf"), float("-inf")
    loss, saved = cross_entropy(x, w, t, save=True)
    bad = torch.tensor([3, 30, 1099], device="cuda")
    keep = torch.ones(M, dtype=torch.bool, device="cuda")
    keep[bad] = False
    assert torch.equal(loss[keep], good[keep]) and not torch.isfinite(loss[bad]).any() and not torch.isfinite(saved[bad, 0]).any()
    w[V - 1, 1] = float("-inf")
    keep &= t != V - 1
    never = keep & (x[:, 1] > 0) if dtype == "bf16" else torch.zeros_like(keep)
    loss, _ = cross_entropy(x, w, t)
    rest, _ = cross_entropy(x, w[:V - 1], t)
    assert not torch.isfinite(loss[~never]).any()
    # (tiles' columns are the same, and what is added for the token is 0)
    assert torch.equal(loss[never], rest[never]) and (dtype == "f32" or never.any())


@pytest.mark.parametrize("K", [0, 5])
def test_gradient_against_differences_among_many_rows(K):
    """Five rows of 1100 have a gradient, and the loss is added up over them: the bound is that of five rows."""
    from paper_2504_05638_amd import train
    M, D, V, h, temperature, some = 1100, 33, 41, 2.0 ** -5, 1.0 if not K else 2.0, 5
    ids, logits = _terms(M, V, K or 1, 3, False)
    x, w, c = _randn((M, D), 1, torch.float32), _randn((V, D), 2, torch.float32, D ** -0.5), torch.rand(M, device="cuda") + 0.5
    rows = torch.tensor([0, 1, 517, 1024, 1099], device="cuda")
    c = torch.zeros_like(c).index_copy_(0, rows, c[rows])
    if K:
        call = lambda save: train.distill(x, w, ids, logits, temperature=temperature, save=save)  # noqa: E731
    else:
        ids = ids[:, 0].contiguous()
        call = lambda save: train.cross_entropy(x, w, ids, save=save)  # noqa: E731
    _, saved = call(True)
    dw = torch.empty_like(w)
    dx = (train.distill_backward(c, x, w, ids, logits, saved, temperature=temperature, dw=dw) if K
          else train.cross_entropy_backward(c, x, w, ids, saved, dw=dw))
    assert not dx[c == 0].any()
    for t, grad, places in ((x, dx, [(0, 0), (1099, 32), (517, 11)]), (w, dw, [(0, 0), (40, 32), (int(ids.view(M, -1)[0, 0]) % V, 5)])):
        for at in places:
            was = t[at].item()
            side = []
            for sign in (1, -1):
                t[at] = was + sign * h
                side.append(float((call(False)[0].double() * c.double()).sum()))
            t[at] = was
            assert abs((side[0] - side[1]) / (2 * h) - grad[at].item()) < 1.5 * 1.5 * some * 64 * h * h / 6 * 0.1 + 1.5 * some * 2.0 ** -19 / h, at


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


@pytest.mark.parametrize("M", [60, 1100])
@pytest.mark.parametrize("K", [0, 2])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nothing_but_ds_has_fewer_bits(dtype, K, M):
    """Where ds is a number of eight bits, gradients are float32's sums, rounded once: scores of 0 over 128 tokens make shares of 2^-7, and a term's ds is
    2^-7 less 1, or less a half."""
    from paper_2504_05638_amd import train
    D, V = 200, 128
    gen = torch.Generator(device="cuda").manual_seed(5)
    ids = torch.randint(0, V, (M, K or 1), generator=gen, device="cuda")
    if K:
        ids[:, 1] = (ids[:, 0] + 1 + torch.randint(0, V - 1, (M,), generator=gen, device="cuda")) % V       # (another one)
    logits = torch.full((M, K or 1), 1.5, device="cuda")
    ds = torch.full((M, V), 2.0 ** -7, device="cuda", dtype=torch.float64).scatter_add_(1, ids, torch.full(ids.shape, -1.0 / (K or 1), device="cuda", dtype=torch.float64))
    for zero in ("x", "w"):
        x, w = _randn((M, D), 1, T[dtype]), _randn((V, D), 2, T[dtype])
        (x if zero == "x" else w).zero_()
        more, t = ((logits,), ids) if K else ((), ids[:, 0].contiguous())
        forward, backward = (train.distill, train.distill_backward) if K else (train.cross_entropy, train.cross_entropy_backward)
        _, saved = forward(x, w, t, *more, save=True)
        dw = torch.empty_like(w)
        dx = backward(torch.ones((), device="cuda"), x, w, t, *more, saved, dw=dw)
        # (ds in float32 is off by some E of the shares' exponent, 7, and is then rounded to the eight bits that it should have, or held)
        for got, a, b in ((dx, ds, w.double()), (dw, ds.t(), x.double())):
            size = a.abs() @ b.abs()
            _near(got, a @ b, ((a.shape[1] + 16) * 2 + (40 if dtype == "f32" else 0)) * E * size, T[dtype], (zero, got.shape))
