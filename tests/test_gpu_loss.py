"""Losses over a vocabulary against float64: cross entropy and a teacher's divergence, forward and backward, both types, odd
sizes, strides and alignments, rows without a term, several pieces of the vocabulary.

Bounds, with E = 2^-24 (the products' are the linear layers'): a score is within (in + 8) 2 E of the sum of its products' magnitudes; a
log-sum of exponentials moves by no more than its scores, and its own additions are fewer than 64 + vocab / 512 in a row; an exponential's
argument is rounded by 4 E of its parts.  ds is rounded by half a step of the operands' type before the two products."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
T = {"f32": torch.float32, "bf16": torch.bfloat16}
SHAPES = [(1, 1, 1), (1, 64, 200), (1, 4096, 1000), (3, 64, 5), (17, 100, 31), (33, 128, 257), (64, 256, 1000), (65, 72, 4097), (129, 65, 130), (200, 777, 1001),
          (300, 64, 5003), (2048, 512, 2304), (1025, 96, 333), (70, 24, 130_001), (300, 72, 30_011)]


def _randn(shape, seed, dtype, scale=1.0, ld_more=0, shift=0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    m, n = shape
    buf = torch.full((m * (n + ld_more) + shift,), float("nan"), device="cuda", dtype=dtype)
    t = buf[shift:].view(m, n + ld_more)[:, :n]
    t.copy_(torch.randn(m, n, generator=gen, device="cuda") * scale)
    return t


def _half(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else E


def _near(got, ref, err, dtype, what):
    off = (got.double() - ref).abs()
    bound = err + _half(dtype) * (ref.abs() + err)
    assert torch.isfinite(got).all(), what
    assert torch.all(off <= bound + 1e-38), (what, float((off - bound).max()), float(off.max()))


def _terms(M, V, K, seed, empty, long=True):
    """ids [M, K], some none, some twice in a row, rows without any; logits, some -infinity."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    ids = torch.randint(0, V, (M, K), generator=gen, device="cuda")
    logits = torch.randn((M, K), generator=gen, device="cuda") * 3
    if K > 1:
        ids[:, 1] = torch.where(torch.rand(M, generator=gen, device="cuda") < 0.3, ids[:, 0], ids[:, 1])
        ids[torch.rand((M, K), generator=gen, device="cuda") < 0.2] = -1
        logits[torch.rand((M, K), generator=gen, device="cuda") < 0.1] = -math.inf
    if empty:
        rows = torch.rand(M, generator=gen, device="cuda") < 0.3
        ids[rows] = torch.tensor([-100, V, V + 5, -1], device="cuda")[torch.randint(0, 4, (int(rows.sum()), K), generator=gen, device="cuda")]
        if K > 1 and M > 4:
            logits[M // 2] = -math.inf
    return (ids if long else ids.int()), logits


class Ref:
    """The definition in float64, and bounds of what float32 makes of it."""

    def __init__(self, x, w, ids, logits, temperature):
        V, k = w.shape
        ids = ids.view(len(x), -1).long()
        there = (ids >= 0) & (ids < V)
        if logits is not None:
            there &= logits > -math.inf
        self.there, self.any = there, there.any(1)
        xd, wd = torch.where(self.any[:, None], x.double(), 0.0), w.double()
        self.xd, self.wd, self.t = xd, wd, temperature
        self.s = xd @ wd.t() / temperature
        self.s_err = (k + 8) * 2 * E * (xd.abs() @ wd.abs().t()) / temperature + 2 * E * self.s.abs()
        self.lse = torch.logsumexp(self.s, 1, keepdim=True)
        self.lse_err = self.s_err.amax(1, keepdim=True) + (64 + V / 512) * E + 6 * E * (1 + self.s.abs().amax(1, keepdim=True) + self.lse.abs())
        self.at = torch.where(there, ids, 0)
        K = ids.shape[1]
        if logits is None:
            self.q, self.log_q, self.q_rel = there.double(), torch.zeros_like(ids).double(), torch.zeros(len(x), 1, device="cuda")
        else:
            a = torch.where(there, logits.double() / temperature, -1e300)
            self.log_q = torch.where(there, torch.log_softmax(a, 1), 0.0)
            self.q = torch.where(there, self.log_q.exp(), 0.0)
            self.q_rel = (K + 20) * E + 8 * E * torch.where(there, a.abs(), 0.0).amax(1, keepdim=True)
        self.mine, self.mine_err = (torch.where(there, t.gather(1, self.at), 0.0) for t in (self.s, self.s_err))

    def loss(self):
        each = self.q * (self.log_q + self.lse - self.mine)
        size = self.q * (self.log_q.abs() + self.lse.abs() + self.mine.abs())
        err = (self.q * (self.lse_err + self.mine_err) + (self.q_rel + (self.q.shape[1] + 8) * E) * size + self.q * self.q_rel).sum(1)
        return each.sum(1), err

    def backward(self, dloss, dtype):
        g = torch.where(self.any, dloss.double(), 0.0)[:, None] / self.t
        p = (self.s - self.lse).exp()
        p_err = p * (self.s_err + 8 * E * (1 + self.s.abs() + self.lse.abs()) + 2 * E * self.lse.abs())
        ds = p.clone()
        ds.scatter_add_(1, self.at, -self.q)
        q = torch.zeros_like(p).scatter_add_(1, self.at, self.q)
        err = p_err + q * (self.q_rel + (self.q.shape[1] + 4) * E) + 4 * E * (p + q)
        ds, err = ds * g, err * g.abs()
        held = err + _half(dtype) * (ds.abs() + err) + 3e-38     # (bfloat16 parts of a float32 end at the normal numbers)
        sums = lambda a, b, n: (a.abs() @ b.abs()) * (n + 16) * 2 * E  # noqa: E731
        return (ds @ self.wd, held @ self.wd.abs() + sums(ds, self.wd, ds.shape[1])), (ds.t() @ self.xd, held.t() @ self.xd.abs() + sums(ds.t(), self.xd, len(ds)))


def _check(shape, dtype, K, temperature, empty, add, seed, odd, backward=True, repeat=False):
    from paper_2504_05638_amd import train
    M, D, V = shape
    ids, logits = _terms(M, V, K or 1, seed, empty, long=not odd)
    logits = logits if K else None
    x, w = _randn((M, D), seed + 1, dtype, 1.0, 3 * odd, odd), _randn((V, D), seed + 2, dtype, 3 * D ** -0.5, 5 * odd, 3 * odd)
    ref = Ref(x, w, ids, logits, temperature)
    x[~ref.any] = float("nan")      # (rows without a term are not looked at)
    if K:
        loss, saved = train.distill(x, w, ids, logits, temperature=temperature, save=True)
    else:
        ids = ids[:, 0].contiguous()
        loss, saved = train.cross_entropy(x, w, ids, save=True)
    want, err = ref.loss()
    _near(loss, want, err, torch.float32, ("loss", shape))
    _near(saved[:, :1], ref.lse * ref.any[:, None], ref.lse_err, torch.float32, ("lse", shape))
    _near(saved[:, 1:], ref.mine, ref.mine_err, torch.float32, ("scores", shape))
    assert not loss[~ref.any].any() and not saved[~ref.any].any()
    if not backward:
        return
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed + 7)
    dloss = torch.randn(M, generator=gen, device="cuda") if not odd else torch.full((1,), 1.0 / M, device="cuda")
    bucket = _randn((1, 7 + V * D + 5), seed + 5, dtype)[0]
    was = bucket.clone()
    dw = bucket[7:7 + V * D].view(V, D)
    saved = torch.cat([torch.where(ref.any[:, None], ref.lse, 0.0), ref.mine], 1).float()
    call = lambda: (train.distill_backward(dloss, x, w, ids, logits, saved, temperature=temperature, dw=dw, accumulate=add) if K  # noqa: E731
                    else train.cross_entropy_backward(dloss, x, w, ids, saved, dw=dw, accumulate=add))
    dx = call()
    (rx, ex), (rw, ew) = ref.backward(dloss.expand(M), dtype)
    _near(dx, rx, ex, dtype, ("dx", shape))
    assert not dx[~ref.any].any()
    if add:
        rw = rw + was[7:7 + V * D].view(V, D).double()
    _near(dw, rw, ew + 2 * E * rw.abs(), dtype, ("dw", shape))
    assert torch.equal(bucket[:7], was[:7]) and torch.equal(bucket[-5:], was[-5:])
    if repeat:
        first = bucket.clone()
        bucket.copy_(was)
        assert torch.equal(call(), dx) and torch.equal(bucket, first)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_cross_entropy(shape, dtype):
    for i in range(4):
        print("[case] cross entropy", shape, dtype, i, flush=True)
        _check(shape, T[dtype], 0, 1.0, i % 2 == 1, i >= 2, 10 * i, i in (1, 2), repeat=i == 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_distill(shape, dtype):
    for i, (K, temperature) in enumerate([(1, 1.0), (2, 3.0), (17, 2.0), (100, 0.7)]):
        print("[case] distill", shape, dtype, K, flush=True)
        _check(shape, T[dtype], K, temperature, i % 2 == 1, i >= 2, 10 * i, i in (1, 2), repeat=i == 2)


def test_most_terms():
    _check((19, 40, 3001), torch.bfloat16, 1024, 1.5, True, False, 3, 0)


@pytest.mark.parametrize("K", [4, 5, 33])
@pytest.mark.parametrize("shape", [(40, 24, 262_144), (40, 24, 262_177), (1500, 72, 1000)], ids=str)
def test_terms_listed_and_looked_for(shape, K):
    """On both sides of the terms, and of the vocabulary, up to which they are listed by strips."""
    print("[case] terms", shape, K, flush=True)
    _check(shape, torch.bfloat16, K, 1.0, True, False, 61, K == 5)


def test_terms_in_one_place():
    """All rows' terms in one strip, or all of them one token."""
    from paper_2504_05638_amd.train import distill
    M, D, V, K = 1300, 64, 9000, 128
    x, w = _randn((M, D), 71, torch.bfloat16), _randn((V, D), 72, torch.bfloat16, D ** -0.5)
    gen = torch.Generator(device="cuda").manual_seed(73)
    logits = torch.randn((M, K), generator=gen, device="cuda")
    for ids in (torch.randint(8970, 9000, (M, K), generator=gen, device="cuda"), torch.full((M, K), 8999, device="cuda"), torch.zeros((M, K), dtype=torch.int64, device="cuda")):
        loss, saved = distill(x, w, ids, logits, save=True)
        ref = Ref(x, w, ids, logits, 1.0)
        _near(loss, *ref.loss(), torch.float32, "loss")
        _near(saved[:, 1:], ref.mine, ref.mine_err, torch.float32, "scores")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pieces_of_the_vocabulary_backward(dtype):
    """ds of 65536 rows: some thousand tokens at a time."""
    print("[case] pieces, backward", dtype, flush=True)
    _check((65536, 40, 5003), T[dtype], 0, 1.0, True, True, 1, 0)


@pytest.mark.parametrize("shape,dtype", [((1400, 2001, 60_001), "f32"), ((300, 4001, 70_001), "bf16")], ids=str)
def test_pieces_of_the_vocabulary_forward(shape, dtype):
    """Weights that have to be laid out, more than a piece of them."""
    print("[case] pieces, forward", shape, dtype, flush=True)
    _check(shape, T[dtype], 0, 1.0, True, False, 1, 0, backward=dtype == "bf16")


def test_few_rows_over_pieces_of_the_vocabulary():
    """Each piece's scores as parts of sums, those of the last piece cut in their own way."""
    _check((60, 4096, 26000), torch.float32, 0, 1.0, True, True, 41, 0, repeat=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_tiles(dtype):
    print("[case] large tiles", dtype, flush=True)
    _check((4001, 1032, 4120), T[dtype], 3, 1.0, False, True, 1, 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(16, 64, 8192), (64, 200, 4096), (1000, 72, 4096)], ids=str)
def test_a_vocabulary_of_whole_rounds(shape, dtype):
    for K in (0, 7):
        _check(shape, T[dtype], K, 1.0, True, False, 81, 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(3001, 1031, 901), (2100, 2056, 300), (70, 41, 300)], ids=str)
def test_dx_of_a_small_vocabulary(shape, dtype):
    """Whole sums of tiles, rows without terms among the others; into a view, whose surroundings stay."""
    from paper_2504_05638_amd.train import cross_entropy, cross_entropy_backward
    _check(shape, T[dtype], 0, 1.0, True, False, 51, 1)
    M, D, V = shape
    ids = _terms(M, V, 1, 52, True)[0][:, 0].contiguous()
    x, w, one = _randn((M, D), 53, T[dtype]), _randn((V, D), 54, T[dtype], D ** -0.5), torch.ones((), device="cuda")
    _, saved = cross_entropy(x, w, ids, save=True)
    want = cross_entropy_backward(one, x, w, ids, saved)
    room = torch.full((M, D + 9), 7.0, device="cuda", dtype=T[dtype])
    cross_entropy_backward(one, x, w, ids, saved, dx=room[:, 5:5 + D])
    assert torch.equal(room[:, 5:5 + D], want) and (room[:, :5] == 7).all() and (room[:, 5 + D:] == 7).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_without_any_term(dtype):
    """No row counts: losses 0, dx 0, dw 0 or as it was."""
    from paper_2504_05638_amd.train import cross_entropy, cross_entropy_backward
    for M in (1, 40, 300):
        x, w = torch.full((M, 64), float("nan"), device="cuda", dtype=T[dtype]), _randn((333, 64), 1, T[dtype])
        t = torch.full((M,), -100, device="cuda")
        loss, saved = cross_entropy(x, w, t, save=True)
        assert not loss.any() and not saved.any()
        dw = torch.ones_like(w)
        dx = cross_entropy_backward(torch.ones(M, device="cuda"), x, w, t, saved, dw=dw, accumulate=True)
        assert not dx.any() and torch.equal(dw, torch.ones_like(w))
        cross_entropy_backward(torch.ones(M, device="cuda"), x, w, t, saved, dw=dw)
        assert not dw.any()


def test_no_rows_and_shapes():
    from paper_2504_05638_amd.train import cross_entropy, cross_entropy_backward
    w = _randn((50, 16), 1, torch.float32)
    x, t = torch.empty(0, 16, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda")
    loss, saved = cross_entropy(x, w, t, save=True)
    assert loss.shape == (0,) and saved.shape == (0, 2)
    dw = torch.ones_like(w)
    cross_entropy_backward(torch.empty(0, device="cuda"), x, w, t, saved, dw=dw, accumulate=True)
    assert float(dw.sum()) == dw.numel()
    cross_entropy_backward(torch.empty(0, device="cuda"), x, w, t, saved, dw=dw)
    assert not dw.any()
    from paper_2504_05638_amd import binding as B
    for dtype, width in ((torch.float32, 16), (torch.bfloat16, 15)):     # nothing but a result: zeros
        dw = torch.ones((50, width), device="cuda", dtype=dtype)
        a = B.tagc_loss_grad(rows=0, in_=width, vocab=50, terms=1, dtype=int(dtype == torch.bfloat16), temperature=1.0, dw=dw.data_ptr(), lddw=width)
        ws = torch.empty(B.tagc_loss_backward_workspace(a), dtype=torch.uint8, device="cuda")
        B.tagc_loss_backward(a, ws.data_ptr(), torch.cuda.current_stream().cuda_stream)
        assert not dw.any()
    x, t = _randn((6, 16), 2, torch.float32), torch.arange(6, device="cuda")
    want, _ = cross_entropy(x, w, t)
    got, _ = cross_entropy(x.view(2, 3, 16), w, t.view(2, 3))
    assert got.shape == (2, 3) and torch.equal(got.view(6), want)
    one, _ = cross_entropy(x[4], w, t[4])
    assert one.shape == () and abs(float(one) - float(want[4])) < 1e-5


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_far_apart(dtype):
    """Scores of some thousands: exponentials only against the largest; a row that is certain has loss 0 and no gradient."""
    from paper_2504_05638_amd.train import cross_entropy, cross_entropy_backward
    x, w = _randn((70, 64), 1, T[dtype], 40.0), _randn((300, 64), 2, T[dtype], 20.0)
    s = x.double() @ w.double().t()
    t = s.argmax(1)
    loss, saved = cross_entropy(x, w, t, save=True)
    ref = Ref(x, w, t, None, 1.0)
    _near(loss, *ref.loss(), torch.float32, "loss")
    assert float(s.abs().max()) > 5000
    dx = cross_entropy_backward(torch.ones((), device="cuda"), x, w, t, saved)
    top = s.topk(2, dim=1).values
    sure = top[:, 0] - top[:, 1] > 120      # the others' share is under float32's numbers
    assert sure.any() and float(dx[sure].abs().max()) <= 2 * 70 * float(w.abs().max()) * float(ref.lse_err.max() + ref.s_err.max())


@pytest.mark.parametrize("temperature", [1.0, 0.5, 30.0])
@pytest.mark.parametrize("shape", [(50, 64, 300), (1100, 64, 300), (1100, 64, 7700)], ids=str)
def test_a_teachers_mask_of_the_lowest_value(shape, temperature):
    """Where all of a row's logits are float32's lowest value their shares are alike, as of any other equal ones; beside others they
    have none.  (What is added for such a term is less than 10^-34, which no sum of float32 here takes notice of: equal results.)"""
    from paper_2504_05638_amd.train import distill, distill_backward
    M, D, V = shape
    x, w = _randn((M, D), 1, torch.bfloat16), _randn((V, D), 2, torch.bfloat16, D ** -0.5)
    ids, logits = _terms(M, V, 9, 3, True)
    least = torch.finfo(torch.float32).min
    some = torch.rand(logits.shape, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda") < 0.4
    some[:, 0] = False
    ids[:, 0] = ids[:, 0].clamp(0, V - 1)           # (each row has a term that is not masked so)
    logits[:, 0] = logits[:, 0].clamp(min=-9.0)
    masked, plain = logits.masked_fill(some, least), logits.masked_fill(some, -math.inf)
    masked[::7], plain[::7] = least, 0.0
    (got, saved), (want, other) = (distill(x, w, ids, t, temperature=temperature, save=True) for t in (masked, plain))
    assert torch.isfinite(want).all() and torch.equal(got, want) and torch.equal(saved[:, 0], other[:, 0])
    one = torch.ones((), device="cuda")
    dw, dwant = torch.empty_like(w), torch.empty_like(w)
    dx = distill_backward(one, x, w, ids, masked, saved, temperature=temperature, dw=dw)
    assert torch.equal(dx, distill_backward(one, x, w, ids, plain, other, temperature=temperature, dw=dwant)) and torch.equal(dw, dwant)


def test_not_finite_rows_stay_where_they_are():
    from paper_2504_05638_amd.train import cross_entropy
    x, w, t = _randn((40, 96), 1, torch.float32), _randn((200, 96), 2, torch.float32), torch.arange(40, device="cuda")
    good, _ = cross_entropy(x, w, t)
    x[3, 5], x[30, 95] = float("nan"), float("inf")
    loss, _ = cross_entropy(x, w, t)
    keep = torch.ones(40, dtype=torch.bool, device="cuda")
    keep[[3, 30]] = False
    assert torch.equal(loss[keep], good[keep]) and not torch.isfinite(loss[[3, 30]]).any()
    w[7, 1] = float("-inf")      # a token that no row can have, or that is infinitely likely
    assert not torch.isfinite(cross_entropy(x, w, t)[0]).any()


@pytest.mark.parametrize("K", [0, 5])
def test_gradient_against_differences(K):
    from paper_2504_05638_amd import train
    M, D, V, h, temperature = 5, 33, 41, 2.0 ** -5, 1.0 if not K else 2.0
    ids, logits = _terms(M, V, K or 1, 3, False)
    x, w, c = _randn((M, D), 1, torch.float32), _randn((V, D), 2, torch.float32, D ** -0.5), torch.rand(M, device="cuda") + 0.5
    if K:
        call = lambda save: train.distill(x, w, ids, logits, temperature=temperature, save=save)  # noqa: E731
    else:
        ids = ids[:, 0].contiguous()
        call = lambda save: train.cross_entropy(x, w, ids, save=save)  # noqa: E731
    _, saved = call(True)
    dw = torch.empty_like(w)
    dx = (train.distill_backward(c, x, w, ids, logits, saved, temperature=temperature, dw=dw) if K
          else train.cross_entropy_backward(c, x, w, ids, saved, dw=dw))
    for t, grad, places in ((x, dx, [(0, 0), (4, 32), (2, 11)]), (w, dw, [(0, 0), (40, 32), (int(ids.view(-1)[0]), 5)])):
        for at in places:
            was = t[at].item()
            side = []
            for sign in (1, -1):
                t[at] = was + sign * h
                side.append(float((call(False)[0].double() * c.double()).sum()))
            t[at] = was
            # a log-sum's third derivative is at most 1.5 times the largest change of a score cubed (4 a unit of w, 1 of x); rounding 2^-19 a row
            assert abs((side[0] - side[1]) / (2 * h) - grad[at].item()) < 1.5 * 1.5 * M * 64 * h * h / 6 * 0.1 + 1.5 * M * 2.0 ** -19 / h, at
