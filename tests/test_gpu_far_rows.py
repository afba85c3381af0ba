"""Norms, embeddings and losses whose rows lie so far apart that offsets pass 32 bits: the same bits as from rows side by side."""
import pytest
import torch

pytestmark = pytest.mark.gpu

N, LD = 70_000, 65_536       # 4.6 G elements from the first row to the last


def _apart(t):
    """The same numbers, LD elements from row to row; what lies between is whatever memory holds."""
    far = torch.empty(len(t) * LD, dtype=t.dtype, device="cuda").view(len(t), LD)[:, 3:3 + t.shape[1]]
    far.copy_(t)
    return far


def _randn(*shape, seed, dtype=torch.bfloat16):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


@pytest.fixture(autouse=True)
def room():
    if torch.cuda.mem_get_info()[1] < 150 << 30:
        pytest.skip("memory of a large card is wanted")
    yield
    torch.cuda.empty_cache()


def test_norm():
    from paper_2504_05638_amd.train import norm, norm_backward
    x, dy, w = _randn(N, 100, seed=1), _randn(N, 100, seed=2), _randn(100, seed=3)
    y, stats = norm(x, w, save=True)
    fx, fy = _apart(x), _apart(dy)
    got, s = norm(fx, w, save=True, out=_apart(x))
    assert torch.equal(got, y) and torch.equal(s, stats)
    dw, want_dw = torch.empty_like(w), torch.empty_like(w)
    want = norm_backward(dy, x, w, stats, dw=want_dw)
    got = norm_backward(fy, fx, w, stats, dx=fy, dw=dw)
    assert torch.equal(got, want) and torch.equal(dw, want_dw)


def test_embedding():
    from paper_2504_05638_amd.train import embedding, embedding_backward
    for width, tokens in ((64, 300), (99, 100), (99, 20_000)):
        table = _randn(N, width, seed=1)
        ids = torch.randint(0, N, (tokens,), generator=torch.Generator(device="cuda").manual_seed(4), device="cuda")
        ids[0], ids[1] = N - 1, N - 1
        far = _apart(table)
        assert torch.equal(embedding(ids, far, scale=2.0), embedding(ids, table, scale=2.0))
        dy = _randn(tokens, width, seed=5)
        want = torch.empty_like(table)
        embedding_backward(dy, ids, want)
        embedding_backward(dy, ids, far)
        assert torch.equal(far, want)
        embedding_backward(dy, ids, want, accumulate=True)
        embedding_backward(dy, ids, far, accumulate=True)
        assert torch.equal(far, want)
        del far


@pytest.mark.parametrize("rows", [5, 300, 1500])
def test_loss_over_far_weights(rows):
    from paper_2504_05638_amd.train import cross_entropy, cross_entropy_backward
    x, w = _randn(rows, 64, seed=1), _randn(N, 64, seed=2)
    t = torch.randint(0, N, (rows,), generator=torch.Generator(device="cuda").manual_seed(4), device="cuda")
    t[0], one = N - 1, torch.ones((), device="cuda")
    near = w.new_empty(N, 72)[:, 3:67]      # (laid out as the far ones are: no row begins at a multiple of four bytes)
    near.copy_(w)
    far, far_dw, dw = _apart(w), _apart(w), torch.empty_like(w)
    loss, saved = cross_entropy(x, near, t, save=True)
    got, s = cross_entropy(x, far, t, save=True)
    assert torch.equal(got, loss) and torch.equal(s, saved)
    dx = cross_entropy_backward(one, x, near, t, saved, dw=dw)
    assert torch.equal(cross_entropy_backward(one, x, far, t, saved, dw=far_dw), dx) and torch.equal(far_dw, dw)


def test_loss_of_far_rows():
    from paper_2504_05638_amd.train import cross_entropy, cross_entropy_backward
    x, w = _randn(N, 64, seed=1), _randn(300, 64, seed=2)
    t = torch.randint(-30, 300, (N,), generator=torch.Generator(device="cuda").manual_seed(4), device="cuda")
    one, far = torch.ones((), device="cuda"), _apart(x)
    loss, saved = cross_entropy(x, w, t, save=True)
    got, s = cross_entropy(far, w, t, save=True)
    assert torch.equal(got, loss) and torch.equal(s, saved)
    dw, far_dw = torch.empty_like(w), torch.empty_like(w)
    dx = cross_entropy_backward(one, x, w, t, saved, dw=dw)
    assert torch.equal(cross_entropy_backward(one, far, w, t, saved, dx=_apart(x), dw=far_dw), dx) and torch.equal(far_dw, dw)
