"""Token embeddings against float64: lookups, and the table's gradient with its sorting, at sizes around what is not sorted
(128 tokens), a chunk of what is (4096) and a piece of summed tokens (8 or 32).

Bounds, with E = 2^-24: a lookup is one multiplication and one addition, a gradient's row of n tokens n additions, and half a step of
the result's type."""
import pytest
import torch

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
T = {"f32": torch.float32, "bf16": torch.bfloat16}


def _randn(shape, seed, dtype, scale=1.0, ld_more=0, shift=0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    m, n = shape
    buf = torch.full((m * (n + ld_more) + shift,), float("nan"), device="cuda", dtype=dtype)
    t = buf[shift:].view(m, n + ld_more)[:, :n]
    t.copy_(torch.randn(m, n, generator=gen, device="cuda") * scale)
    return t


def _ids(n, vocab, seed, kind):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    if kind == "one":
        return torch.full((n,), vocab - 1, device="cuda")
    if kind == "few":
        return torch.randint(0, min(3, vocab), (n,), generator=gen, device="cuda") * (vocab // 3 if vocab >= 3 else 0)
    ids = torch.randint(0, vocab, (n,), generator=gen, device="cuda")
    if kind == "none among them":
        ids[torch.rand(n, generator=gen, device="cuda") < 0.4] = -1
        ids[::7] = vocab
        if n > 3:
            ids[3] = 1 << 40
    if kind == "none":
        ids.fill_(-100)
    return ids


KINDS = ["any", "one", "few", "none among them", "none"]


def _half(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else E


def _near(got, ref, err, dtype, what):
    off = (got.double() - ref).abs()
    bound = err + _half(dtype) * (ref.abs() + err)
    assert torch.isfinite(got).all(), what
    assert torch.all(off <= bound + 1e-40), (what, float((off - bound).max()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("width", [1, 5, 8, 64, 333, 768, 1024, 1025, 2047, 2048, 2056, 4099])
def test_lookup(width, dtype):
    from paper_2504_05638_amd.train import embedding
    t = T[dtype]
    for i, (n, vocab) in enumerate([(1, 1), (3, 10), (130, 77), (1000, 5000)]):
        for kind in KINDS:
            odd = (i + len(kind)) % 2
            print("[case] lookup", dtype, width, n, vocab, kind, flush=True)
            ids = _ids(n, vocab, i, kind)
            ids = ids if kind == "none among them" or i % 2 else ids.int()
            table = _randn((vocab, width), 1, t, ld_more=3 * odd, shift=odd)
            res = _randn((n, width), 2, t, ld_more=odd, shift=3 * odd) if i != 1 else None
            out = _randn((n, width), 3, t, ld_more=5 * odd, shift=odd) if odd else None
            y = embedding(ids, table, scale=1.7, residual=res, out=out)
            assert out is None or y is out
            there = (ids >= 0) & (ids < vocab)
            part = table[torch.where(there, ids, 0).long()].double() * float(torch.tensor(1.7)) * there[:, None]
            ref = part + (res.double() if res is not None else 0)
            _near(y, ref, E * part.abs() + E * ref.abs(), t, kind)
    if dtype == "f32":
        y = embedding(torch.zeros((2, 3), dtype=torch.int32, device="cuda"), table)
        assert y.shape == (2, 3, width) and torch.equal(y, table[:1].expand(6, width).reshape(2, 3, width))


def test_lookup_in_the_residuals_place():
    from paper_2504_05638_amd.train import embedding
    table, res, ids = _randn((50, 300), 1, torch.bfloat16), _randn((40, 300), 2, torch.bfloat16), _ids(40, 50, 3, "any")
    want = embedding(ids, table, residual=res)
    assert embedding(ids, table, residual=res, out=res) is res and torch.equal(res, want)


def _gradient(n, vocab, width, dtype, kind, add, seed, odd):
    from paper_2504_05638_amd.train import embedding_backward
    ids = _ids(n, vocab, seed, kind)
    ids = ids if odd or kind == "none among them" else ids.int()
    dy = _randn((n, width), seed + 1, dtype, ld_more=3 * odd, shift=odd)
    # a place in a flat gradient, at an odd offset, between things that stay
    bucket = _randn((1, 5 + vocab * width + 4), seed + 2, dtype)[0]
    was = bucket.clone()
    dtable = bucket[5:5 + vocab * width].view(vocab, width)
    embedding_backward(dy, ids, dtable, scale=0.3, accumulate=add)
    there = (ids >= 0) & (ids < vocab)
    at, rows = ids[there].long(), dy[there].double()
    s = float(torch.tensor(0.3))
    ref = torch.zeros(vocab, width, device="cuda", dtype=torch.float64).index_add_(0, at, rows) * s
    size = torch.zeros(vocab, width, device="cuda", dtype=torch.float64).index_add_(0, at, rows.abs()) * s
    count = torch.bincount(at, minlength=vocab)[:, None].double()
    old = was[5:5 + vocab * width].view(vocab, width)
    if add:
        ref = ref + old.double()
    _near(dtable, ref, (count + 2) * E * size + E * ref.abs(), dtype, (n, vocab, width, kind))
    untouched = count[:, 0] == 0
    assert torch.equal(dtable[untouched], old[untouched] if add else torch.zeros_like(old[untouched]))
    assert torch.equal(bucket[:5], was[:5]) and torch.equal(bucket[-4:], was[-4:])
    bucket.copy_(was)
    first = dtable.clone()
    embedding_backward(dy, ids, dtable, scale=0.3, accumulate=add)
    second = dtable.clone()
    bucket.copy_(was)
    embedding_backward(dy, ids, dtable, scale=0.3, accumulate=add)
    assert torch.equal(second, dtable) and first.shape == second.shape


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", KINDS)
def test_gradient(kind, dtype):
    for i, (n, vocab, width) in enumerate([(1, 1, 1), (1, 40, 64), (15, 7, 33), (16, 100, 8), (17, 3, 130), (64, 64, 64), (65, 1000, 5), (333, 50, 777), (128, 40, 2049), (129, 40, 33),
                                           (1023, 5000, 256), (4095, 300, 40), (4096, 301, 64), (4097, 302, 72), (9000, 20000, 32), (13000, 9, 2050)]):
        print("[case] embedding gradient", kind, dtype, n, vocab, width, flush=True)
        _gradient(n, vocab, width, T[dtype], kind, i % 3 == 1, 3 * i, i % 2)


def test_long_batches():
    for n, vocab, width in ((16384, 700, 40), (16385, 701, 33), (70_000, 50257, 64), (200_001, 1000, 24)):
        print("[case] embedding gradient, long", n, vocab, width, flush=True)
        _gradient(n, vocab, width, torch.bfloat16, "none among them", False, 1, 1)


def test_no_tokens():
    from paper_2504_05638_amd.train import embedding, embedding_backward
    table, ids = torch.ones(5, 9, device="cuda"), torch.empty((0,), dtype=torch.int64, device="cuda")
    assert embedding(ids, table).shape == (0, 9)
    embedding_backward(torch.empty(0, 9, device="cuda"), ids, table, accumulate=True)
    assert float(table.sum()) == 45.0
    embedding_backward(torch.empty(0, 9, device="cuda"), ids, table)
    assert float(table.abs().sum()) == 0.0


def test_not_finite_rows_of_no_token_stay_out():
    from paper_2504_05638_amd.train import embedding_backward
    dy = torch.ones(100, 40, device="cuda")
    ids = torch.arange(100, device="cuda") % 7
    ids[::10] = -1
    dy[::10] = float("nan")
    dtable = torch.empty(7, 40, device="cuda")
    embedding_backward(dy, ids, dtable)
    assert torch.equal(dtable, torch.bincount(ids[ids >= 0], minlength=7)[:, None].float().expand(7, 40))


def _checked_and_repeated(n, vocab, width, dtype, kind, add):
    """The result that is compared with float64 is what a second call makes, too, bit for bit; what lies around it stays."""
    from paper_2504_05638_amd.train import embedding_backward
    ids, dy = _ids(n, vocab, 5, kind), _randn((n, width), 6, dtype)
    bucket = _randn((1, 5 + vocab * width + 4), 7, dtype)[0]
    was = bucket.clone()
    dtable, old = bucket[5:5 + vocab * width].view(vocab, width), was[5:5 + vocab * width].view(vocab, width)
    embedding_backward(dy, ids, dtable, accumulate=add)
    first = bucket.clone()
    bucket.copy_(was)
    embedding_backward(dy, ids, dtable, accumulate=add)
    assert torch.equal(bucket, first) and torch.equal(bucket[:5], was[:5]) and torch.equal(bucket[-4:], was[-4:])
    there = (ids >= 0) & (ids < vocab)
    at, rows = ids[there], dy[there].double()
    count = torch.bincount(at, minlength=vocab)[:, None].double()

    def sums(t):        # (float64's additions to one place go one behind the other: a hundred thousand take half a minute)
        out = torch.zeros(vocab, width, device="cuda", dtype=torch.float64)
        if kind not in ("one", "few"):
            return out.index_add_(0, at, t)
        for v in at.unique().tolist():
            out[v] = t[at == v].sum(0)
        return out

    ref, size = sums(rows), sums(rows.abs())
    if add:
        ref = ref + old.double()
    _near(dtable, ref, (count + 2) * E * size + E * ref.abs(), dtype, (n, vocab, width, kind))
    untouched = count[:, 0] == 0
    assert torch.equal(dtable[untouched], old[untouched] if add else torch.zeros_like(old[untouched]))


@pytest.mark.parametrize("add", [False, True], ids=["written", "added"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", KINDS)
def test_what_is_checked_repeats(kind, dtype, add):
    """One launch, one chunk, a list merged of chunks, one of merged lists; zeros beside the sort, and behind it (from 16385 tokens on)."""
    for n, vocab, width in ((100, 64, 70), (3000, 900, 130), (9000, 20000, 32), (16384, 700, 40), (16385, 701, 33), (70_000, 50257, 24), (150_001, 1000, 9)):
        print("[case] embedding gradient, repeated", kind, dtype, add, n, vocab, width, flush=True)
        _checked_and_repeated(n, vocab, width, T[dtype], kind, add)
