"""Norms against float64, forward and backward: both kinds and types, widths around every way a row is held, odd
strides, offsets and alignments.

Bounds, with E = 2^-24: a row's sums are taken by threads of at most 32 elements, then through at most 22 more additions: within
64 E of the sum of magnitudes.  Each other operation adds E (root and quotient 4 E) of what it makes.  A result is rounded by half a
step of its type."""
import pytest
import torch

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
T = {"f32": torch.float32, "bf16": torch.bfloat16}
WIDTHS = [1, 2, 7, 8, 9, 64, 333, 511, 512, 513, 768, 1023, 1024, 1025, 2047, 2048, 2050, 4095, 4096, 4099, 8192, 8193, 11008, 16383, 16384]


def _randn(shape, seed, dtype, scale=1.0, ld_more=0, shift=0, mean=0.0):
    """A matrix whose rows lie ld_more elements apart, shift elements into its buffer, NaN between them."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    m, n = shape
    buf = torch.full((m * (n + ld_more) + shift,), float("nan"), device="cuda", dtype=dtype)
    t = buf[shift:].view(m, n + ld_more)[:, :n]
    t.copy_(torch.randn(m, n, generator=gen, device="cuda") * scale + mean)
    return t


def _half(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else E


def _near(got, ref, err, dtype, what):
    off = (got.double() - ref).abs()
    bound = err + _half(dtype) * (ref.abs() + err)
    assert torch.isfinite(got).all(), what
    assert torch.all(off <= bound + 1e-40), (what, float((off - bound).max()))


def _stats(x, kind, eps):
    """(mean, r) in float64 and bounds of their errors."""
    x = x.double()
    mean, mean_err = torch.zeros_like(x[:, :1]), torch.zeros_like(x[:, :1])
    if kind == "layer":
        mean = x.mean(1, keepdim=True)
        mean_err = 65 * E * x.abs().mean(1, keepdim=True)
    z = x - mean
    z_err = mean_err + E * z.abs()
    var = z.square().mean(1, keepdim=True)
    var_err = (2 * z.abs() * z_err + z_err * z_err).mean(1, keepdim=True) + 66 * E * var
    r = (var + eps) ** -0.5
    r_rel = 0.5 * var_err / (var + eps - var_err).clamp(min=1e-300) + 10 * E
    return mean, mean_err, z, z_err, r, r_rel


def _forward(shape, dtype, kind, affine, seed, odd):
    from paper_2504_05638_amd.train import norm
    M, D = shape
    x = _randn((M, D), seed, dtype, 2.0, 3 * odd, odd, mean=0.5)
    w = _randn((1, D), seed + 1, dtype, 0.2, shift=odd, mean=1.0)[0] if affine else None
    b = _randn((1, D), seed + 2, dtype, 0.2, shift=3 * odd)[0] if affine and kind == "layer" else None
    out = _randn((M, D), seed + 3, dtype, ld_more=5 * odd, shift=odd) if odd else None
    y, stats = norm(x, w, b, kind=kind, eps=1e-5, save=True, out=out)
    assert out is None or y is out
    mean, mean_err, z, z_err, r, r_rel = _stats(x, kind, 1e-5)
    wd = w.double() if affine else torch.ones(D, device="cuda", dtype=torch.float64)
    ref = z * r * wd + (b.double() if b is not None else 0)
    err = (wd * r).abs() * z_err * (1 + r_rel) + (z * r * wd).abs() * (r_rel + 4 * E) + 2 * E * ref.abs()
    _near(y, ref, err, dtype, (shape, kind))
    _near(stats[:, :1], mean, mean_err + 1e-12, torch.float32, "mean")
    _near(stats[:, 1:], r, r * r_rel, torch.float32, "r")
    again, none = norm(x, w, b, kind=kind, eps=1e-5)
    assert none is None and torch.equal(again, y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_forward(kind, dtype):
    for i, D in enumerate(WIDTHS):
        for M in (1, 3, 70):
            print("[case] norm", kind, dtype, M, D, flush=True)
            _forward((M, D), T[dtype], kind, (i + M) % 3 > 0, 10 * i, (i + M) % 2)


def _backward(shape, dtype, kind, affine, residual, add, seed, odd):
    from paper_2504_05638_amd.train import norm_backward
    M, D = shape
    layer = kind == "layer"
    x = _randn((M, D), seed, dtype, 2.0, 3 * odd, odd, mean=0.5)
    w = _randn((1, D), seed + 1, dtype, 0.2, shift=odd, mean=1.0)[0] if affine else None
    dy = _randn((M, D), seed + 2, dtype, 1.0, odd, 3 * odd)
    res = _randn((M, D), seed + 3, dtype, 1.0, 2 * odd) if residual else None
    mean, _, _, _, r, _ = _stats(x, kind, 1e-5)
    stats = torch.cat([mean, r], 1).float().contiguous()
    bucket = _randn((1, 2 * D + 9), seed + 4, dtype)[0]
    was = bucket.clone()
    dw, db = bucket[5:5 + D], bucket[5 + D:5 + 2 * D] if layer else None
    dx = norm_backward(dy, x, w, stats, kind=kind, residual=res, dw=dw, db=db, accumulate=add)
    mean, r = stats[:, :1].double(), stats[:, 1:].double()
    xd, g, wd = x.double(), dy.double(), (w.double() if affine else torch.ones(D, device="cuda", dtype=torch.float64))
    h, u = (xd - mean) * r, g * wd
    h_err = 3 * E * (xd - mean).abs() * r
    u_err = E * u.abs()
    s1 = u.mean(1, keepdim=True) if layer else torch.zeros_like(mean)
    s1_err = 66 * E * u.abs().mean(1, keepdim=True) if layer else 0
    s2 = (u * h).mean(1, keepdim=True)
    s2_err = (u.abs() * h_err + 68 * E * (u * h).abs()).mean(1, keepdim=True)
    ref = r * (u - s1 - h * s2)
    err = r * (u_err + s1_err + h_err * (s2.abs() + s2_err) + h.abs() * s2_err + 4 * E * (u.abs() + s1.abs() + (h * s2).abs()))
    if residual:
        ref = ref + res.double()
    _near(dx, ref, err + 2 * E * ref.abs(), dtype, ("dx", shape, kind))
    old = was.double() if add else torch.zeros_like(was).double()
    ref = (g * h).sum(0) + old[5:5 + D]
    _near(dw, ref, (g.abs() * h_err).sum(0) + (M + 40) * E * (g * h).abs().sum(0) + 2 * E * ref.abs(), dtype, ("dw", shape, kind))
    if layer:
        ref = g.sum(0) + old[5 + D:5 + 2 * D]
        _near(db, ref, (M + 40) * E * g.abs().sum(0) + 2 * E * ref.abs(), dtype, ("db", shape, kind))
    assert torch.equal(bucket[:5], was[:5]) and torch.equal(bucket[5 + (1 + layer) * D:], was[5 + (1 + layer) * D:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_backward(kind, dtype):
    for i, D in enumerate(WIDTHS):
        for M in (1, 3, 70):
            print("[case] norm_backward", kind, dtype, M, D, flush=True)
            _backward((M, D), T[dtype], kind, (i + M) % 3 > 0, i % 2 == 0, (i + M) % 4 == 1, 10 * i, (i + M) % 2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_many_rows(kind, dtype):
    """More rows than workgroups take at once."""
    for M, D in ((9001, 130), (5003, 1100), (2500, 8200)):
        print("[case] many rows", kind, dtype, M, D, flush=True)
        _forward((M, D), T[dtype], kind, True, 5, 1)
        _backward((M, D), T[dtype], kind, True, True, True, 6, 1)


def test_more_rows_than_a_launch_takes():
    from paper_2504_05638_amd.train import norm
    M = (1 << 21) + 3
    x = torch.randn(M, 2, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    y, stats = norm(x, save=True)
    for part in (slice(0, 9), slice((1 << 21) - 4, M)):
        few, also = norm(x[part].contiguous(), save=True)
        assert torch.equal(y[part], few) and torch.equal(stats[part], also)


def test_rows_far_from_zero():
    """A mean a thousand times the spread: the variance is that of what is left, not a difference of sums."""
    from paper_2504_05638_amd.train import norm
    x = _randn((40, 768), 1, torch.float32, 1.0, mean=1000.0)
    y, stats = norm(x, save=True)
    z = x.double() - x.double().mean(1, keepdim=True)
    # the mean is off by at most 65 E of 1000, which is 0.004 of the spread, the variance by that squared, and z by it
    assert float((y.double() - z / (z.square().mean(1, keepdim=True) + 1e-5).sqrt()).abs().max()) < 65 * E * 1000 * 1.2
    one = torch.full((3, 100), 7.25, device="cuda")
    y, stats = norm(one, save=True)     # nothing but the mean: zeros, r = 1 / sqrt(eps)
    assert torch.equal(y, torch.zeros_like(y)) and torch.allclose(stats[:, 1], torch.full((3,), 1e-5 ** -0.5, device="cuda"), rtol=1e-6)


def test_not_finite_rows_stay_where_they_are():
    from paper_2504_05638_amd.train import norm, norm_backward
    for D in (100, 1500, 9000):
        x = _randn((9, D), 1, torch.float32)
        good, _ = norm(x)
        x[2, 5], x[7, D - 1] = float("nan"), float("inf")
        y, stats = norm(x, save=True)
        keep = torch.tensor([0, 1, 3, 4, 5, 6, 8], device="cuda")
        assert torch.equal(y[keep], good[keep]) and torch.isnan(y[[2, 7]]).any(1).all()
        dx = norm_backward(torch.ones_like(x), x, None, stats)
        assert torch.isfinite(dx[keep]).all() and torch.isnan(dx[[2, 7]]).any(1).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_few_rows_and_more(kind, dtype):
    """On both sides of the number of rows up to which dw and db are made beside dx."""
    for i, (M, D) in enumerate([(511, 260), (512, 67), (513, 260), (512, 1031), (512, 5), (512, 8200), (200, 16384)]):
        print("[case] few rows", kind, dtype, M, D, flush=True)
        _backward((M, D), T[dtype], kind, i % 3 > 0, i % 2 == 0, i % 4 == 1, 10 * i, i % 2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_few_rows_in_place(dtype):
    """dx over dy or x, whose dw and db are made of what was there before."""
    from paper_2504_05638_amd.train import norm, norm_backward
    M, D = 300, 700
    x, dy, w = _randn((M, D), 1, T[dtype], 2.0), _randn((M, D), 2, T[dtype]), _randn((1, D), 3, T[dtype])[0]
    _, stats = norm(x, w, save=True)
    want = norm_backward(dy, x, w, stats)
    g, h = dy.double(), (x.double() - stats[:, :1].double()) * stats[:, 1:].double()
    for place in (None, "dy", "x"):
        a, b, dw, db = dy.clone(), x.clone(), torch.empty_like(w), torch.empty_like(w)
        dx = norm_backward(a, b, w, stats, dw=dw, db=db, dx={"dy": a, "x": b}.get(place))
        assert torch.equal(dx, want), place
        _near(dw, (g * h).sum(0), (M + 43) * E * (g * h).abs().sum(0), T[dtype], ("dw", place))
        _near(db, g.sum(0), (M + 40) * E * g.abs().sum(0), T[dtype], ("db", place))


def test_in_place_and_shapes():
    from paper_2504_05638_amd.train import norm, norm_backward
    x, w = _randn((30, 700), 1, torch.bfloat16), _randn((1, 700), 2, torch.bfloat16)[0]
    y, stats = norm(x, w, kind="rms", save=True)
    y3, _ = norm(x.view(5, 6, 700), w, kind="rms")
    assert y3.shape == (5, 6, 700) and torch.equal(y3.view(30, 700), y)
    y1, s1 = norm(x[4], w, kind="rms", save=True)
    assert y1.shape == (700,) and torch.equal(y1, y[4]) and torch.equal(s1, stats[4:5])
    z = x.clone()
    assert norm(z, w, kind="rms", out=z)[0] is z and torch.equal(z, y)
    dy, res = _randn((30, 700), 3, torch.bfloat16), _randn((30, 700), 4, torch.bfloat16)
    dx = norm_backward(dy, x, w, stats, kind="rms", residual=res)
    for which in range(3):
        a = [dy.clone(), x.clone(), res.clone()]
        assert torch.equal(norm_backward(a[0], a[1], w, stats, kind="rms", residual=a[2], dx=a[which]), dx)
    dw = torch.empty_like(w)
    assert norm_backward(dy, x, w, stats, kind="rms", dw=dw, need_dx=False) is None
    full = torch.empty_like(w)
    norm_backward(dy, x, w, stats, kind="rms", dw=full)
    assert torch.equal(dw, full)


def test_no_rows():
    from paper_2504_05638_amd.train import norm, norm_backward
    x, w = torch.empty(0, 50, device="cuda"), torch.ones(50, device="cuda")
    y, stats = norm(x, w, w, save=True)
    assert y.shape == (0, 50) and stats.shape == (0, 2)
    dw, db = torch.ones(50, device="cuda"), torch.ones(50, device="cuda")
    norm_backward(x, x, w, stats, dw=dw, db=db, accumulate=True)
    assert float(dw.sum() + db.sum()) == 100.0
    norm_backward(x, x, w, stats, dw=dw, db=db)
    assert float(dw.abs().sum() + db.abs().sum()) == 0.0


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_gradient_against_differences(kind):
    """d(sum(c * y)) / dx, dw, db by central differences of the library's own forward."""
    from paper_2504_05638_amd.train import norm, norm_backward
    M, D, h = 4, 37, 2.0 ** -6
    x, w, b, c = (_randn(s, 20 + i, torch.float32) for i, s in enumerate([(M, D), (1, D), (1, D), (M, D)]))
    w, b = w[0], b[0] if kind == "layer" else None
    _, stats = norm(x, w, b, kind=kind, save=True)
    dw, db = torch.empty_like(w), torch.empty_like(w) if kind == "layer" else None
    dx = norm_backward(c, x, w, stats, kind=kind, dw=dw, db=db)
    for t, grad, places in ((x, dx, [(0, 0), (3, 36), (2, 11)]), (w, dw, [(0,), (20,)]), (b, db, [(36,)])):
        if t is None:
            continue
        for at in places:
            was = t[at].item()
            side = []
            for sign in (1, -1):
                t[at] = was + sign * h
                side.append(float((norm(x, w, b, kind=kind)[0].double() * c.double()).sum()))
            t[at] = was
            # third derivatives in x are under 50 for rows of spread 0.7 and more, weights and slopes under 4; the sums' rounding is M D 2^-20 / h
            assert abs((side[0] - side[1]) / (2 * h) - grad[at].item()) < 50 * h * h + M * D * 2.0 ** -20 / h, at
