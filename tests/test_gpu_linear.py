"""Linear layers against float64: forward and backward, both types, every activation, odd sizes, strides,
offsets and alignments, from one row on.

Bounds per element, with e = 2^-24: a float32 sum of k products is within (k + 8) 2 e of the sum of the
products' magnitudes, which also covers the 2^-23 that taking float32 operands apart leaves out; no activation's
slope exceeds 1.13; its own evaluation is within 2^-20 (1 + |z|); a bfloat16 result is rounded by 2^-8 at
most (half an ulp below the next power of two)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]
T = {"f32": torch.float32, "bf16": torch.bfloat16}
SHAPES = [(1, 1, 1), (1, 4096, 1000), (2, 777, 333), (3, 64, 5), (4, 130, 64), (5, 64, 64), (17, 100, 31), (64, 256, 64),
          (129, 65, 130), (128, 128, 128), (200, 1000, 300), (333, 777, 1001), (1000, 64, 520), (2048, 512, 2304), (16, 4096, 640)]


def _act(z, kind):
    if kind == "relu":
        return z.clamp(min=0)
    if kind == "gelu":
        return 0.5 * z * torch.erfc(-z / math.sqrt(2))
    if kind == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if kind == "silu":
        return z * torch.sigmoid(z)
    return z


def _randn(shape, seed, dtype, scale=1.0, ld_more=0, shift=0):
    """A matrix whose rows lie ld_more elements apart, shift elements into its buffer."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    m, n = shape
    buf = torch.full((m * (n + ld_more) + shift,), float("nan"), device="cuda", dtype=dtype)
    t = buf[shift:].view(m, n + ld_more)[:, :n]
    t.copy_(torch.randn(m, n, generator=gen, device="cuda") * scale)
    return t


def _half(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else E


def _forward_ref(x, w, b, r, act):
    xd, wd = x.double(), w.double()
    z = xd @ wd.t() + (0 if b is None else b.double())
    size = xd.abs() @ wd.abs().t() + (0 if b is None else b.double().abs())
    err = (x.shape[1] + 8) * 2 * E * size
    y = _act(z, act) + (0 if r is None else r.double())
    y_err = 1.13 * err + (0 if act in ("none", "relu") else 2.0 ** -20 * (1 + z.abs())) + 2 * E * y.abs()
    return z, err, y, y_err


def _near(got, ref, err, dtype, what):
    off = (got.double() - ref).abs()
    bound = err + _half(dtype) * (ref.abs() + err)
    assert torch.isfinite(got).all(), what
    assert torch.all(off <= bound + 1e-40), (what, float((off - bound).max()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward(shape, dtype):
    from paper_2504_05638_amd.train import linear
    M, K, N = shape
    t = T[dtype]
    for i, act in enumerate(ACTS):
        odd = i % 2
        print("[case] forward", shape, dtype, act, flush=True)
        x = _randn((M, K), 1 + i, t, ld_more=3 * odd, shift=odd)
        w = _randn((N, K), 2 + i, t, K ** -0.5, ld_more=5 * odd, shift=3 * odd)
        b = _randn((1, N), 3 + i, t)[0] if i != 3 else None
        r = _randn((M, N), 4 + i, t, ld_more=odd) if i in (1, 2) else None
        out = _randn((M, N), 9, t, ld_more=2 * odd, shift=odd) if odd else None
        save = i != 4
        y, pre = linear(x, w, b, r, activation=act, save=save, out=out)
        torch.cuda.synchronize()
        assert out is None or y is out
        z, z_err, ref, err = _forward_ref(x, w, b, r, act)
        _near(y, ref, err, t, act)
        if save:
            _near(pre, z, z_err, t, "pre")
        else:
            assert pre is None


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_backward(shape, dtype):
    from paper_2504_05638_amd.train import linear_backward
    M, K, N = shape
    t = T[dtype]
    for i, act in enumerate(ACTS):
        odd, add = i % 2, i in (1, 4)
        print("[case] backward", shape, dtype, act, flush=True)
        x = _randn((M, K), 1 + i, t, ld_more=odd, shift=odd)
        w = _randn((N, K), 2 + i, t, K ** -0.5, ld_more=2 * odd)
        dy = _randn((M, N), 3 + i, t, ld_more=3 * odd, shift=odd)
        pre = _randn((M, N), 4 + i, t, 2.0, ld_more=odd) if act != "none" else None
        # a place in a bucket's flat gradient, at an odd offset, between things that stay
        bucket = _randn((1, 7 + N * K + N + 5), 5, t)[0]
        was = bucket.clone()
        dw, db = bucket[7:7 + N * K].view(N, K), bucket[7 + N * K:7 + N * K + N]
        dx = linear_backward(dy, x, w, pre, activation=act, dw=dw, db=db, accumulate=add)
        torch.cuda.synchronize()
        s, slope_err = torch.ones((), device="cuda", dtype=torch.float64), 0.0
        if act == "relu":
            s = (pre > 0).double()      # 0 at 0, as the operator's slope is defined (clamp's is 1 there)
        elif act != "none":
            z = pre.double().requires_grad_()
            (s,) = torch.autograd.grad(_act(z, act).sum(), z)
            slope_err = 2.0 ** -20 * (1 + pre.double().abs())
        dz = dy.double() * s
        dz_err = dy.double().abs() * slope_err + 2 * E * dz.abs()
        held = dz_err + (_half(t) * dz.abs() if act != "none" else 0)     # rounded before the products
        wd, xd = w.double(), x.double()
        _near(dx, dz @ wd, held @ wd.abs() + (N + 8) * 2 * E * (dz.abs() @ wd.abs()), t, "dx")
        old = was.double() if add else torch.zeros_like(was).double()
        ref = dz.t() @ xd + old[7:7 + N * K].view(N, K)
        _near(dw, ref, held.t() @ xd.abs() + (M + 8) * 2 * E * (dz.abs().t() @ xd.abs()) + 2 * E * ref.abs(), t, "dw")
        ref = dz.sum(0) + old[7 + N * K:7 + N * K + N]
        _near(db, ref, dz_err.sum(0) + (M + 8) * 2 * E * dz.abs().sum(0) + 2 * E * ref.abs(), t, "db")
        assert torch.equal(bucket[:7], was[:7]) and torch.equal(bucket[-5:], was[-5:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(4001, 4006, 4003), (3904, 4096, 4160)], ids=str)
def test_large_tiles(shape, dtype):
    """Sizes at which every product, forward and backward, takes the large tiles, with and without laying operands out."""
    from paper_2504_05638_amd.train import linear, linear_backward
    M, K, N = shape
    t = T[dtype]
    x, w, b, dy = _randn((M, K), 1, t), _randn((N, K), 2, t, K ** -0.5), _randn((1, N), 3, t)[0], _randn((M, N), 4, t)
    y, pre = linear(x, w, b, activation="silu", save=True)
    z, z_err, ref, err = _forward_ref(x, w, b, None, "silu")
    _near(y, ref, err, t, "y")
    _near(pre, z, z_err, t, "pre")
    del y, z, z_err, ref, err
    dw, db = torch.empty_like(w), torch.empty_like(b)
    dx = linear_backward(dy, x, w, dw=dw, db=db)
    dz, xd, wd = dy.double(), x.double(), w.double()
    _near(dx, dz @ wd, (N + 8) * 2 * E * (dz.abs() @ wd.abs()), t, "dx")
    _near(dw, dz.t() @ xd, (M + 8) * 2 * E * (dz.abs().t() @ xd.abs()), t, "dw")
    _near(db, dz.sum(0), (M + 8) * 2 * E * dz.abs().sum(0), t, "db")


# float32 rows end inside, at and behind a slab of the product, one or many slabs to a tile; the last shape has tiles enough to be
# laid out beforehand
@pytest.mark.parametrize("shape", [(m, k, n) for k in (1, 31, 32, 33, 63, 65, 97, 161, 1537) for m, n in ((17, 130), (130, 200))] + [(2700, 100, 2650)], ids=str)
def test_float32_rows_ending_anywhere(shape):
    from paper_2504_05638_amd.train import linear
    M, K, N = shape
    print("[case] float32 rows", shape, flush=True)
    x, w = _randn((M, K), 5, torch.float32, ld_more=5, shift=3), _randn((N, K), 6, torch.float32, ld_more=1)
    _, _, ref, err = _forward_ref(x, w, None, None, "none")
    _near(linear(x, w)[0], ref, err, torch.float32, shape)


@pytest.mark.parametrize("act", ACTS)
def test_gradient_against_differences(act):
    """d(sum(c * y)) / dw, dx, db by central differences of the library's own forward in float32."""
    from paper_2504_05638_amd.train import linear, linear_backward
    M, K, N, h = 7, 33, 19, 2.0 ** -6
    x, w, b = (_randn(s, 20 + i, torch.float32) for i, s in enumerate([(M, K), (N, K), (1, N)]))
    w.mul_(K ** -0.5)
    b = b[0]
    c = _randn((M, N), 30, torch.float32)
    _, pre = linear(x, w, b, activation=act, save=True)
    if act == "relu":   # (no kink within a step of the differences)
        b = b + torch.where((pre.abs() < 0.2).any(0), 9.0, 0.0)
        _, pre = linear(x, w, b, activation=act, save=True)
        assert float(pre.abs().min()) > 0.1
    dw, db = torch.empty_like(w), torch.empty_like(b)
    dx = linear_backward(c, x, w, pre if act != "none" else None, activation=act, dw=dw, db=db)
    for t, grad, places in ((w, dw, [(0, 0), (18, 32), (7, 11)]), (x, dx, [(0, 0), (6, 32), (3, 9)]), (b, db, [(0,), (18,)])):
        for at in places:
            was = t[at].item()
            side = []
            for sign in (1, -1):
                t[at] = was + sign * h
                side.append(float((linear(x, w, b, activation=act)[0].double() * c.double()).sum()))
            t[at] = was
            # third derivatives are under 2.5 a value of z, moved by at most |x| h < 4 h, over M or N values of |c| < 4;
            # the sums' own rounding is 2 E * K * M * N / h at most
            bound = 2.5 * 64 * h * h / 6 * 4 * max(M, N) * 0.1 + 2 * E * K * M * N / h
            assert abs((side[0] - side[1]) / (2 * h) - grad[at].item()) < bound, (act, at)


def test_float32_is_float32():
    """Rounding errors of sums of 2048 products, as a 2-norm: far below what bfloat16 (1e-3) or two parts of
    each operand (2^-16) would leave."""
    from paper_2504_05638_amd.train import linear
    x, w = _randn((500, 2048), 1, torch.float32), _randn((600, 2048), 2, torch.float32)
    y, _ = linear(x, w)
    ref = x.double() @ w.double().t()
    assert float((y.double() - ref).norm() / ref.norm()) < 2e-6


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_wide_range_and_not_finite(dtype):
    from paper_2504_05638_amd.train import linear, linear_backward
    t = T[dtype]
    for M in (3, 40):
        x, w = _randn((M, 96), 1, t), _randn((70, 96), 2, t)
        x[0] *= 1e30
        x[1] *= 1e-30
        y, _ = linear(x, w)
        z, _, ref, err = _forward_ref(x, w, None, None, "none")
        _near(y, ref, err, t, "range")
        x[2, 5], w[9, 3] = float("inf"), float("nan")
        y, _ = linear(x, w, activation="relu")
        torch.cuda.synchronize()
        bad = torch.zeros(M, 70, dtype=torch.bool, device="cuda")
        bad[:, 9] = True
        assert torch.isnan(y[:, 9]).all()
        bad[2] = True
        assert torch.isfinite(y[~bad]).all()
        assert (~torch.isfinite(y[2]) | (y[2] == 0)).all()   # (relu of minus infinity is 0)
        dx = linear_backward(_randn((M, 70), 3, t), x, w, need_dx=True)
        assert torch.isnan(dx[:, 3]).all() and torch.isfinite(dx[:, 4]).all()


def test_large_values_of_the_argument():
    from paper_2504_05638_amd.train import linear, linear_backward
    z = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 5.0, -5.0, 20.0, -20.0, 90.0, -90.0, 1e4, -1e4, 1e30, -1e30, 3e38, -3e38], device="cuda")
    one = torch.ones(1, 1, device="cuda")
    for act in ACTS:
        y, pre = linear(z.view(-1, 1), one, activation=act, save=True)
        dx = linear_backward(torch.ones_like(y), z.view(-1, 1), one, pre if act != "none" else None, activation=act)
        assert torch.equal(pre.view(-1), z)
        big = z.abs() > 50
        assert torch.equal(y.view(-1)[big], z[big].clamp(min=0) if act != "none" else z[big]), act
        assert torch.equal(dx.view(-1)[big], (z[big] > 0).float() if act != "none" else torch.ones_like(z[big])), act
        assert torch.isfinite(y).all() and torch.isfinite(dx).all(), act


def test_empty_sides():
    from paper_2504_05638_amd.train import linear, linear_backward
    for t in T.values():
        for M, K, N in ((0, 8, 8), (5, 0, 8), (40, 0, 9), (5, 8, 0)):
            x, w, b = torch.ones(M, K, device="cuda", dtype=t), torch.ones(N, K, device="cuda", dtype=t), torch.full((N,), 2.0, device="cuda", dtype=t)
            y, pre = linear(x, w, b, activation="relu", save=True)
            assert y.shape == (M, N) and torch.equal(y, x.sum(1, keepdim=True) + b) and torch.equal(pre, y)
            dw, db = torch.full((N, K), 7.0, device="cuda", dtype=t), torch.full((N,), 7.0, device="cuda", dtype=t)
            dy = torch.ones(M, N, device="cuda", dtype=t)
            dx = linear_backward(dy, x, w, dw=dw, db=db)
            assert torch.equal(dx, dy @ w if N else torch.zeros(M, K, device="cuda", dtype=t))
            assert torch.equal(dw, torch.full((N, K), float(M), device="cuda", dtype=t))
            assert torch.equal(db, torch.full((N,), float(M), device="cuda", dtype=t))
            dx = linear_backward(dy, x, w, dw=dw, db=db, accumulate=True)
            assert torch.equal(db, torch.full((N,), 2.0 * M, device="cuda", dtype=t))


def test_parts_of_the_gradient_and_leading_dimensions():
    from paper_2504_05638_amd.train import linear, linear_backward
    x = _randn((6, 64), 1, torch.bfloat16).view(2, 3, 64)
    w = _randn((32, 64), 2, torch.bfloat16)
    y, _ = linear(x, w)
    assert y.shape == (2, 3, 32)
    dy = _randn((6, 32), 3, torch.bfloat16).view(2, 3, 32)
    dw, db = torch.zeros_like(w), torch.zeros(32, device="cuda", dtype=torch.bfloat16)
    dx = linear_backward(dy, x, w, dw=dw, db=db)
    assert dx.shape == x.shape
    only = torch.zeros_like(w)
    assert linear_backward(dy, x, w, dw=only, need_dx=False) is None and torch.equal(only, dw)
    only = torch.zeros_like(db)
    linear_backward(dy, x, w, db=only, need_dx=False)
    assert torch.equal(only, db)
    assert torch.equal(linear_backward(dy, x, w), dx)


def test_residual_in_place_and_repeatable():
    from paper_2504_05638_amd.train import linear
    for t in T.values():
        x, w = _randn((300, 640), 1, t), _randn((200, 640), 2, t)
        r = _randn((300, 200), 3, t)
        want, _ = linear(x, w, residual=r)
        again, _ = linear(x, w, residual=r)
        inplace, _ = linear(x, w, residual=r, out=r)
        assert torch.equal(want, again) and torch.equal(want, inplace) and inplace is r


def test_more_than_32_bits_of_results():
    from paper_2504_05638_amd.train import linear
    M, K, N = 66_000, 64, 65_664
    x, w = _randn((M, K), 1, torch.bfloat16), _randn((N, K), 2, torch.bfloat16, 0.125)
    y, _ = linear(x, w)
    for rows in (slice(0, 40), slice(M // 2, M // 2 + 40), slice(M - 40, M)):
        z, _, ref, err = _forward_ref(x[rows], w, None, None, "none")
        _near(y[rows], ref, err, torch.bfloat16, rows)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_replayed_from_a_graph_on_another_stream(dtype):
    from paper_2504_05638_amd.train import linear, linear_backward
    t = T[dtype]
    x, w, b = _randn((70, 200), 1, t), _randn((130, 200), 2, t, 0.1), _randn((1, 130), 3, t)[0]
    dy = _randn((70, 130), 4, t)
    dw, db = torch.zeros_like(w), torch.zeros_like(b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        y, pre = linear(x, w, b, activation="silu", save=True)
        dx = linear_backward(dy, x, w, pre, activation="silu", dw=dw, db=db, accumulate=True)
    for rep in range(3):
        x.copy_(_randn((70, 200), 10 + rep, t))
        dw.fill_(1.0)
        db.fill_(1.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        ew, eb = torch.ones_like(w), torch.ones_like(b)
        ey, ep = linear(x, w, b, activation="silu", save=True)
        ex = linear_backward(dy, x, w, ep, activation="silu", dw=ew, db=eb, accumulate=True)
        torch.cuda.synchronize()
        for got, want in ((y, ey), (pre, ep), (dx, ex), (dw, ew), (db, eb)):
            assert torch.equal(got, want)


def test_given_stream():
    from paper_2504_05638_amd.train import linear
    x, w = _randn((200, 100), 1, torch.float32), _randn((64, 100), 2, torch.float32)
    want, _ = linear(x, w)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got, _ = linear(x, w, stream=s)
    s.synchronize()
    assert torch.equal(want, got)


def test_refusals():
    from paper_2504_05638_amd.train import linear, linear_backward
    x, w = torch.zeros(4, 8, device="cuda"), torch.zeros(6, 8, device="cuda")
    dy = torch.zeros(4, 6, device="cuda")
    for args, kw in (((x.cpu(), w), {}), ((x.half(), w.half()), {}), ((x, w.t()), {}), ((x, w.bfloat16()), {}), ((x, w[:, :7]), {}),
                     ((x, w, torch.zeros(5, device="cuda")), {}), ((x, w, None, torch.zeros(4, 5, device="cuda")), {}),
                     ((x, w), dict(activation="swish")), ((x, w), dict(out=torch.zeros(6, 4, device="cuda").t())),
                     ((x, w), dict(pre=torch.zeros(4, 6, device="cuda"))), ((x.t().contiguous().t(), w), {})):
        with pytest.raises(ValueError):
            linear(*args, **kw)
    for args, kw in (((dy, x, w), dict(activation="relu")), ((dy, x, w, dy), {}), ((dy[:3], x, w), {}),
                     ((dy, x, w), dict(dw=torch.zeros(8, 6, device="cuda"))), ((dy, x, w), dict(need_dx=False, dx=x)),
                     ((dy, x, w), dict(db=torch.zeros(6, device="cuda", dtype=torch.bfloat16)))):
        with pytest.raises(ValueError):
            linear_backward(*args, **kw)
