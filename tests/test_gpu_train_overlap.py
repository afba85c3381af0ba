"""Matrices in one buffer: side by side they are taken, over one another they are refused."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_side_by_side(dtype):
    """x, residual, result and what the activation takes as columns of one buffer, gradients as those of another."""
    from paper_2504_05638_amd.train import linear, linear_backward
    M, K, N = 150, 96, 40
    buf = torch.randn(M, K + 3 * N, device="cuda").to(dtype)
    x, r, y, pre = torch.split(buf, [K, N, N, N], 1)
    w, b = torch.randn(N, K, device="cuda").to(dtype), torch.randn(N, device="cuda").to(dtype)
    keep = [t.clone() for t in (x, r)]
    want, z = linear(*(t.clone() for t in (x, w, b, r)), activation="gelu", save=True)
    got, gz = linear(x, w, b, r, activation="gelu", save=True, out=y, pre=pre)
    assert torch.equal(got, want) and torch.equal(gz, z) and all(torch.equal(a, o) for a, o in zip((x, r), keep))
    dy = torch.randn(M, N, device="cuda").to(dtype)
    both = torch.zeros(M, K + N, device="cuda", dtype=dtype)
    dx, held = torch.split(both, [K, N], 1)
    held.copy_(dy)
    wide = torch.zeros(N, 2 * K, device="cuda", dtype=dtype)
    linear_backward(held, x, w, pre, activation="gelu", dx=dx, dw=wide[:, K:])
    dw = torch.zeros(N, K, device="cuda", dtype=dtype)
    assert torch.equal(linear_backward(dy, x.clone(), w, z, activation="gelu", dw=dw), dx) and torch.equal(wide[:, K:], dw)
    assert torch.equal(held, dy) and not wide[:, :K].any()
    # without an activation what it would take is the result
    y2, p2 = linear(x, w, b, save=True, out=y, pre=y)
    assert p2 is y and torch.equal(y2, linear(x, w, b)[0])


def test_over_one_another():
    from paper_2504_05638_amd.binding import TagcError
    from paper_2504_05638_amd.train import linear, linear_backward
    x, w = torch.randn(64, 48, device="cuda").bfloat16(), torch.randn(48, 48, device="cuda").bfloat16()
    buf = torch.randn(65, 48, device="cuda").bfloat16()
    before = [t.clone() for t in (x, w, buf)]
    for kw in (dict(out=x), dict(residual=buf[:64], out=buf[1:]), dict(save=True, pre=buf[1:], out=buf[:64]), dict(save=True, pre=x)):
        with pytest.raises(TagcError):
            linear(x, w, activation="relu", **kw)
    for kw in (dict(dx=buf[:64]), dict(dx=x, dw=torch.empty_like(w)), dict(dw=w), dict(dx=torch.empty_like(x), db=w[3])):
        with pytest.raises(TagcError):
            linear_backward(buf[1:], x, w, **kw)
    assert all(torch.equal(a, b) for a, b in zip(before, (x, w, buf)))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shift", [0, 1])
def test_in_the_place_of_what_has_been_read(dtype, shift):
    """Behind an activation dx may lie over dy or pre; in float32 gradients may lie over operands."""
    from paper_2504_05638_amd.train import linear_backward
    M, K = 500, 320

    def make():
        gen = torch.Generator(device="cuda")
        gen.manual_seed(4)
        return [torch.randn(n * K + shift, generator=gen, device="cuda").to(dtype)[shift:].view(n, K) for n in (M, M, M, K)]

    def run(place, act):
        dy, pre, x, w = make()
        dx = {"dy": dy, "pre": pre, "x": x, "none": None}[place]
        dw = w if place == "x" else torch.empty_like(w)
        db = torch.empty(K, device="cuda", dtype=dtype)
        return linear_backward(dy, x, w, pre if act else None, activation=act, dx=dx, dw=dw, db=db), dw, db

    want = run("none", "gelu")
    for place in ("dy", "pre"):
        assert all(torch.equal(a, b) for a, b in zip(run(place, "gelu"), want))
    if dtype == torch.float32:
        for act in (None, "silu"):
            assert all(torch.equal(a, b) for a, b in zip(run("x", act), run("none", act)))
