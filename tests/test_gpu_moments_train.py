"""Training with 8-bit moments against training with 32-bit ones.

A code's neighbours are an eighth of it or less apart and rounding is unbiased: the error of an element's m is a random walk with
steps of at most 0.125 / sqrt(6) of it and a decay of 0.1 a step, about 0.12; v, which moves by 0.05 a step, is rounded
with a chance of half at most, 0.125 / 2 / sqrt(2 * 0.05), 0.2, of which the root takes half.  An update is so off by some 0.16
of itself, and elements and steps independently of one another: the mean goes where float32's goes, and the square grows by
0.025.  A loss that falls by gradients like these may differ by a few times that; a quarter is allowed at every tenth step, on losses
that fall by a factor of ten and more."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_losses_fall_alike(dtype):
    from paper_2504_05638_amd.train import AdamW, linear, linear_backward
    gen = torch.Generator(device="cuda")
    gen.manual_seed(11)
    M, K, H, N, steps = 512, 96, 256, 48, 150
    x = torch.randn(M, K, generator=gen, device="cuda").to(dtype)
    true = torch.randn(N, K, generator=gen, device="cuda") * K ** -0.5
    target = torch.tanh(x.float() @ true.t())
    start = [torch.randn(s, generator=gen, device="cuda") * s[-1] ** -0.5 for s in ((H, K), (N, H))]
    losses = {}
    for bits in (32, 8):
        params = [p.clone() for p in start] + [torch.zeros(H, device="cuda"), torch.zeros(N, device="cuda")]
        used = params if dtype == torch.float32 else [p.to(dtype) for p in params]
        grads = [torch.zeros_like(u) for u in used]
        opt = AdamW(params=params, grads=grads, copies=None if dtype == torch.float32 else used, betas=(0.9, 0.95), bits=bits, max_norm=10.0,
                    groups=[(2e-3, 0.01)], seed=3)
        out = []
        for _ in range(steps):
            h, pre = linear(x, used[0], used[2], activation="gelu", save=True)
            y, _ = linear(h, used[1], used[3])
            off = y.float() - target
            out.append(off.square().mean())
            dh = linear_backward((off * (2.0 / off.numel())).to(dtype), h, used[1], dw=grads[1], db=grads[3])
            linear_backward(dh, x, used[0], pre, activation="gelu", dw=grads[0], db=grads[2], need_dx=False)
            opt.grad_norm()
            opt.step()
        losses[bits] = torch.stack(out).cpu()
        assert opt.control[:3].tolist() == [steps, 0, 1]
    a, b = losses[32], losses[8]
    assert a[-1] < 0.1 * a[0] and b[-1] < 0.1 * b[0], (a[-1], b[-1], a[0])
    for i in range(0, steps, 10):
        assert abs(float(b[i] / a[i]) - 1) < 0.25, (i, float(a[i]), float(b[i]))
