"""Tensors of a device that is not the current one.  There is one device here: another one is made out to be the current one, and
what is asked is that every call of the library is made with the tensors' own."""
import pytest
import torch

pytestmark = pytest.mark.gpu

CALLS = ["tagc_linear_forward_workspace", "tagc_linear_forward", "tagc_linear_backward_workspace", "tagc_linear_backward", "tagc_optim_upload",
         "tagc_grad_norm", "tagc_adamw_step", "tagc_adamw_unpack"]


def test_calls_are_made_with_the_tensors_device(monkeypatch):
    from paper_2504_05638_amd import train
    on, made = [7], []

    class Device:
        def __init__(self, device):
            self.index = torch.device(device).index

        def __enter__(self):
            on.append(self.index)

        def __exit__(self, *a):
            on.pop()

    x, w, dy = torch.randn(70, 30, device="cuda"), torch.randn(20, 30, device="cuda"), torch.randn(70, 20, device="cuda")
    g = torch.randn(500, device="cuda")
    monkeypatch.setattr(train, "_current_device", lambda: on[-1])
    monkeypatch.setattr(torch.cuda, "device", Device)
    for name in CALLS:
        call = getattr(train.B, name)
        monkeypatch.setattr(train.B, name, lambda *a, call=call, name=name: (made.append((name, on[-1])), call(*a))[1])
    y, _ = train.linear(x, w)
    dx = train.linear_backward(dy, x, w, dw=torch.empty_like(w))
    opt = train.AdamW(params=[torch.zeros_like(g)], grads=[g], bits=8)
    opt.grad_norm()
    opt.step()
    opt.unpack()
    assert on == [7]
    assert sorted({n for n, _ in made}) == sorted(CALLS) and {d for _, d in made} == {x.device.index}
    monkeypatch.undo()
    assert torch.equal(y, train.linear(x, w)[0]) and torch.equal(dx, train.linear_backward(dy, x, w))


def test_a_stream_of_another_device_is_refused():
    from paper_2504_05638_amd.train import AdamW, linear, linear_backward

    class Other:
        device, cuda_stream = torch.device("cuda", 1), 0

    x, w = torch.randn(70, 30, device="cuda"), torch.randn(20, 30, device="cuda")
    opt = AdamW(params=[w.clone()], grads=[w])
    for call in (lambda s: linear(x, w, out=torch.empty(70, 20, device="cuda"), stream=s),
                 lambda s: linear_backward(torch.randn(70, 20, device="cuda"), x, w, dx=torch.empty_like(x), stream=s),
                 lambda s: opt.grad_norm(stream=s), lambda s: opt.step(1, stream=s), lambda s: opt.unpack(stream=s)):
        with pytest.raises(ValueError, match="device"):
            call(Other())
