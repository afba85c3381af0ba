"""Calls on a given stream: what they make is that stream's memory, and what they keep is not reused under them.

The allocator hands out memory of the current stream's that is free there, which says only that the current
stream's later work may use it: another stream that writes it at once meets what is still running."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _owner(address):
    """The stream whose memory an address is, as the allocator has it."""
    for segment in torch.cuda.memory_snapshot():
        if segment["address"] <= address < segment["address"] + segment["total_size"]:
            return segment["stream"]
    raise AssertionError("not the allocator's")


@pytest.fixture
def side():
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    yield s
    s.synchronize()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_layers_make_the_streams_own_memory(dtype, side, monkeypatch):
    from paper_2504_05638_amd import train
    # (odd features in, so that bfloat16 operands are laid out in the workspace; tiles enough that float32 ones are)
    x, w = torch.randn(2700, 101, device="cuda").to(dtype), torch.randn(2650, 101, device="cuda").to(dtype)
    dy, dw, db = torch.randn(2700, 2650, device="cuda").to(dtype), torch.empty_like(w), torch.empty(2650, device="cuda", dtype=dtype)
    torch.cuda.synchronize()
    used = []
    for name in ("tagc_linear_forward", "tagc_linear_backward"):
        call = getattr(train.B, name)
        monkeypatch.setattr(train.B, name, lambda a, at, on, call=call: (used.append((at, on)), call(a, at, on))[1])
    y, pre = train.linear(x, w, activation="silu", save=True, stream=side)
    dx = train.linear_backward(dy, x, w, pre, activation="silu", dw=dw, db=db, stream=side)
    assert len(used) == 2 and all(at and on == side.cuda_stream for at, on in used)
    for address in [at for at, _ in used] + [y.data_ptr(), pre.data_ptr(), dx.data_ptr()]:
        assert _owner(address) == side.cuda_stream
    side.synchronize()
    want, z = train.linear(x, w, activation="silu", save=True)
    assert torch.equal(y, want) and torch.equal(pre, z)
    assert _owner(want.data_ptr()) == torch.cuda.current_stream().cuda_stream
    ew, eb = torch.empty_like(dw), torch.empty_like(db)
    ex = train.linear_backward(dy, x, w, z, activation="silu", dw=ew, db=eb)
    assert torch.equal(dx, ex) and torch.equal(dw, ew) and torch.equal(db, eb)


def test_unpacked_moments_are_the_streams_own_memory(side):
    from paper_2504_05638_amd.train import AdamW
    opt = AdamW(params=[torch.zeros(5000, device="cuda")], grads=[torch.randn(5000, device="cuda")], bits=8)
    opt.step(1)
    side.wait_stream(torch.cuda.current_stream())
    m, v = opt.unpack(stream=side)
    assert _owner(m.data_ptr()) == _owner(v.data_ptr()) == side.cuda_stream
    side.synchronize()
    em, ev = opt.unpack()
    assert torch.equal(m, em) and torch.equal(v, ev)


def test_a_result_is_kept_for_the_stream_that_has_it(side):
    """A result that is dropped while the current stream still reads it is not handed out on `side` again."""
    from paper_2504_05638_amd.train import linear
    x, w = torch.ones(64, 256, device="cuda"), torch.ones(512, 256, device="cuda")
    torch.cuda.synchronize()
    y, _ = linear(x, w, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    a = torch.randn(4096, 4096, device="cuda")
    for _ in range(20):
        a = a @ a * 1e-3
    late = y.clone()        # behind a few ms of products
    was = y.data_ptr()
    del y
    with torch.cuda.stream(side):
        again = torch.empty(64, 512, device="cuda")
    busy = not torch.cuda.current_stream().query()
    assert not busy or again.data_ptr() != was
    torch.cuda.synchronize()
    assert torch.equal(late, torch.full_like(late, 256.0))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("given", [True, False])
def test_an_optimizer_dropped_early_keeps_its_memory(bits, given, side):
    """Table, control block and moments of an optimizer that goes while another stream has yet to run its step."""
    from paper_2504_05638_amd.train import AdamW
    n = 3_000_000
    grads, params = [torch.randn(n, device="cuda")], [torch.zeros(n, device="cuda")]
    a = torch.randn(4096, 4096, device="cuda")
    opt = AdamW(params=params, grads=grads, bits=bits, groups=[(1e-2, 0.0)])
    parts = [opt.table, opt.control, *opt.m, *opt.v, *(opt.bases or [])]
    held = [(t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in parts]
    sizes = [t.numel() * t.element_size() for t in parts]
    with torch.cuda.stream(side):
        for _ in range(20):
            a = a @ a * 1e-3        # a few ms
    if given:
        opt.grad_norm(stream=side)
        opt.step(stream=side)
    else:
        with torch.cuda.stream(side):
            opt.grad_norm()
            opt.step()
    del opt, parts
    new = [torch.empty(k, dtype=torch.uint8, device="cuda") for k in sizes for _ in range(4)]
    if not side.query():
        for t in new:
            assert not any(lo <= t.data_ptr() < hi for lo, hi in held)
    side.synchronize()
    assert torch.allclose(params[0], -1e-2 * grads[0] / (grads[0].abs() + 1e-8), atol=1e-5)
