"""The operators together: layers, exchange and optimizer train a small block, and leave what they should."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("train_block", os.path.join(ROOT, "examples", "train_block.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_the_loss_falls():
    losses = _example().train(steps=40, ranks=3, width=256, rows=128)
    assert all(l == l for l in losses)
    assert losses[-1] < 0.6 * losses[0], losses


def test_the_optimizer_reads_what_the_decoder_wrote():
    """A step from the decoder's dense output is the step from the decoded pairs."""
    from paper_2504_05638_amd import binding as B
    from paper_2504_05638_amd.bucket import TagcBucket
    from paper_2504_05638_amd.train import AdamW, dense_views
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    lengths = [4099, 33, 70_001, 5]
    segments, at = [], 0
    for i, n in enumerate(lengths):
        segments.append((at, n, 50_000, B.TAGC_SEG_COMPRESS if i != 1 else 0))
        at += n
    b = TagcBucket(segments, B.TAGC_F32, 2, sizing_milli=3000, dense=True)
    grads = [torch.randn(at, generator=gen, device="cuda") * 1e-3 for _ in range(2)]
    b.run(grads)
    torch.cuda.synchronize()
    assert b.status()["n_unresolved"] == 0
    views = dense_views(b)
    assert [v is None for v in views] == [False, True, False, False]
    idx, val = b.outputs()
    want = torch.zeros(b.out_dense.view(torch.float32).numel(), device="cuda")
    want[torch.as_tensor(idx.astype("int64"), device="cuda")] = torch.as_tensor(val, device="cuda")
    c = 0
    for n, v in zip(lengths, views):
        if v is None:
            continue
        assert v.numel() == n and torch.equal(v, want[c:c + n])
        c += -(-n // 32) * 32
    used = [v for v in views if v is not None]
    params = [torch.ones(v.numel(), device="cuda") for v in used]
    opt = AdamW(params=params, grads=used, groups=[(0.5, 0.0)], grad_scale=0.5)
    norm, _ = opt.grad_norm()
    opt.step()
    assert abs(float(norm) - 0.5 * float(want.double().norm())) < 1e-6 * float(norm)
    for p, v in zip(params, used):      # the first step goes by the gradient's sign alone; where nothing was sent, nothing moves
        assert torch.equal(p[v == 0], torch.ones_like(p[v == 0]))
        big = v.abs() > 1e-4
        assert torch.allclose(p[big], 1 - 0.5 * torch.sign(v[big]), atol=1e-3)
    b.close()
