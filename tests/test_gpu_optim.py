"""The optimizer behind the exchange against its formulas: norm and control block, AdamW with 32-bit moments
(float64, bounds per element), AdamW with 8-bit moments (codes and bases bit for bit)."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

LENGTHS = [0, 1, 3, 255, 256, 257, 4095, 4096, 4097, 10007, 64, 8192 * 3 + 5]
BETAS, EPS = (0.9, 0.95), 1e-8
GROUPS = [(2e-3, 0.1), (1e-3, 0.0)]
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _mix32(x):
    x = np.asarray(x, np.uint32)
    with np.errstate(over="ignore"):
        x = x ^ (x >> np.uint32(16))
        x = x * np.uint32(0x6A09E667)
        x = x ^ (x >> np.uint32(15))
        x = x * np.uint32(0xBB67AE85)
        return x ^ (x >> np.uint32(16))


def _bits16(tensor, n, seed, step):
    """The 16 + 16 random bits of a tensor's elements, whole blocks."""
    lo, hi = seed & 0xFFFFFFFF, seed >> 32
    with np.errstate(over="ignore"):
        key = _mix32(np.uint32(lo) ^ _mix32(np.uint32(hi) + np.uint32(0x9E3779B9) * np.uint32(step + 1)))
        key = _mix32(np.uint32(tensor) * np.uint32(0x9E3779B9) + key)
    i = np.arange(-(-n // 256) * 256, dtype=np.uint32)
    word = _mix32((i >> np.uint32(2)) ^ key).astype(np.uint64)
    turn = (8 * (i & 3)).astype(np.uint64)
    word = ((word >> turn) | (word << (32 - turn))) & 0xFFFFFFFF
    return (word & 0xFFFF).astype(np.int64), (word >> 16).astype(np.int64)


def _blocks(x):
    out = np.zeros(-(-len(x) // 256) * 256, np.float32)
    out[:len(x)] = x
    return out.reshape(-1, 256)


def _pack(x, u, codes):
    """codes and bases of a moment by the definition, on float32 numbers."""
    x, u = _blocks(x), u.reshape(-1, 256)
    bits = np.abs(x).view(np.int32).astype(np.int64)
    q = np.minimum((bits + 16 * u) >> 20, np.maximum(0x7F7, bits >> 20))
    base = np.maximum(q.max(1, keepdims=True, initial=0) - codes, 0)
    least = ((base + 1) << 20).astype(np.int32).view(np.float32)
    low = x > 0 if codes == 255 else u.astype(np.float32) * np.float32(2 ** -16) * least < np.abs(x)
    return np.where(q > base, q - base, low.astype(np.int64)), base


def _unpack(c, base, n):
    return np.where(c > 0, (c + base) << 20, 0).astype(np.int32).view(np.float32).reshape(-1)[:n]


class Setup:
    """Tensors one behind the other in flat buffers that start `shift` elements in."""

    def __init__(self, lengths, params, grads, bits=32, copies=True, seed=0, shift=1, scale=1.0, **kw):
        from paper_2504_05638_amd.train import AdamW
        self.lengths, self.bits = lengths, bits
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        total = sum(lengths)

        def flat(t):
            buf = torch.zeros(total + shift, device="cuda", dtype=t.dtype)
            buf[shift:] = t
            return list(torch.split(buf[shift:], lengths))

        g = torch.randn(total, generator=gen, device="cuda") * 1e-3 * scale
        g[::7] = 0
        self.grads = flat(g.to(TYPES[grads]))
        self.params = flat((torch.randn(total, generator=gen, device="cuda") * 0.02).to(TYPES[params]))
        self.copies = flat(torch.zeros(total, device="cuda", dtype=torch.bfloat16)) if copies else None
        m0 = torch.randn(total, generator=gen, device="cuda") * 3e-4 * scale
        v0 = torch.rand(total, generator=gen, device="cuda") ** 4 * 1e-6 * scale * scale
        v0[::5] = 0
        if bits == 32:
            self.m, self.v, self.bases = flat(m0), flat(v0), None
        else:
            self.m = flat(torch.randint(0, 256, (total,), generator=gen, device="cuda").to(torch.uint8))
            self.v = flat(torch.randint(0, 256, (total,), generator=gen, device="cuda").to(torch.uint8))
            self.bases = [(torch.full((-(-n // 256),), 780 | 620 << 16, device="cuda", dtype=torch.int32)
                           + torch.randint(0, 60, (-(-n // 256),), generator=gen, device="cuda").int()) for n in lengths]
        self.group_of = [i % 2 for i in range(len(lengths))]
        self.kw = dict(betas=BETAS, eps=EPS, bits=bits, seed=0x123456789ABCDEF, groups=GROUPS, group_of=self.group_of)
        self.kw.update(kw)
        self.opt = AdamW(params=self.params, grads=self.grads, m=self.m, v=self.v, bases=self.bases, copies=self.copies, **self.kw)

    def before(self):
        def n(ts):
            return [t.detach().cpu().float().numpy() if t.dtype != torch.uint8 else t.cpu().numpy() for t in ts]
        return dict(p=n(self.params), g=n(self.grads), m=n(self.m), v=n(self.v),
                    b=[t.cpu().numpy() for t in self.bases] if self.bases else None)


def _host(t):
    return t.detach().cpu().double().numpy()


def _check(s, old, step, factor, lr_scale=1.0):
    """All outputs of one step against the formulas.  Bounds: m and v are two products and a sum, each
    rounded (3 roundings of half an ulp, 2^-24, of what is added); p a product, a quotient and a
    difference: an ulp of p, and 16 ulps of the update (root, two products, sum, quotient, product, and the
    sums in m and v, at most 2 ulps each); bfloat16 half an ulp of its own, 2^-9, on top."""
    e = 2.0 ** -24
    for i, n in enumerate(s.lengths):
        lr, wd = GROUPS[s.group_of[i]]
        lr *= lr_scale
        g = old["g"][i].astype(np.float64) * factor
        if s.bits == 32:
            m0, v0 = old["m"][i].astype(np.float64), old["v"][i].astype(np.float64)
        else:
            b = np.repeat(old["b"][i].astype(np.int64), 256)[:n]
            c, d = old["m"][i].astype(np.int64), old["v"][i].astype(np.int64)
            m0 = _unpack(c & 127, b & 0xFFFF, n).astype(np.float64) * np.where(c > 127, -1, 1)
            v0 = _unpack(d, b >> 16, n).astype(np.float64)
        m = BETAS[0] * m0 + (1 - BETAS[0]) * g
        v = BETAS[1] * v0 + (1 - BETAS[1]) * g * g
        m_err = 4 * e * (np.abs(BETAS[0] * m0) + np.abs((1 - BETAS[0]) * g))
        update = lr / (1 - BETAS[0] ** step) * m / (np.sqrt(v) / math.sqrt(1 - BETAS[1] ** step) + EPS)
        update_err = 16 * e * np.abs(update) + lr / (1 - BETAS[0] ** step) * m_err / (np.sqrt(v) / math.sqrt(1 - BETAS[1] ** step) + EPS)
        p = old["p"][i].astype(np.float64) * (1 - lr * wd) - update
        p_err = 4 * e * np.abs(old["p"][i]) + update_err
        half = 2.0 ** -8 * (np.abs(p) + p_err) if s.params[i].dtype == torch.bfloat16 else 0
        assert np.all(np.abs(_host(s.params[i]) - p) <= p_err + half + 1e-45), i
        if s.copies is not None and s.params[i].dtype == torch.float32:
            assert torch.equal(s.copies[i], s.params[i].to(torch.bfloat16)), i
        if s.bits == 32:
            assert np.all(np.abs(_host(s.m[i]) - m) <= m_err + 1e-45), i
            assert np.all(np.abs(_host(s.v[i]) - v) <= 6 * e * v + 1e-44), i
            continue
        # float32, rounded operation by operation, and the codes exactly
        f = np.float32
        gf = old["g"][i] * f(factor)
        m = m0.astype(f) * f(BETAS[0]) + gf * f(1 - BETAS[0])
        v = v0.astype(f) * f(BETAS[1]) + (gf * gf) * f(1 - BETAS[1])
        um, uv = _bits16(i, n, s.kw["seed"], step)
        mc, mb = _pack(m, um, 127)
        vc, vb = _pack(v, uv, 255)
        sign = (_blocks(m) < 0).astype(np.int64) << 7
        assert np.array_equal(s.m[i].cpu().numpy(), (mc | sign).reshape(-1)[:n].astype(np.uint8)), i
        assert np.array_equal(s.v[i].cpu().numpy(), vc.reshape(-1)[:n].astype(np.uint8)), i
        assert np.array_equal(s.bases[i].cpu().numpy(), (mb | vb << 16).reshape(-1).astype(np.int32)), i


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("params,grads", [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("shift", [0, 1])
def test_step_against_the_formulas(bits, params, grads, shift):
    s = Setup(LENGTHS, params, grads, bits, grad_scale=1 / 3, shift=shift, seed=bits + shift)
    for step in (1, 2, 1000):
        old = s.before()
        s.opt.step(step)
        torch.cuda.synchronize()
        _check(s, old, step, np.float32(1 / 3))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("max_norm", [0.0, 1e-4, 1e3])
def test_norm_control_and_clipped_step(bits, max_norm):
    s = Setup(LENGTHS, "f32", "bf16", bits, grad_scale=0.25, max_norm=max_norm, first_step=7, seed=3)
    s.opt.lr_scale.fill_(0.5)
    for step in (7, 8):
        old = s.before()
        norm, factor = s.opt.grad_norm()
        s.opt.step()
        torch.cuda.synchronize()
        ref = 0.25 * math.sqrt(sum(float((g.astype(np.float64) ** 2).sum()) for g in old["g"]))
        want = 0.25 * min(1.0, max_norm / ref) if max_norm else 0.25
        # both are float64 to the last rounding
        assert abs(float(norm) - ref) <= 2.0 ** -23 * ref and abs(float(factor) - want) <= 2.0 ** -23 * want
        assert s.opt.control[:3].tolist() == [step, 0, 1]
        _check(s, old, step, float(factor), 0.5)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("bits", [32, 8])
def test_a_gradient_that_is_not_finite_changes_nothing(bad, bits):
    s = Setup(LENGTHS, "f32", "f32", bits, max_norm=1.0)
    s.grads[9][5000] = bad
    everything = [t.clone() for ts in (s.params, s.m, s.v, s.copies, s.bases or []) for t in ts]
    norm, _ = s.opt.grad_norm()
    s.opt.step()
    torch.cuda.synchronize()
    assert not math.isfinite(float(norm)) and s.opt.control[:3].tolist() == [0, 1, 0]
    for was, now in zip(everything, [t for ts in (s.params, s.m, s.v, s.copies, s.bases or []) for t in ts]):
        assert torch.equal(was, now)
    s.grads[9][5000] = 0.0      # and the next step is the first
    old = s.before()
    _, factor = s.opt.grad_norm()
    s.opt.step()
    torch.cuda.synchronize()
    assert s.opt.control[:3].tolist() == [1, 1, 1]
    _check(s, old, 1, float(factor))


@pytest.mark.parametrize("scale", [1e-30, 1e15, 1e19])
def test_gradients_of_extreme_scale(scale):
    """Squares under and over float32's range count in the norm; 8-bit moments stay finite where float32 ones
    do (the largest gradient here squares to 1e33)."""
    s = Setup([4097, 300], "f32", "f32", 8, scale=scale)
    old = s.before()
    norm, _ = s.opt.grad_norm()
    s.opt.step()
    torch.cuda.synchronize()
    ref = math.sqrt(sum(float((g.astype(np.float64) ** 2).sum()) for g in old["g"]))
    assert abs(float(norm) - ref) <= 2.0 ** -23 * ref + 1e-45
    _check(s, old, 1, 1.0)


def test_all_gradients_zero():
    for bits in (32, 8):
        s = Setup([257, 4096], "f32", "bf16", bits, max_norm=1.0)
        for t in s.grads:
            t.zero_()
        old = s.before()
        norm, factor = s.opt.grad_norm()
        s.opt.step()
        torch.cuda.synchronize()
        assert float(norm) == 0.0 and float(factor) == 1.0
        _check(s, old, 1, 1.0)


def test_fresh_moments_and_unpack():
    from paper_2504_05638_amd.train import AdamW
    lengths = [5, 0, 256, 4099]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    grads = [torch.randn(n, generator=gen, device="cuda") for n in lengths]
    params = [torch.randn(n, generator=gen, device="cuda") for n in lengths]
    want = [p.clone() for p in params]
    opt = AdamW(params=params, grads=grads, bits=8, groups=[(1e-2, 0.0)])
    m, v = opt.unpack()
    assert m.numel() == v.numel() == sum(lengths) and not m.any() and not v.any()
    opt.step(1)
    m, v = opt.unpack()
    torch.cuda.synchronize()
    at = 0
    for n, p, w, g, mc, vc, b in zip(lengths, params, want, grads, opt.m, opt.v, opt.bases):
        # the first step goes by the sign alone
        assert torch.allclose(p, w - 1e-2 * g / (g.abs() + 1e-8), atol=2e-7, rtol=0)
        base = b.cpu().numpy().astype(np.int64).repeat(256)[:n]
        c, d = mc.cpu().numpy().astype(np.int64), vc.cpu().numpy().astype(np.int64)
        ref = _unpack(c & 127, base & 0xFFFF, n) * np.where(c > 127, np.float32(-1), np.float32(1))
        assert np.array_equal(m[at:at + n].float().cpu().numpy(), ref)
        assert np.array_equal(v[at:at + n].float().cpu().numpy(), _unpack(d, base >> 16, n))
        # 3 bits behind the leading one, up or down: within an eighth; far under the block's largest, within that
        assert torch.all((m[at:at + n].float() - 0.1 * g).abs() <= 0.125 * 0.1 * g.abs() + 1e-4)
        assert torch.all((v[at:at + n].float() - 1e-3 * g * g).abs() <= 0.126 * 1e-3 * g * g + 1e-11)
        at += n


def test_rounding_is_unbiased():
    """Over many steps of the same gradient a second moment that moves by a thousandth a step gets where it
    would get in float32 (to nearest it would stand still).  4096 elements, the mean's standard error: a rounding
    is off by less than an eighth of the number, steps add up like a random walk that the decay bounds:
    0.125 / sqrt(2 * 0.001 * 4096) < 5 %, of which five are allowed on the mean of v over all."""
    from paper_2504_05638_amd.train import AdamW
    n = 1 << 16
    g = torch.ones(n, device="cuda")
    opt = AdamW(params=[torch.zeros(n, device="cuda")], grads=[g], bits=8, betas=(0.9, 0.999), groups=[(0.0, 0.0)])
    g[::256] = 8.0     # the block's largest is another one
    for step in range(1, 701):
        opt.step(step)
    m, v = opt.unpack()
    rest = torch.ones(n, dtype=torch.bool, device="cuda")
    rest[::256] = False
    assert abs(float(v.float()[rest].mean()) / (1 - 0.999 ** 700) - 1) < 0.02
    assert abs(float(m.float()[rest].mean()) - 1) < 0.02


def test_result_does_not_depend_on_the_run():
    a, b = (Setup(LENGTHS, "f32", "bf16", 8, max_norm=1e-3, seed=5) for _ in range(2))
    for s in (a, b):
        for _ in range(3):
            s.opt.grad_norm()
            s.opt.step()
    torch.cuda.synchronize()
    assert torch.equal(a.opt.control, b.opt.control)
    for x, y in zip(a.params + a.m + a.v + a.bases, b.params + b.m + b.v + b.bases):
        assert torch.equal(x, y)


def test_only_empty_tensors_and_norm_only():
    from paper_2504_05638_amd.train import AdamW
    opt = AdamW(grads=[torch.zeros(0, device="cuda")], max_norm=1.0)
    norm, factor = opt.grad_norm()
    assert float(norm) == 0.0 and float(factor) == 1.0
    with pytest.raises(Exception):
        AdamW(grads=[torch.ones(4, device="cuda")]).step(1)


def test_a_gradient_past_32_bits():
    from paper_2504_05638_amd.train import AdamW
    n = (1 << 32) + 4099
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[-1], g[0], g[1 << 32] = 3.0, 4.0, 12.0
    norm, _ = AdamW(grads=[g]).grad_norm()
    assert float(norm) == 13.0


@pytest.mark.parametrize("bits", [32, 8])
def test_replayed_from_a_graph_on_another_stream(bits):
    s, e = (Setup(LENGTHS, "f32", "bf16", bits, max_norm=1e-3, seed=9) for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        s.opt.grad_norm()
        s.opt.step()
    for rep in range(4):
        for a, b in zip(s.grads, e.grads):
            a.mul_(1.5)
            b.mul_(1.5)
        s.opt.lr_scale.fill_(1.0 / (rep + 1))
        e.opt.lr_scale.fill_(1.0 / (rep + 1))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        e.opt.grad_norm()
        e.opt.step()
        torch.cuda.synchronize()
        assert s.opt.control[0].item() == rep + 1
        for a, b in zip(s.params + s.m + s.v + s.copies, e.params + e.m + e.v + e.copies):
            assert torch.equal(a, b)


def test_refusals():
    from paper_2504_05638_amd.train import AdamW
    g = torch.zeros(8, device="cuda")
    for kw in (dict(grads=[]), dict(grads=[g], params=[]), dict(grads=[g], params=[g.double()]), dict(grads=[g.half()]),
               dict(grads=[g], params=[torch.zeros(9, device="cuda")]), dict(grads=[torch.zeros(8, 8, device="cuda").t()]),
               dict(grads=[g], params=[g], bits=16), dict(grads=[g], params=[g], bits=8, m=[g], v=[g], bases=[g]),
               dict(grads=[g], params=[g], copies=[g]), dict(grads=[g], group_of=[1]), dict(grads=[g], params=[g.cpu()])):
        with pytest.raises((ValueError, KeyError)):
            AdamW(**kw)
