"""GELU far to the left, where the result is a small share of its argument: errors against the result itself.

z below(z), with below(z) = erfc(-z / sqrt(2)) / 2.  An argument off by a relative d moves erfc(u) by at most (2 u^2 + 1.5) d
of itself for u > 1, that is (z^2 + 1.5) d, and exp(-z^2 / 2) by z^2 d.  With e = 2^-24, float32: the argument takes two
roundings and one of the constant, erfc itself 16 ulps at most (2 e each), three products more; the bell's exponent
two roundings and the constant's, exp2 two ulps.  Slope: below(z) + z bell(z) / sqrt(2 pi), to the left of -2 of opposite signs and
no cancellation to speak of: z bell is at least 4 times below.  bfloat16: 2^-12 for the polynomial instead of erfc's own, and the result's
rounding, 2^-8."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

E = 2.0 ** -24


def _through(z, dtype):
    from paper_2504_05638_amd.train import linear, linear_backward
    one = torch.ones(1, 1, device="cuda", dtype=dtype)
    y, pre = linear(z.view(-1, 1), one, activation="gelu", save=True)
    slope = linear_backward(torch.ones_like(y), z.view(-1, 1), one, pre, activation="gelu")
    assert torch.equal(pre.view(-1), z)
    d = z.double()
    below, bell = 0.5 * torch.erfc(-d / math.sqrt(2)), torch.exp(-d * d / 2)
    return y.view(-1).double(), d * below, slope.view(-1).double(), below + d * bell / math.sqrt(2 * math.pi), d


def test_float32_left_tail():
    z = -torch.linspace(2.0, 12.0, 20_001, device="cuda")
    y, ref, slope, slope_ref, d = _through(z, torch.float32)
    rel = ((d * d + 1.5) * 3 + 32 + 4) * E
    assert torch.all((y - ref).abs() <= rel * ref.abs())
    # four thirds of the bell's share and a third of below's
    rel = (4 * (d * d * 3 + 8) + ((d * d + 1.5) * 3 + 36)) / 3 * E
    assert torch.all((slope - slope_ref).abs() <= rel * slope_ref.abs())


def test_bfloat16_left_tail():
    """Every bfloat16 from -2 to -12.5."""
    z = torch.arange(0x4000, 0x4149, device="cuda", dtype=torch.int32).to(torch.int16).view(torch.bfloat16).neg()
    assert float(z[0]) == -2.0 and float(z[-1]) == -12.5
    y, ref, slope, slope_ref, d = _through(z, torch.bfloat16)
    below, bell, half = 2.0 ** -12 + (3 * d * d + 40) * E, (3 * d * d + 8) * E, 2.0 ** -8
    assert torch.all((y - ref).abs() <= (below + half) * ref.abs())
    assert torch.all((slope - slope_ref).abs() <= ((4 * bell + below) / 3 + half) * slope_ref.abs())
