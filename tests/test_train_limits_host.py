"""Limits of an optimizer's plan.  Nothing here touches a device."""
import pytest

from paper_2504_05638_amd import binding as B

AT = 1 << 20
CHUNK = 4096


def _plan(chunks, bits, params=True):
    """The chunks that a plan over five tensors of so many together has, or the error's code."""
    lengths = [(chunks // 5) * CHUNK] * 4 + [(chunks - 4 * (chunks // 5)) * CHUNK - 5]
    more = dict(param=AT, m=AT, v=AT, bases=AT if bits == 8 else None) if params else {}
    cfg = B.tagc_optim_config(beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=1.0, moment_bits=bits)
    try:
        plan = B.tagc_optim_plan(cfg, [B.tagc_tensor(grad=AT, length=n, **more) for n in lengths])
    except B.TagcError as e:
        return e.code
    n = B.tagc_optim_plan_sizes(plan).n_chunks
    B.tagc_optim_destroy(plan)
    return n


@pytest.mark.parametrize("bits,most", [(8, 1 << 23), (32, 1 << 24)])
def test_a_plan_that_no_launch_takes_is_refused(bits, most):
    """A step's workgroups have 512 threads with 8-bit moments, 256 with 32-bit ones; a launch has fewer than 2^32 threads."""
    assert _plan(most - 1, bits) == most - 1
    assert _plan(most, bits) == -2


def test_a_plan_for_the_norm_alone_may_have_more():
    assert _plan(1 << 23, 8, params=False) == 1 << 23
