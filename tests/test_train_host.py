"""Host side of the optimizer and the linear layers: plans, sizes, workspaces and refusals.  Nothing here
touches a device; addresses are numbers that the library checks and never reads."""
import ctypes as C

import pytest

from paper_2504_05638_amd import binding as B

AT = 1 << 20  # an aligned address


def _cfg(**kw):
    d = dict(beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=1.0, max_norm=0.0, seed=0, moment_bits=32)
    d.update(kw)
    return B.tagc_optim_config(**d)


def _tensor(**kw):
    d = dict(param=AT, grad=AT, m=AT, v=AT, length=1000)
    d.update(kw)
    return B.tagc_tensor(**d)


def _code(f, *a, **kw):
    with pytest.raises(B.TagcError) as e:
        f(*a, **kw)
    return e.value.code


def test_structs_have_the_headers_sizes():
    assert C.sizeof(B.tagc_optim_control) == 64
    assert C.sizeof(B.tagc_tensor) == 72
    assert C.sizeof(B.tagc_optim_config) == 56
    assert C.sizeof(B.tagc_linear) == 24 + 8 + 8 * 11
    assert C.sizeof(B.tagc_linear_grad) == 24 + 8 + 8 * 13 + 8


def test_optimizer_plan_counts_its_tensors():
    lengths = [0, 1, 256, 257, 4096, 4097]
    plan = B.tagc_optim_plan(_cfg(), [_tensor(length=n) for n in lengths])
    z = B.tagc_optim_plan_sizes(plan)
    assert z.n_elems == sum(lengths)
    assert z.n_blocks == 0 + 1 + 1 + 2 + 16 + 17
    assert z.n_chunks == 0 + 1 + 1 + 1 + 1 + 2
    assert z.table_bytes >= 80 * len(lengths) + 8 * z.n_chunks
    B.tagc_optim_destroy(plan)
    plan = B.tagc_optim_plan(_cfg(), [])   # no tensors: a plan that has nothing to do
    assert B.tagc_optim_plan_sizes(plan).n_chunks == 0
    B.tagc_adamw_step(plan, AT, [], 1)
    B.tagc_optim_destroy(plan)


@pytest.mark.parametrize("bad", [dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=float("nan")), dict(eps=-1.0),
                                 dict(eps=float("inf")), dict(grad_scale=0.0), dict(grad_scale=float("nan")), dict(max_norm=-1.0),
                                 dict(max_norm=float("inf")), dict(moment_bits=16), dict(reserved=1)])
def test_optimizer_refuses_values(bad):
    assert _code(B.tagc_optim_plan, _cfg(**bad), [_tensor()]) == -1


@pytest.mark.parametrize("bad,code", [(dict(grad=None), -1), (dict(grad=AT + 2), -1), (dict(param=AT + 1), -1), (dict(m=None), -1),
                                      (dict(v=AT + 2), -1), (dict(copy=AT + 1), -1), (dict(bases=AT), -1), (dict(param_type=2), -1),
                                      (dict(grad_type=9), -1), (dict(group=16), -1), (dict(reserved=1), -1),
                                      (dict(length=1 << 34), -2), (dict(param=None), -1)])
def test_optimizer_refuses_tensors(bad, code):
    assert _code(B.tagc_optim_plan, _cfg(), [_tensor(), _tensor(**bad)]) == code


def test_optimizer_refuses_what_does_not_go_together():
    assert _code(B.tagc_optim_plan, _cfg(moment_bits=8), [_tensor()]) == -1          # no bases
    assert _code(B.tagc_optim_plan, _cfg(moment_bits=8), [_tensor(bases=AT + 2)]) == -1
    assert _code(B.tagc_optim_plan, _cfg(), [_tensor(length=1 << 33)] * 9) == -2       # too many chunks
    # 8-bit codes and 2-byte types may lie anywhere their element may
    plan = B.tagc_optim_plan(_cfg(moment_bits=8), [_tensor(m=AT + 1, v=AT + 3, bases=AT + 4, grad=AT + 2, grad_type=1,
                                                           param=AT + 6, param_type=1, copy=AT + 2)])
    assert _code(B.tagc_adamw_step, plan, AT, [], 1) == -1                      # group 0 is named, none given
    assert _code(B.tagc_adamw_step, plan, AT, [(1e-3, 0.0)] * 17, 1) == -1
    assert _code(B.tagc_adamw_step, plan, AT, [(float("nan"), 0.0)], 1) == -1
    assert _code(B.tagc_adamw_step, plan, AT, [(1e-3, 0.0)], 0, None) == -1      # no step and no control
    assert _code(B.tagc_adamw_step, plan, AT + 8, [(1e-3, 0.0)], 1) == -1
    assert _code(B.tagc_adamw_step, plan, None, [(1e-3, 0.0)], 1) == -1
    assert _code(B.tagc_grad_norm, plan, AT, None) == -1
    assert _code(B.tagc_grad_norm, plan, AT, AT + 4) == -1
    assert _code(B.tagc_adamw_unpack, plan, AT, None, AT) == -1
    assert _code(B.tagc_adamw_unpack, plan, AT, AT + 1, AT) == -1
    assert _code(B.tagc_optim_upload, plan, None) == -1
    B.tagc_optim_destroy(plan)
    plan = B.tagc_optim_plan(_cfg(), [_tensor()])
    assert _code(B.tagc_adamw_unpack, plan, AT, AT, AT) == -3                   # 32-bit moments
    B.tagc_optim_destroy(plan)
    plan = B.tagc_optim_plan(_cfg(), [B.tagc_tensor(grad=AT, length=5)])         # for the norm only
    assert _code(B.tagc_adamw_step, plan, AT, [(1e-3, 0.0)], 1) == -1
    B.tagc_optim_destroy(plan)


def _fwd(**kw):
    d = dict(rows=100, in_=128, out=64, dtype=B.TAGC_BF16, x=AT, ldx=128, w=AT, ldw=128, y=AT, ldy=64)
    d.update(kw)
    return B.tagc_linear(**d)


def _bwd(**kw):
    d = dict(rows=100, in_=128, out=64, dtype=B.TAGC_BF16, x=AT, ldx=128, w=AT, ldw=128, dy=AT, lddy=64, dx=AT, lddx=128,
             dw=AT, lddw=128)
    d.update(kw)
    return B.tagc_linear_grad(**d)


@pytest.mark.parametrize("bad,code", [(dict(dtype=2), -1), (dict(activation=5), -1), (dict(x=None), -1), (dict(w=None), -1), (dict(y=None), -1),
                                      (dict(x=AT + 1), -1), (dict(ldx=127), -1), (dict(ldw=1), -1), (dict(ldy=63), -1),
                                      (dict(residual=AT, ldr=63), -1), (dict(pre=AT + 1, ldp=64), -1), (dict(bias=AT + 1), -1),
                                      (dict(dtype=0, x=AT + 2), -1), (dict(rows=1 << 22), -2), (dict(in_=1 << 22, ldx=1 << 22, ldw=1 << 22), -2),
                                      (dict(rows=1 << 20, out=1 << 18, ldy=1 << 18), -2)])
def test_forward_refuses(bad, code):
    assert _code(B.tagc_linear_forward_workspace, _fwd(**bad)) == code
    assert _code(B.tagc_linear_forward, _fwd(**bad), AT) == code


@pytest.mark.parametrize("bad", [dict(dtype=2), dict(activation=9), dict(dy=None), dict(x=None), dict(w=None), dict(reserved=1),
                                 dict(accumulate=2), dict(lddx=5), dict(lddw=5), dict(db=AT + 1), dict(dw=AT + 1), dict(activation=1),
                                 dict(pre=AT, ldp=64)])
def test_backward_refuses(bad):
    assert _code(B.tagc_linear_backward_workspace, _bwd(**bad)) == -1
    assert _code(B.tagc_linear_backward, _bwd(**bad), AT) == -1


def test_workspaces():
    assert B.tagc_linear_forward_workspace(_fwd(rows=0)) == 0
    assert B.tagc_linear_forward_workspace(_fwd(rows=1)) == 0          # the weights as they lie
    # rows off a 16-byte boundary are laid out anew: 100 rows of 128
    assert (B.tagc_linear_forward_workspace(_fwd(x=AT + 2)) - B.tagc_linear_forward_workspace(_fwd())) == 100 * 128 * 2
    # float32 is taken apart in the product where tiles are few, in the workspace where they are many
    assert B.tagc_linear_forward_workspace(_fwd(dtype=B.TAGC_F32, rows=4096, out=4096, ldy=4096)) >= 2 * 4096 * 128 * 6
    # behind an activation dz is laid out, and a bias's gradient has partial sums
    behind = dict(pre=AT, ldp=64, activation=B.TAGC_ACT_SILU)
    need = B.tagc_linear_backward_workspace(_bwd(**behind))
    assert need >= 100 * 64 * 2
    assert B.tagc_linear_backward_workspace(_bwd(db=AT, **behind)) > need
    assert _code(B.tagc_linear_backward, _bwd(**behind), None) == -1
    assert _code(B.tagc_linear_backward, _bwd(**behind), AT + 16) == -1
    assert B.tagc_linear_backward_workspace(_bwd(dx=None, w=None, **behind)) <= need
    assert B.tagc_linear_backward_workspace(_bwd(dx=None, dw=None)) == 0
