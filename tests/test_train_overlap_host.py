"""Operands and results that share memory: what the layers refuse, and what they have to take.  Nothing here touches a device;
addresses are numbers that the library checks and never reads."""
import random

import pytest

from paper_2504_05638_amd import binding as B


def _bytes(at, rows, width, ld):
    return {at + i * ld + j for i in range(rows) for j in range(width)} if at else set()


def test_whether_rows_meet():
    rng = random.Random(1)
    seen = {True: 0, False: 0}
    for _ in range(30_000):
        ld = rng.randrange(1, 12)
        a, b = ((100 + rng.randrange(40), rng.randrange(0, 6), rng.randrange(0, k + 1), k) for k in (ld, ld if rng.random() < 0.6 else rng.randrange(1, 12)))
        want = bool(_bytes(*a) & _bytes(*b))
        assert B.tagc_rows_meet_host(a, b) == want == B.tagc_rows_meet_host(b, a), (a, b)
        seen[want] += 1
    assert min(seen.values()) > 5_000
    assert not B.tagc_rows_meet_host((0, 5, 5, 5), (0, 5, 5, 5))


X, W, Y, P, R, D = (1 << 30, 2 << 30, 3 << 30, 4 << 30, 5 << 30, 6 << 30)


def _refused(f, a):
    with pytest.raises(B.TagcError) as e:
        f(a, 1 << 40)
    return e.value.code == -1


@pytest.mark.parametrize("bad", [dict(y=X), dict(y=X + 99 * 256), dict(y=W + 2), dict(y=R + 2), dict(y=R, ldr=72), dict(bias=Y + 4), dict(pre=X), dict(pre=W),
                                 dict(pre=R), dict(pre=Y), dict(pre=Y + 128), dict(pre=Y, residual=None, activation=1),
                                 dict(pre=Y + 64, ldp=66, residual=None), dict(bias=P)])
def test_forward(bad):
    d = dict(rows=100, in_=128, out=64, dtype=B.TAGC_BF16, x=X, ldx=128, w=W, ldw=128, bias=D, residual=R, ldr=64, y=Y, ldy=64, pre=P, ldp=64)
    d.update(bad)
    assert _refused(B.tagc_linear_forward, B.tagc_linear(**d))


OVER = [dict(dx=X), dict(dx=W), dict(dw=W), dict(dw=X), dict(db=Y), dict(db=R + 100), dict(dw=Y + 512)]
OVER_DY = [dict(dx=D), dict(dw=D + 2), dict(dx=D + 99 * 128)]      # (behind an activation dy and pre have been read before)


@pytest.mark.parametrize("bad,activation", [(o, 0) for o in OVER + OVER_DY] + [(o, 1) for o in OVER])
def test_backward(bad, activation):
    d = dict(rows=100, in_=128, out=64, dtype=B.TAGC_BF16, x=X, ldx=128, w=W, ldw=128, dy=D, lddy=64, dx=Y, lddx=128, dw=R, lddw=128, db=7 << 30)
    if activation:
        d.update(activation=activation, pre=P, ldp=64)
    d.update(bad)
    assert _refused(B.tagc_linear_backward, B.tagc_linear_grad(**d))


@pytest.mark.parametrize("bad", [dict(dx=R), dict(db=Y), dict(db=R + 100)])
def test_backward_float32(bad):
    d = dict(rows=100, in_=128, out=64, dtype=B.TAGC_F32, x=X, ldx=128, w=W, ldw=128, dy=D, lddy=64, dx=Y, lddx=128, dw=R, lddw=128, db=7 << 30)
    d.update(bad)
    assert _refused(B.tagc_linear_backward, B.tagc_linear_grad(**d))
