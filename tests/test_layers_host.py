"""Host side of norms, embeddings and losses: sizes, workspaces and refusals.  Nothing here touches a device; addresses are numbers
that the library checks and never reads."""
import ctypes as C
import math

import pytest

from paper_2504_05638_amd import binding as B

A, X, Y, Z, W, V, U, S = (k << 36 for k in range(1, 9))


def _code(f, *a):
    with pytest.raises(B.TagcError) as e:
        f(*a)
    return e.value.code


def test_structs_have_the_headers_sizes():
    assert C.sizeof(B.tagc_norm) == 24 + 8 + 8 * 8 - 8
    assert C.sizeof(B.tagc_norm_grad) == 24 + 8 * 12 + 8
    assert C.sizeof(B.tagc_embedding) == 32 + 8 + 8 * 7
    assert C.sizeof(B.tagc_embedding_grad) == 32 + 8 + 8 * 5 + 8
    assert C.sizeof(B.tagc_loss) == 24 + 16 + 8 + 8 * 8
    assert C.sizeof(B.tagc_loss_grad) == 24 + 16 + 8 + 8 * 8 + 8 + 8 * 4


def _norm(**kw):
    d = dict(rows=100, width=64, dtype=B.TAGC_BF16, kind=0, eps=1e-5, x=X, ldx=64, w=W, b=V, y=Y, ldy=64, stats=S)
    d.update(kw)
    return B.tagc_norm(**d)


@pytest.mark.parametrize("bad,code", [(dict(dtype=2), -1), (dict(kind=2), -1), (dict(eps=-1.0), -1), (dict(eps=math.nan), -1), (dict(eps=math.inf), -1),
                                      (dict(kind=1), -1), (dict(x=None), -1), (dict(y=None), -1), (dict(x=X + 1), -1), (dict(ldx=63), -1), (dict(ldy=63), -1),
                                      (dict(w=W + 1), -1), (dict(stats=S + 4), -1), (dict(width=16385, ldx=16385, ldy=16385), -2), (dict(rows=1 << 31), -2),
                                      (dict(y=X + 2), -1), (dict(y=X, ldy=72), -1), (dict(y=X + 64 * 2 * 99), -1), (dict(y=W), -1), (dict(b=Y + 2), -1),
                                      (dict(stats=Y), -1), (dict(stats=X + 64), -1)])
def test_norm_refuses(bad, code):
    assert _code(B.tagc_norm_forward, _norm(**bad)) == code


def _norm_grad(**kw):
    d = dict(rows=100, width=64, dtype=B.TAGC_BF16, kind=0, x=X, ldx=64, w=W, stats=S, dy=Y, lddy=64, residual=Z, ldr=64, dx=A, lddx=64, dw=V, db=U)
    d.update(kw)
    return B.tagc_norm_grad(**d)


@pytest.mark.parametrize("bad,code", [(dict(dtype=2), -1), (dict(kind=2), -1), (dict(kind=1), -1), (dict(reserved=1), -1), (dict(accumulate=2), -1), (dict(x=None), -1),
                                      (dict(dy=None), -1), (dict(stats=None), -1), (dict(dx=None), -1), (dict(lddx=3), -1), (dict(dw=V + 1), -1), (dict(stats=S + 4), -1),
                                      (dict(width=1 << 15, ldx=1 << 15, lddy=1 << 15, ldr=1 << 15, lddx=1 << 15), -2), (dict(dx=X + 2), -1), (dict(dx=Y, lddx=66), -1),
                                      (dict(dx=Z + 128), -1), (dict(dx=W), -1), (dict(dx=S + 16), -1), (dict(dw=U + 2), -1), (dict(db=A + 4), -1)])
def test_norm_backward_refuses(bad, code):
    assert _code(B.tagc_norm_backward_workspace, _norm_grad(**bad)) == code
    assert _code(B.tagc_norm_backward, _norm_grad(**bad), A) == code


def test_norm_workspace():
    need = B.tagc_norm_backward_workspace(_norm_grad(rows=1000))
    assert need >= 1000 // 4 * 2 * 64 * 4
    assert B.tagc_norm_backward_workspace(_norm_grad(dw=None, db=None)) == 0
    assert B.tagc_norm_backward_workspace(_norm_grad(rows=0)) == 0
    for place in (X, Y, Z):     # dx in the place of what it is made of
        assert B.tagc_norm_backward_workspace(_norm_grad(rows=1000, dx=place)) == need
    assert _code(B.tagc_norm_backward, _norm_grad(rows=1000), None) == -1
    assert _code(B.tagc_norm_backward, _norm_grad(rows=1000), A + 16) == -1
    # few rows' dw and db are made beside dx, unless that is written over what they are made of
    assert B.tagc_norm_backward_workspace(_norm_grad()) == B.tagc_norm_backward_workspace(_norm_grad(dx=Z)) == 0
    assert B.tagc_norm_backward_workspace(_norm_grad(dx=X)) == B.tagc_norm_backward_workspace(_norm_grad(dx=Y)) > 0


@pytest.mark.parametrize("of", ["dw", "db"])
@pytest.mark.parametrize("place", [X, Y, Z, W, S])
@pytest.mark.parametrize("rows", [100, 1000])
def test_norm_gradients_over_operands_are_refused(of, place, rows):
    assert _code(B.tagc_norm_backward_workspace, _norm_grad(rows=rows, **{of: place})) == -1


def _embed(**kw):
    d = dict(rows=100, width=64, vocab=1000, dtype=B.TAGC_BF16, id_type=1, scale=1.0, ids=A, table=X, ldt=64, residual=Z, ldr=64, y=Y, ldy=64)
    d.update(kw)
    return B.tagc_embedding(**d)


@pytest.mark.parametrize("bad,code", [(dict(dtype=2), -1), (dict(id_type=2), -1), (dict(scale=math.inf), -1), (dict(scale=1e39), -1), (dict(ids=None), -1), (dict(table=None), -1),
                                      (dict(y=None), -1), (dict(ids=A + 4), -1), (dict(ldt=63), -1), (dict(ldy=63), -1), (dict(ldr=1), -1), (dict(table=X + 1), -1),
                                      (dict(rows=1 << 22), -2), (dict(vocab=1 << 22), -2), (dict(width=1 << 22, ldt=1 << 22, ldr=1 << 22, ldy=1 << 22), -2),
                                      (dict(rows=1 << 21, width=1 << 15, ldt=1 << 15, ldr=1 << 15, ldy=1 << 15), -2), (dict(y=X + 999 * 128), -1), (dict(y=A), -1),
                                      (dict(y=Z, ldy=72), -1), (dict(y=Z + 2), -1)])
def test_embedding_refuses(bad, code):
    assert _code(B.tagc_embedding_forward, _embed(**bad)) == code


def _embed_grad(**kw):
    d = dict(rows=100, width=64, vocab=1000, dtype=B.TAGC_BF16, id_type=1, scale=1.0, ids=A, dy=Y, lddy=64, dtable=X, ldt=64)
    d.update(kw)
    return B.tagc_embedding_grad(**d)


@pytest.mark.parametrize("bad,code", [(dict(dtype=2), -1), (dict(id_type=2), -1), (dict(scale=math.nan), -1), (dict(ids=None), -1), (dict(dy=None), -1), (dict(dtable=None), -1),
                                      (dict(ids=A + 4), -1), (dict(lddy=63), -1), (dict(ldt=63), -1), (dict(reserved=1), -1), (dict(accumulate=2), -1), (dict(rows=1 << 22), -2),
                                      (dict(dtable=Y), -1), (dict(dtable=Y + 99 * 128), -1), (dict(dtable=A + 8), -1)])
def test_embedding_backward_refuses(bad, code):
    assert _code(B.tagc_embedding_backward_workspace, _embed_grad(**bad)) == code
    assert _code(B.tagc_embedding_backward, _embed_grad(**bad), A) == code


def test_embedding_workspace():
    assert B.tagc_embedding_backward_workspace(_embed_grad()) == 0          # few tokens: one launch
    need = B.tagc_embedding_backward_workspace(_embed_grad(rows=1000))
    assert need >= 1000 * 8 + 125 * 2 * 64 * 4
    assert B.tagc_embedding_backward_workspace(_embed_grad(rows=0, ids=None, dy=None)) == 0
    assert B.tagc_embedding_backward_workspace(_embed_grad(rows=5000)) >= 5000 * 16     # two lists, to merge
    assert B.tagc_embedding_backward_workspace(_embed_grad(id_type=0, ids=A + 4, rows=1000)) == need
    assert _code(B.tagc_embedding_backward, _embed_grad(rows=1000), None) == -1


def _loss(**kw):
    d = dict(rows=100, in_=64, vocab=1000, terms=1, dtype=B.TAGC_BF16, id_type=1, temperature=1.0, x=X, ldx=64, w=W, ldw=64, ids=A, loss=Y, saved=Z)
    d.update(kw)
    return B.tagc_loss(**d)


def _loss_grad(**kw):
    d = dict(rows=100, in_=64, vocab=1000, terms=1, dtype=B.TAGC_BF16, id_type=1, temperature=1.0, x=X, ldx=64, w=W, ldw=64, ids=A, saved=Z, dloss=Y, dloss_step=1,
             dx=U, lddx=64, dw=V, lddw=64)
    d.update(kw)
    return B.tagc_loss_grad(**d)


BOTH = [(dict(dtype=2), -1), (dict(id_type=2), -1), (dict(in_=0), -1), (dict(vocab=0), -1), (dict(terms=0), -1), (dict(terms=2), -1), (dict(temperature=0.0), -1),
        (dict(temperature=-1.0), -1), (dict(temperature=math.nan), -1), (dict(temperature=math.inf), -1), (dict(temperature=1e-40), -1), (dict(temperature=1e60), -1),
        (dict(x=None), -1), (dict(w=None), -1), (dict(ids=None), -1), (dict(saved=Z + 2), -1), (dict(ids=A + 4), -1), (dict(ldx=63), -1), (dict(ldw=63), -1), (dict(x=X + 1), -1),
        (dict(rows=1 << 22), -2), (dict(vocab=1 << 22), -2), (dict(dtype=0, vocab=1 << 20), -2), (dict(terms=1025, logits=S), -2), (dict(logits=S + 2), -1), (dict(reserved=1), -1),
        (dict(rows=1 << 21, terms=16, logits=S), -2), (dict(rows=1 << 18, vocab=1 << 20), -2)]


@pytest.mark.parametrize("bad,code", BOTH + [(dict(loss=None), -1), (dict(loss=X), -1), (dict(loss=W + 4), -1), (dict(loss=A), -1), (dict(saved=X + 64), -1), (dict(saved=Y + 396), -1),
                                             (dict(logits=Y + 4), -1)])
def test_loss_refuses(bad, code):
    assert _code(B.tagc_loss_forward_workspace, _loss(**bad)) == code
    assert _code(B.tagc_loss_forward, _loss(**bad), A) == code


@pytest.mark.parametrize("bad,code", BOTH + [(dict(saved=None), -1), (dict(dloss=None), -1), (dict(dloss=Y + 2), -1), (dict(dloss_step=2), -1), (dict(accumulate=2), -1),
                                             (dict(lddx=63), -1), (dict(lddw=63), -1), (dict(dx=X), -1), (dict(dx=W), -1), (dict(dx=A + 8), -1), (dict(dx=Z + 64), -1), (dict(dx=Y), -1),
                                             (dict(dw=W), -1), (dict(dw=X + 128), -1), (dict(dw=U + 99 * 128), -1), (dict(dw=Z), -1), (dict(dw=Y + 4), -1)])
def test_loss_backward_refuses(bad, code):
    assert _code(B.tagc_loss_backward_workspace, _loss_grad(**bad)) == code
    assert _code(B.tagc_loss_backward, _loss_grad(**bad), A) == code


@pytest.mark.parametrize("dtype", [B.TAGC_BF16, B.TAGC_F32])
@pytest.mark.parametrize("terms", [1, 5, 1024])
def test_loss_workspaces_of_any_size(dtype, terms):
    """Whole pieces, single tiles, and what lies between."""
    for rows in (1, 2, 16, 17, 64, 65, 128, 1000, 1024, 1025, 4096):
        for vocab in (1, 31, 32, 64, 255, 256, 4095, 4096, 8192, 12288, 32000, 65536, 131072, 262144, 262145):
            for width in (1, 8, 64, 777, 4096):
                kw = dict(rows=rows, vocab=vocab, in_=width, ldx=width, ldw=width, terms=terms, dtype=dtype, logits=S if terms > 1 else None)
                if rows * terms < 1 << 25:
                    assert B.tagc_loss_forward_workspace(_loss(**kw)) > 0
                    assert B.tagc_loss_backward_workspace(_loss_grad(lddx=width, lddw=width, **kw)) > 0


def test_loss_workspaces():
    """What is held does not grow with the vocabulary, but for scores of few rows."""
    big = [B.tagc_loss_forward_workspace(_loss(rows=8192, in_=4096, ldx=4096, ldw=4096, vocab=v)) for v in (1 << 18, 1 << 19, 1 << 20)]
    assert max(big) - min(big) < 1 << 20 and max(big) < 8192 * 4096 * 2 + (550 << 20)
    back = [B.tagc_loss_backward_workspace(_loss_grad(rows=8192, in_=4096, ldx=4096, ldw=4096, lddx=4096, lddw=4096, vocab=v)) for v in (1 << 18, 1 << 19, 1 << 20)]
    assert max(back) - min(back) < 64 << 20 and max(back) < 8192 * 4096 * 6 + (550 << 20) < 8192 * (1 << 18) * 2
    assert B.tagc_loss_forward_workspace(_loss()) >= 100 * 1000 * 4          # few rows: their scores
    assert B.tagc_loss_forward_workspace(_loss(rows=0, x=None, ids=None)) == 0
    assert B.tagc_loss_backward_workspace(_loss_grad(dx=None, dw=None)) == 0
    assert B.tagc_loss_backward_workspace(_loss_grad(dx=None)) < B.tagc_loss_backward_workspace(_loss_grad())
    assert _code(B.tagc_loss_forward, _loss(), None) == -1
    assert _code(B.tagc_loss_forward, _loss(), A + 128) == -1
    assert _code(B.tagc_loss_backward, _loss_grad(), None) == -1


def test_norm_eps_that_float32_does_not_hold():
    """It would count as an infinity, and rows as their bias."""
    for eps in (1e39, 1e300):
        assert _code(B.tagc_norm_forward, _norm(eps=eps)) == -1


def test_sizes_that_are_allowed_together():
    """On both sides of what the header says of products of sizes."""
    wide = (1 << 22) - 1
    for rows, width in ((wide, 4096), (4096, wide), (1 << 17, 1 << 17), (1, wide), (wide, 1)):
        assert rows * width <= 1 << 34
        # (a result over an operand, which is found behind sizes: nothing is launched)
        assert _code(B.tagc_embedding_forward, _embed(rows=rows, width=width, y=A, ldt=width, ldr=width, ldy=width)) == -1
        assert B.tagc_embedding_backward_workspace(_embed_grad(rows=rows, width=width, vocab=1, lddy=width, ldt=width, dtable=1 << 48)) >= 0
    for terms, rows in ((1024, (1 << 15) - 1), (16, (1 << 21) - 1), (1000, 33554)):
        assert rows * terms < 1 << 25 <= (rows + 1) * terms
        assert B.tagc_loss_forward_workspace(_loss(rows=rows, terms=terms, logits=S, loss=1 << 48, saved=None)) > 0
        assert _code(B.tagc_loss_forward_workspace, _loss(rows=rows + 1, terms=terms, logits=S, loss=1 << 48, saved=None)) == -2
    for width, allowed in (((1 << 17) - 64, True), ((1 << 17) - 63, False), (1 << 17, False)):
        a = _loss(rows=10, vocab=1 << 17, in_=width, ldx=width, ldw=width)
        if allowed:
            assert B.tagc_loss_forward_workspace(a) > 0
        else:
            assert _code(B.tagc_loss_forward_workspace, a) == -2
