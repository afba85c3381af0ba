"""The two ends of a data-parallel step around the exchange: the layers whose backward pass
writes into a bucket's gradient -- linear ones, norms, the tokens' table, the loss over the vocabulary --,
and the optimizer behind it.  Device memory and argument marshalling only; all arithmetic is the library's
(include/tagc_train.h).

    x = embedding(ids, table)
    h, stats = norm(x, gain, kind="rms", save=True)
    y, pre = linear(x, w, b, activation="gelu", save=True)
    loss, saved = cross_entropy(y, head, targets, save=True)
    dy = cross_entropy_backward(dloss, y, head, targets, saved, dw=bucket_grad_view)
    dh = linear_backward(dy, h, w, pre, activation="gelu", dw=bucket_grad_view, db=...)
    dx = norm_backward(dh, x, gain, stats, kind="rms", residual=dy, dw=...)
    embedding_backward(dx, ids, bucket_grad_view)
    ...                                # the exchange: bucket.TagcBucket
    opt = AdamW(params=..., grads=dense_views(bucket), max_norm=1.0, bits=8)
    opt.grad_norm()                    # norm, clip factor and step count, on the device
    opt.step()
"""
from __future__ import annotations

import contextlib
import math
import warnings

import torch
from torch.autograd.graph import increment_version

from . import binding as B
from .bucket import _bytes, _stream_ptr

_TYPES = {torch.float32: B.TAGC_F32, torch.bfloat16: B.TAGC_BF16}
_ACTS = {None: B.TAGC_ACT_NONE, "none": B.TAGC_ACT_NONE, "relu": B.TAGC_ACT_RELU,
         "gelu": B.TAGC_ACT_GELU, "gelu_tanh": B.TAGC_ACT_GELU_TANH, "silu": B.TAGC_ACT_SILU}


def _need(condition, what):
    if not condition:
        raise ValueError(what)


# (the address of the device's current stream, without the object around it where torch offers that: a
# third of what a small call costs the host)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream_of(stream, device):
    if stream is None and _raw_stream is not None and device.index is not None:
        return _raw_stream(device.index)
    return _stream_ptr(stream)


_HERE = contextlib.nullcontext()


def _at(device, stream=None):
    """Calls are made with the tensors' device as the current one: launches go to its streams, and the library cuts work by
    its compute units.  Under a given stream what they make is that stream's own: memory of the current stream's may still
    be in use there."""
    if stream is not None:
        return torch.cuda.stream(stream)
    return _HERE if _current_device() == device.index else torch.cuda.device(device)


def _hand_over(user, *made):
    """What was made under a given stream is not used again there before what `user`, the caller's stream, does with it is done."""
    for t in made:
        if t is not None:
            t.record_stream(user)


def _rows_of(t, name, rows, cols, dtype, device):
    """(address, elements from row to row) of a [rows, cols] matrix; (None, 0) for None."""
    if t is None:
        return None, 0
    if t.dtype != dtype or t.device != device:
        raise ValueError("%s: a %s on %s is wanted" % (name, dtype, device))
    if t.shape != (rows, cols):
        raise ValueError("%s has shape %s, %s is wanted" % (name, tuple(t.shape), (rows, cols)))
    ld, step = t.stride()
    if rows <= 1 or cols == 0:  # (of a single row the stride says nothing; of no elements neither does the address)
        ld = cols
    if (step != 1 and cols > 1 and rows > 0) or ld < cols:
        raise ValueError("%s: a row's elements must be neighbours, and rows must not overlap" % name)
    return t.data_ptr() or None, ld


def _vector(t, name, n, dtype, device):
    if t is None:
        return None
    if t.dtype != dtype or t.device != device or t.shape != (n,) or not (t.is_contiguous() or n <= 1):
        raise ValueError("%s: a contiguous vector of %d, %s on %s, is wanted" % (name, n, dtype, device))
    return t.data_ptr() or None


def _check_stream(stream, device):
    _need(stream.device == device, "stream: one of the tensors' device is wanted")


def _check_input(x, w, activation, stream):
    if stream is not None:
        _check_stream(stream, x.device)
    if not x.is_cuda or x.dtype not in _TYPES:
        raise ValueError("x: a CUDA tensor of float32 or bfloat16 is wanted")
    if w.dim() != 2 or x.dim() < 2 or x.shape[-1] != w.shape[1]:
        raise ValueError("x is [..., in] and w [out, in]: got %s and %s" % (tuple(x.shape), tuple(w.shape)))
    if activation not in _ACTS:
        raise ValueError("activation: one of %s is wanted" % ", ".join(k for k in _ACTS if k))


def _counted(tensors):
    """Of tensors that calls write to those whose version autograd counts, views that share a count once."""
    once = {}
    for t in tensors:
        if t is not None and not t.is_inference():
            t = t._base if t._is_view() else t
            once[id(t)] = t
    return tuple(once.values())


def _flat(t, rows, cols):
    """[..., cols] as [rows, cols] without a copy (ValueError if its strides need one)."""
    if t is None or t.dim() == 2:
        return t
    try:
        return t.view(rows, cols)
    except RuntimeError as e:
        raise ValueError(str(e)) from None


def _work(nbytes, x):
    """A call's workspace (its tensor and its address), the current stream's own: reused behind the call only."""
    if not nbytes:
        return None, None
    ws = torch.empty(nbytes, dtype=torch.uint8, device=x.device)
    return ws, ws.data_ptr()


def linear(x, w, bias=None, residual=None, activation=None, save=False, out=None, pre=None, stream=None):
    """(y, pre): y = activation(x w^T + bias) + residual.  x: [..., in], w: [out, in].  `save`: pre =
    x w^T + bias for linear_backward (else None).  `out` and `pre` may be given; `out` may be
    the residual.  No autograd graph is recorded (linear_backward is the gradient): with tensors that require one, outside
    torch.no_grad(), there is a warning.  With `stream` the call runs there: what it reads has to be ready there, and stay
    until it is done; what it makes (results, workspace) is `stream`'s memory."""
    _check_input(x, w, activation, stream)
    if (x.requires_grad or w.requires_grad or (bias is not None and bias.requires_grad)
            or (residual is not None and residual.requires_grad)) and torch.is_grad_enabled():
        warnings.warn("linear records no autograd graph: gradients are linear_backward's; call it under torch.no_grad()", stacklevel=2)
    n, k = w.shape
    shape, dtype, device = x.shape, x.dtype, x.device
    m = shape[0] if len(shape) == 2 else math.prod(shape[:-1])
    _need(pre is None or save, "pre is given, but save is not")
    xp, ldx = _rows_of(_flat(x, m, k), "x", m, k, dtype, device)
    wp, ldw = _rows_of(w, "w", n, k, dtype, device)
    bp = _vector(bias, "bias", n, dtype, device)
    rp, ldr = _rows_of(_flat(residual, m, n), "residual", m, n, dtype, device)
    yp, ldy = _rows_of(_flat(out, m, n), "out", m, n, dtype, device)
    pp, ldp = _rows_of(_flat(pre, m, n), "pre", m, n, dtype, device)
    given, user = (out, pre), torch.cuda.current_stream(device) if stream is not None else None
    with _at(device, stream):
        if out is None:
            out = x.new_empty((*shape[:-1], n))
            yp, ldy = out.data_ptr() or None, n
        if save and pre is None:
            pre = x.new_empty((*shape[:-1], n))
            pp, ldp = pre.data_ptr() or None, n
        a = B.tagc_linear(m, k, n, _TYPES[dtype], _ACTS[activation], xp, ldx, wp, ldw, bp, rp, ldr, yp, ldy, pp, ldp)
        ws, at = _work(B.tagc_linear_forward_workspace(a), x)
        B.tagc_linear_forward(a, at, _stream_of(stream, device))
    if stream is not None:
        _hand_over(user, out if given[0] is None else None, pre if given[1] is None else None)
    if given[0] is not None or given[1] is not None:
        # (as torch's in-place operations do: a graph that kept one of them raises in its backward pass)
        increment_version(_counted(given))
    return out, pre


def linear_backward(dy, x, w, pre=None, activation=None, dx=None, dw=None, db=None, accumulate=False,
                    need_dx=True, stream=None):
    """dx (None without need_dx).  With `dw` ([out, in], a view into a bucket's gradient) and `db` ([out])
    given, the weight's and the bias's gradient are written there, or added to what is there
    (accumulate).  `pre`: what linear(save=True) gave; None without an activation.  `stream`: as for linear."""
    _check_input(x, w, activation, stream)
    n, k = w.shape
    shape, dtype, device = x.shape, x.dtype, x.device
    m = shape[0] if len(shape) == 2 else math.prod(shape[:-1])
    act = _ACTS[activation]
    _need((act != B.TAGC_ACT_NONE) == (pre is not None), "pre is wanted with an activation, and only then")
    _need(need_dx or dx is None, "dx is given, but need_dx is not")
    xp, ldx = _rows_of(_flat(x, m, k), "x", m, k, dtype, device)
    wp, ldw = _rows_of(w, "w", n, k, dtype, device)
    pp, ldp = _rows_of(_flat(pre, m, n), "pre", m, n, dtype, device)
    yp, ldy = _rows_of(_flat(dy, m, n), "dy", m, n, dtype, device)
    dp, ldd = _rows_of(_flat(dx, m, k), "dx", m, k, dtype, device)
    gp, ldg = _rows_of(dw, "dw", n, k, dtype, device)
    bp = _vector(db, "db", n, dtype, device)
    given, user = (dx, dw, db), torch.cuda.current_stream(device) if stream is not None else None
    with _at(device, stream):
        if need_dx and dx is None:
            dx = x.new_empty(shape)
            dp, ldd = dx.data_ptr() or None, k
        a = B.tagc_linear_grad(m, k, n, _TYPES[dtype], act, xp, ldx, wp, ldw, pp, ldp, yp, ldy, dp, ldd, gp, ldg, bp,
                               1 if accumulate else 0, 0)
        ws, at = _work(B.tagc_linear_backward_workspace(a), x)
        B.tagc_linear_backward(a, at, _stream_of(stream, device))
    if stream is not None:
        _hand_over(user, dx if given[0] is None else None)
    if given[0] is not None or dw is not None or db is not None:
        increment_version(_counted(given))
    return dx


_KINDS = {"layer": B.TAGC_NORM_LAYER, "rms": B.TAGC_NORM_RMS}
_IDS = {torch.int32: B.TAGC_ID_I32, torch.int64: B.TAGC_ID_I64}


def _check_tensor(x, name, stream):
    if stream is not None:
        _check_stream(stream, x.device)
    if not x.is_cuda or x.dtype not in _TYPES:
        raise ValueError("%s: a CUDA tensor of float32 or bfloat16 is wanted" % name)


def _no_graph(what, *tensors):
    for t in tensors:
        if t is not None and t.requires_grad and torch.is_grad_enabled():
            warnings.warn("%s records no autograd graph: gradients are %s_backward's; call it under torch.no_grad()" % (what, what), stacklevel=3)
            return


def _all_ids(t, name, shape, device):
    """(address, type) of ids that lie one behind the other."""
    if t.dtype not in _IDS or t.device != device or t.shape != shape or not (t.is_contiguous() or t.numel() <= 1):
        raise ValueError("%s: contiguous int32 or int64 of %s on %s are wanted" % (name, tuple(shape), device))
    return t.data_ptr() or None, _IDS[t.dtype]


def _floats(t, name, shape, device):
    if t is None:
        return None
    if t.dtype != torch.float32 or t.device != device or t.shape != shape or not (t.is_contiguous() or t.numel() <= 1):
        raise ValueError("%s: contiguous float32 of %s on %s are wanted" % (name, tuple(shape), device))
    return t.data_ptr() or None


def _matrix(t, name, rows, cols, dtype, device):
    """_rows_of of a tensor [..., cols]; of one that lies one row behind the other nothing else is asked."""
    if t is None:
        return None, 0
    if t.is_contiguous() and t.dtype == dtype and t.device == device and t.numel() == rows * cols and t.dim() and t.shape[-1] == cols:
        return t.data_ptr() or None, cols
    return _rows_of(_flat(t, rows, cols), name, rows, cols, dtype, device)


def _like(x):
    return torch.empty_like(x) if x.is_contiguous() else x.new_empty(x.shape)


def norm(x, w=None, b=None, kind="layer", eps=1e-5, save=False, out=None, stream=None):
    """(y, stats): y = (x - mean) / sqrt(variance + eps) * w + b over the last dimension, or, kind "rms", without mean
    and b.  `save`: stats, float32 [rows, 2], for norm_backward (else None).  `out` may be given, and be x.  No autograd graph is
    recorded; `stream`: as for linear."""
    _check_tensor(x, "x", stream)
    _need(x.dim() >= 1, "x: a row at least is wanted")
    _need(kind in _KINDS, "kind: one of layer, rms is wanted")
    _no_graph("norm", x, w, b)
    shape, dtype, device = x.shape, x.dtype, x.device
    n = shape[-1]
    m = shape[0] if len(shape) == 2 else math.prod(shape[:-1])
    xp, ldx = _matrix(x, "x", m, n, dtype, device)
    wp, bp = _vector(w, "w", n, dtype, device), _vector(b, "b", n, dtype, device)
    given, stats, sp, user = out, None, None, None if stream is None else torch.cuda.current_stream(device)
    if out is not None:
        _need(out.shape == shape, "out: x's shape is wanted")
        yp, ldy = _matrix(out, "out", m, n, dtype, device)
    with _at(device, stream):
        if out is None:
            out = _like(x)
            yp, ldy = out.data_ptr() or None, n
        if save:
            stats = torch.empty((m, 2), dtype=torch.float32, device=device)
            sp = stats.data_ptr() or None
        B.tagc_norm_forward(B.tagc_norm(m, n, _TYPES[dtype], _KINDS[kind], eps, xp, ldx, wp, bp, yp, ldy, sp), _stream_of(stream, device))
    if stream is not None:
        _hand_over(user, out if given is None else None, stats)
    if given is not None:
        increment_version(_counted((given,)))
    return out, stats


def norm_backward(dy, x, w, stats, kind="layer", residual=None, dx=None, dw=None, db=None, accumulate=False, need_dx=True, stream=None):
    """dx (None without need_dx), plus `residual`, the gradient that came around the layer.  With `dw` and `db` ([width], views
    into a bucket's gradient) given, the weight's and the bias's gradient are written there, or added to what is there (accumulate).
    `w` may be None; `stats`: what norm(save=True) gave; `dx` may be dy, x or the residual.  `stream`: as for linear."""
    _check_tensor(x, "x", stream)
    _need(x.dim() >= 1, "x: a row at least is wanted")
    _need(kind in _KINDS, "kind: one of layer, rms is wanted")
    _need(need_dx or (dx is None and residual is None), "dx or residual is given, but need_dx is not")
    shape, dtype, device = x.shape, x.dtype, x.device
    n = shape[-1]
    m = math.prod(shape[:-1])
    xp, ldx = _matrix(x, "x", m, n, dtype, device)
    yp, ldy = _matrix(dy, "dy", m, n, dtype, device)
    rp, ldr = _matrix(residual, "residual", m, n, dtype, device)
    dp, ldd = _matrix(dx, "dx", m, n, dtype, device)
    wp, gp, bp = (_vector(t, name, n, dtype, device) for t, name in ((w, "w"), (dw, "dw"), (db, "db")))
    sp = _floats(stats, "stats", (m, 2), device)
    given, user = (dx, dw, db), None if stream is None else torch.cuda.current_stream(device)
    with _at(device, stream):
        if need_dx and dx is None:
            dx = _like(x)
            dp, ldd = dx.data_ptr() or None, n
        a = B.tagc_norm_grad(m, n, _TYPES[dtype], _KINDS[kind], xp, ldx, wp, sp, yp, ldy, rp, ldr, dp, ldd, gp, bp, 1 if accumulate else 0, 0)
        ws, at = _work(B.tagc_norm_backward_workspace(a), x)
        B.tagc_norm_backward(a, at, _stream_of(stream, device))
    if stream is not None:
        _hand_over(user, dx if given[0] is None else None)
    if given[0] is not None or dw is not None or db is not None:
        increment_version(_counted(given))
    return dx


def embedding(ids, table, scale=1.0, residual=None, out=None, stream=None):
    """scale * table[ids] + residual, [*ids.shape, width].  ids: int32 or int64; one outside the table is no token, and its row of
    the table counts as zeros.  `out` may be given, and be the residual.  No autograd graph is recorded; `stream`: as for linear."""
    _check_tensor(table, "table", stream)
    _need(table.dim() == 2, "table: [vocab, width] is wanted")
    _no_graph("embedding", table, residual)
    v, n = table.shape
    dtype, device = table.dtype, table.device
    m, shape = ids.numel(), (*ids.shape, n)
    ip, wide = _all_ids(ids, "ids", ids.shape, device)
    tp, ldt = _matrix(table, "table", v, n, dtype, device)
    for t, name in ((residual, "residual"), (out, "out")):
        _need(t is None or t.shape == shape, "%s: the shape %s is wanted" % (name, shape))
    rp, ldr = _matrix(residual, "residual", m, n, dtype, device)
    yp, ldy = _matrix(out, "out", m, n, dtype, device)
    given, user = out, None if stream is None else torch.cuda.current_stream(device)
    with _at(device, stream):
        if out is None:
            out = table.new_empty(shape)
            yp, ldy = out.data_ptr() or None, n
        a = B.tagc_embedding(m, n, v, _TYPES[dtype], wide, scale, ip, tp, ldt, rp, ldr, yp, ldy)
        B.tagc_embedding_forward(a, _stream_of(stream, device))
    if stream is not None:
        _hand_over(user, out if given is None else None)
    if given is not None:
        increment_version(_counted((given,)))
    return out


def embedding_backward(dy, ids, dtable, scale=1.0, accumulate=False, stream=None):
    """The table's gradient, written into `dtable` ([vocab, width], a view into a bucket's gradient; zeros where a row has no
    token), or added to what is there (accumulate).  Sums are taken in the tokens' order: results repeat.  `stream`: as for linear."""
    _check_tensor(dtable, "dtable", stream)
    _need(dtable.dim() == 2, "dtable: [vocab, width] is wanted")
    v, n = dtable.shape
    dtype, device = dtable.dtype, dtable.device
    m = ids.numel()
    ip, wide = _all_ids(ids, "ids", ids.shape, device)
    _need(dy.shape == (*ids.shape, n), "dy: the shape %s is wanted" % ((*ids.shape, n),))
    yp, ldy = _matrix(dy, "dy", m, n, dtype, device)
    tp, ldt = _matrix(dtable, "dtable", v, n, dtype, device)
    with _at(device, stream):
        a = B.tagc_embedding_grad(m, n, v, _TYPES[dtype], wide, scale, ip, yp, ldy, tp, ldt, 1 if accumulate else 0, 0)
        ws, at = _work(B.tagc_embedding_backward_workspace(a), dtable)
        B.tagc_embedding_backward(a, at, _stream_of(stream, device))
    increment_version(_counted((dtable,)))


def _loss_operands(x, w, ids, logits, temperature, stream):
    """What both passes of a loss have: (rows, in, vocab, terms), the operands' fields, the shape of a number for each row."""
    _check_tensor(x, "x", stream)
    if w.dim() != 2 or x.dim() < 1 or x.shape[-1] != w.shape[1]:
        raise ValueError("x is [..., in] and w [vocab, in]: got %s and %s" % (tuple(x.shape), tuple(w.shape)))
    _need(temperature > 0 and math.isfinite(temperature), "temperature: over 0 is wanted")
    dtype, device, shape = x.dtype, x.device, x.shape[:-1]
    v, k = w.shape
    m = math.prod(shape)
    if logits is None:
        terms = 1
        ip, wide = _all_ids(ids, "targets", shape, device)
        ap = None
    else:
        _need(ids.dim() == len(shape) + 1 and ids.shape[:-1] == shape, "ids: [..., terms] of x's rows are wanted")
        terms = ids.shape[-1]
        ip, wide = _all_ids(ids, "ids", ids.shape, device)
        ap = _floats(logits, "logits", ids.shape, device)
    xp, ldx = _matrix(x, "x", m, k, dtype, device)
    wp, ldw = _matrix(w, "w", v, k, dtype, device)
    return (m, k, v, terms), wide, (xp, ldx, wp, ldw, ip, ap), shape


def _loss(x, w, ids, logits, temperature, save, stream):
    size, wide, operands, shape = _loss_operands(x, w, ids, logits, temperature, stream)
    device, saved, sp, user = x.device, None, None, None if stream is None else torch.cuda.current_stream(x.device)
    with _at(device, stream):
        loss = torch.empty(shape, dtype=torch.float32, device=device)
        if save:
            saved = torch.empty((size[0], 1 + size[3]), dtype=torch.float32, device=device)
            sp = saved.data_ptr() or None
        a = B.tagc_loss(*size, _TYPES[x.dtype], wide, 0, temperature, *operands, loss.data_ptr() or None, sp)
        ws, at = _work(B.tagc_loss_forward_workspace(a), x)
        B.tagc_loss_forward(a, at, _stream_of(stream, device))
    if stream is not None:
        _hand_over(user, loss, saved)
    return loss, saved


def _loss_backward(dloss, x, w, ids, logits, saved, temperature, dx, dw, accumulate, need_dx, stream):
    size, wide, operands, shape = _loss_operands(x, w, ids, logits, temperature, stream)
    m, k, v, terms = size
    dtype, device = x.dtype, x.device
    _need(need_dx or dx is None, "dx is given, but need_dx is not")
    sp = _floats(saved, "saved", (m, 1 + terms), device)
    _need(dloss.shape == shape or (dloss.numel() == 1 and dloss.dim() <= 1), "dloss: a number for each row, or one, is wanted")
    one = dloss.numel() > 0 and all(step == 0 or n == 1 for step, n in zip(dloss.stride(), dloss.shape))     # (also one that is expanded)
    gp = _floats(dloss.as_strided((1,), (1,)) if one else dloss, "dloss", (1,) if one else shape, device)
    _need(dx is None or dx.shape == x.shape, "dx: x's shape is wanted")
    dp, ldd = _matrix(dx, "dx", m, k, dtype, device)
    wp, ldw = _matrix(dw, "dw", v, k, dtype, device)
    given, user = (dx, dw), None if stream is None else torch.cuda.current_stream(device)
    with _at(device, stream):
        if need_dx and dx is None:
            dx = _like(x)
            dp, ldd = dx.data_ptr() or None, k
        a = B.tagc_loss_grad(*size, _TYPES[dtype], wide, 1 if accumulate else 0, temperature, *operands, sp, gp, 0 if one else 1, 0, dp, ldd, wp, ldw)
        ws, at = _work(B.tagc_loss_backward_workspace(a), x)
        B.tagc_loss_backward(a, at, _stream_of(stream, device))
    if stream is not None:
        _hand_over(user, dx if given[0] is None else None)
    if given[0] is not None or dw is not None:
        increment_version(_counted(given))
    return dx


def cross_entropy(x, w, targets, save=False, stream=None):
    """(loss, saved): of every row of x [..., in] the softmax cross entropy of its scores x w^T over a vocabulary w [vocab, in] against
    its target (int32 or int64), float32; the scores are no result, and held as a whole only where they are few.  A target outside [0, vocab) is ignored: loss 0, no gradient.
    `save`: saved, float32 [rows, 2] (the log-sum of the scores' exponentials, the target's score), for cross_entropy_backward (else
    None).  No autograd graph is recorded; `stream`: as for linear."""
    _no_graph("cross_entropy", x, w)
    return _loss(x, w, targets, None, 1.0, save, stream)


def cross_entropy_backward(dloss, x, w, targets, saved, dx=None, dw=None, accumulate=False, need_dx=True, stream=None):
    """dx (None without need_dx).  `dloss`: float32, a number for each row, or one for all (such as 1 / the rows that count; an expanded one is one).  With `dw`
    ([vocab, in], a view into a bucket's gradient) given, w's gradient is written there, or added to what is there (accumulate).
    `saved`: what cross_entropy(save=True) gave.  `stream`: as for linear."""
    return _loss_backward(dloss, x, w, targets, None, saved, 1.0, dx, dw, accumulate, need_dx, stream)


def distill(x, w, ids, logits, temperature=1.0, save=False, stream=None):
    """(loss, saved): of every row of x [..., in] the Kullback-Leibler divergence of softmax(x w^T / temperature) over a vocabulary w
    [vocab, in] from a teacher's distribution, which is softmax(logits / temperature) over the row's tokens ids [..., terms] (the teacher's
    largest scores; int32 or int64, logits float32).  A token outside [0, vocab), or one with the logit -inf, is none; a row
    without any has loss 0 and no gradient.  `saved`: [rows, 1 + terms], as for cross_entropy.  (To have gradients of
    the usual size at a temperature, weigh dloss by its square.)"""
    _no_graph("distill", x, w, logits)
    _need(logits is not None, "logits: the teacher's are wanted")
    return _loss(x, w, ids, logits, temperature, save, stream)


def distill_backward(dloss, x, w, ids, logits, saved, temperature=1.0, dx=None, dw=None, accumulate=False, need_dx=True, stream=None):
    """dx and dw of distill, as cross_entropy_backward's; none for the teacher."""
    _need(logits is not None, "logits: the teacher's are wanted")
    return _loss_backward(dloss, x, w, ids, logits, saved, temperature, dx, dw, accumulate, need_dx, stream)


def dense_views(bucket):
    """Per segment of a TagcBucket with a dense output: its summed gradient, float32, a view that the next decode
    fills anew; None for a segment that is not compressed."""
    _need(bucket.out_dense is not None, "a bucket made with dense=True is wanted")
    dense, views, at = bucket.out_dense.view(torch.float32), [], 0
    for _, length, _, flags in bucket.segments:
        if not flags & B.TAGC_SEG_COMPRESS:
            views.append(None)
            continue
        views.append(dense[at:at + length])
        at += -(-length // 32) * 32  # segments begin at multiples of 32 there
    return views


class AdamW:
    """AdamW over a list of tensors, each contiguous: the library's plan, its table on the device, the
    moments (made here, zero, if they are not given) and the control block.

    `params`, `grads`: float32 or bfloat16, tensor by tensor.  `copies`: bfloat16 tensors that get
    the updated parameters, or None (for single ones too).  `bits`: 32, or 8 (m, v: uint8 of the tensor's
    length; bases: int32, one per 256 elements).  `groups`: (lr, weight_decay) pairs, `group_of`: each
    tensor's.  `opt.groups = ...` changes them between steps.  Without params only grad_norm() can be
    called.  The tensors must stay where they are: a gradient is written into, not replaced.  What a step
    writes must lie apart: each parameter is given once."""

    def __init__(self, params=None, grads=(), m=None, v=None, bases=None, copies=None, groups=((1e-3, 0.01),),
                 group_of=None, betas=(0.9, 0.999), eps=1e-8, bits=32, grad_scale=1.0, max_norm=0.0, seed=0,
                 first_step=1):
        self.plan = None
        self._begun = False
        grads = list(grads)
        n = len(grads)
        _need(n > 0, "no gradients")
        self.device = grads[0].device
        _need(self.device.type == "cuda", "libtagc needs a GPU: no CPU path exists")
        group_of = [0] * n if group_of is None else list(group_of)
        self.groups = groups
        self.bits, self.grads, self._clips = bits, grads, max_norm > 0
        self.params = list(params) if params is not None else None
        lists = {"params": self.params, "copies": copies, "m": m, "v": v, "bases": bases, "group_of": group_of}
        for name, given in lists.items():
            _need(given is None or len(given) == n, "%s: %d for %d gradients" % (name, 0 if given is None else len(given), n))
        _need(all(0 <= g < len(self.groups) for g in group_of), "group_of: there are %d groups" % len(self.groups))
        _need(bits in (8, 32), "bits: 8 or 32")
        _need(first_step >= 1, "first_step: 1 or more")
        made = []
        if self.params is not None and m is None:
            _need(v is None and bases is None, "m, v (and bases) are given together or not at all")
            state = torch.float32 if bits == 32 else torch.uint8
            m, v = ([torch.zeros(g.numel(), dtype=state, device=self.device) for g in grads] for _ in range(2))
            if bits == 8:
                bases = [torch.zeros(self._blocks(g), dtype=torch.int32, device=self.device) for g in grads]
            made = [*m, *v, *(bases or ())]
        self.m, self.v, self.bases, self.copies = m, v, bases, copies
        rows = (B.tagc_tensor * n)()
        for i, g in enumerate(grads):
            r, k = rows[i], g.numel()
            r.length, r.group = k, group_of[i]
            r.grad, r.grad_type = self._one(g, "grads", i, k, tuple(_TYPES)), _TYPES[g.dtype]
            if self.params is None:
                continue
            p = self.params[i]
            r.param, r.param_type = self._one(p, "params", i, k, tuple(_TYPES)), _TYPES[p.dtype]
            state = (torch.float32,) if bits == 32 else (torch.uint8,)
            r.m, r.v = self._one(m[i], "m", i, k, state), self._one(v[i], "v", i, k, state)
            if bits == 8:
                r.bases = self._one(bases[i], "bases", i, self._blocks(g), (torch.int32,))
            if copies is not None and copies[i] is not None:
                r.copy = self._one(copies[i], "copies", i, k, (torch.bfloat16,))
        self._check_apart(rows)
        # (a graph that kept a parameter for its backward pass raises there behind a step, as behind torch's own optimizers)
        self._written = _counted([*(self.params or ()), *(copies or ())])
        cfg = B.tagc_optim_config(beta1=betas[0], beta2=betas[1], eps=eps, grad_scale=grad_scale, max_norm=max_norm,
                                  seed=seed, moment_bits=bits)
        self.plan = B.tagc_optim_plan(cfg, rows)
        self.sizes = B.tagc_optim_plan_sizes(self.plan)
        self.table = _bytes(self.sizes.table_bytes, self.device)
        # step, skipped, apply, norm, factor, lr_scale, ...: see tagc_optim_control
        start = torch.zeros(16, dtype=torch.int32)
        start[0] = first_step - 1
        start.view(torch.float32)[5] = 1.0
        self.control = start.to(self.device)
        f = self.control.view(torch.float32)
        self.norm, self.factor, self.lr_scale = f[3], f[4], f[5]
        self._table, self._control = self.table.data_ptr(), self.control.data_ptr()
        # what is made here, and the streams that it has been used on: the one it belongs to first
        home = torch.cuda.current_stream(self.device)
        self._made, self._streams = [self.table, self.control, *made], {home.cuda_stream}
        with _at(self.device):
            B.tagc_optim_upload(self.plan, self._table, home.cuda_stream)
        home.synchronize()

    @staticmethod
    def _blocks(g):
        return -(-g.numel() // B.TAGC_MOMENT_BLOCK)

    def _one(self, t, name, i, k, types):
        _need(t.dtype in types and t.device == self.device and t.numel() == k and (t.is_contiguous() or k <= 1),
              "%s[%d]: a contiguous tensor of %d, %s on %s, is wanted" % (name, i, k, " or ".join(map(str, types)), self.device))
        return t.data_ptr() if k else None

    def _check_apart(self, rows):
        """What a step writes is written by the workgroup that has read it, and by no other one: no parameter twice, no moments
        of two.  (A gradient may lie in the place of something of its tensor's that it is replaced by element by element.)"""
        spans = []
        for r in rows:
            if not r.length or not r.param:
                continue
            size, grad_size = (4, 2)[r.param_type], (4, 2)[r.grad_type]
            own = [(r.param, r.length * size), (r.copy, r.length * 2), (r.bases, -(-r.length // B.TAGC_MOMENT_BLOCK) * 4)]
            own += [(p, r.length * (self.bits // 8)) for p in (r.m, r.v)]
            spans += [(p, p + n, True) for p, n in own if p]
            if (r.grad, r.length * grad_size) not in own:
                spans.append((r.grad, r.grad + r.length * grad_size, False))
        spans.sort()
        written = read = 0      # the ends of what began before
        for start, end, write in spans:
            _need(start >= written and not (write and start < read),
                  "params, m, v, bases, copies and grads: what is written must lie apart from everything else")
            if write:
                written = max(written, end)
            else:
                read = max(read, end)

    def _on(self, stream):
        """The address of the stream that a call runs on.  What was made here is not handed out again before the streams that
        used it are done, also where the object goes first."""
        if stream is not None:
            _check_stream(stream, self.device)
        at = _stream_of(stream, self.device)
        if at not in self._streams:
            s = stream if stream is not None else torch.cuda.current_stream(self.device)
            for t in self._made:
                t.record_stream(s)
            self._streams.add(at)
        return at

    @property
    def groups(self):
        return self._groups

    @groups.setter
    def groups(self, groups):
        groups = tuple((float(lr), float(decay)) for lr, decay in groups)
        _need(not hasattr(self, "_groups") or len(groups) == len(self._groups), "groups: as many as there were are wanted")
        self._groups = groups
        self._group_array = (B.tagc_group * max(len(groups), 1))(*groups)

    def grad_norm(self, stream=None):
        """Begins a step; (norm, factor): device scalars, views of the control block."""
        with _at(self.device):
            B.tagc_grad_norm(self.plan, self._table, self._control, self._on(stream))
        self._begun = True
        return self.norm, self.factor

    def step(self, step=0, stream=None):
        """One step: the one that grad_norm() began, its learning rates times the device scalar
        `lr_scale`; or, with `step` > 0, that one, with the groups' learning rates (not of an optimizer that clips)."""
        if step:
            _need(0 < step < 1 << 32, "step: 1 or more, less than 2^32, or 0 for the one that grad_norm() began")
            _need(not self._clips, "a given step is not clipped, and there is a max_norm: grad_norm(), then step()")
        elif not self._begun:  # (the control block would say that there is nothing to apply)
            raise RuntimeError("step() carries on what grad_norm() began: call that first, or give the step's number")
        with _at(self.device):
            B.tagc_adamw_step(self.plan, self._table, self._group_array, step, self._control, self._on(stream))
        increment_version(self._written)

    def unpack(self, stream=None):
        """(m, v): what 8-bit moments stand for, bfloat16, the tensors one behind the other."""
        at, user = self._on(stream), torch.cuda.current_stream(self.device)
        with _at(self.device, stream):
            m, v = (torch.empty(self.sizes.n_elems, dtype=torch.bfloat16, device=self.device) for _ in range(2))
            B.tagc_adamw_unpack(self.plan, self._table, m.data_ptr() or None, v.data_ptr() or None, at)
        if stream is not None:
            _hand_over(user, m, v)
        return m, v

    def close(self):
        if self.plan is not None:
            B.tagc_optim_destroy(self.plan)
            self.plan = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
