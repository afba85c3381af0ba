"""The two ends of a data-parallel step around the exchange: linear layers whose backward pass
writes into a bucket's gradient, and the optimizer behind it.  Device memory and argument
marshalling only; all arithmetic is the library's (include/tagc_train.h).

    y, pre = linear(x, w, b, activation="gelu", save=True)
    dx = linear_backward(dy, x, w, pre, activation="gelu", dw=bucket_grad_view, db=...)
    ...                                # the exchange: bucket.TagcBucket
    opt = AdamW(params=..., grads=..., max_norm=1.0, bits=8)
    opt.grad_norm()                    # norm, clip factor and step count, on the device
    opt.step()
"""
from __future__ import annotations

import torch

from . import binding as B
from .bucket import _bytes, _stream_ptr

_TYPES = {torch.float32: B.TAGC_F32, torch.bfloat16: B.TAGC_BF16}
_ACTS = {None: B.TAGC_ACT_NONE, "none": B.TAGC_ACT_NONE, "relu": B.TAGC_ACT_RELU,
         "gelu": B.TAGC_ACT_GELU, "gelu_tanh": B.TAGC_ACT_GELU_TANH, "silu": B.TAGC_ACT_SILU}


def _need(condition, what):
    if not condition:
        raise ValueError(what)


def _rows_of(t, name, shape, like):
    """(address, elements from row to row) of a matrix; None for None."""
    if t is None:
        return None, 0
    _need(t.dtype == like.dtype and t.device == like.device, "%s: a %s on %s is wanted" % (name, like.dtype, like.device))
    _need(tuple(t.shape) == tuple(shape), "%s has shape %s, %s is wanted" % (name, tuple(t.shape), tuple(shape)))
    rows, cols = shape
    _need(cols <= 1 or rows == 0 or t.stride(1) == 1, "%s: a row's elements must be neighbours" % name)
    # (of a single row the stride says nothing; of no elements neither does the address)
    ld = t.stride(0) if rows > 1 and cols > 0 else cols
    _need(ld >= cols, "%s: rows must not overlap" % name)
    return t.data_ptr() if t.numel() else None, ld


def _vector(t, name, n, like):
    if t is None:
        return None
    _need(t.dtype == like.dtype and t.device == like.device, "%s: a %s on %s is wanted" % (name, like.dtype, like.device))
    _need(tuple(t.shape) == (n,) and (n <= 1 or t.stride(0) == 1), "%s: a contiguous vector of %d is wanted" % (name, n))
    return t.data_ptr() if n else None


def _check_input(x, w):
    _need(x.is_cuda and x.dtype in _TYPES, "x: a CUDA tensor of float32 or bfloat16 is wanted")
    _need(w.dim() == 2 and x.dim() >= 2 and x.shape[-1] == w.shape[1],
          "x is [..., in] and w [out, in]: got %s and %s" % (tuple(x.shape), tuple(w.shape)))


def _flat(t, cols):
    """[..., cols] as [rows, cols] without a copy."""
    if t is None or t.dim() == 2:
        return t
    rows = t.numel() // cols if cols else t[..., 0:0].flatten(0, -2).shape[0]
    return t.view(rows, cols)


def _act(name):
    _need(name in _ACTS, "activation: one of %s is wanted" % ", ".join(k for k in _ACTS if k))
    return _ACTS[name]


def _work(nbytes, x, stream):
    """A call's workspace; kept from reuse until `stream`, where it is not the current one, is done."""
    if not nbytes:
        return None, None
    ws = _bytes(nbytes, x.device)
    if stream is not None:
        ws.record_stream(stream)
    return ws, ws.data_ptr()


def linear(x, w, bias=None, residual=None, activation=None, save=False, out=None, pre=None, stream=None):
    """(y, pre): y = activation(x w^T + bias) + residual.  x: [..., in], w: [out, in].  `save`: pre =
    x w^T + bias for linear_backward (else None).  `out` and `pre` may be given; `out` may be
    the residual.  Tensors made here belong to the current stream."""
    _check_input(x, w)
    n, k = w.shape
    lead = x.shape[:-1]
    x2 = _flat(x, k)
    m = x2.shape[0]
    act = _act(activation)
    _need(not (pre is not None and not save), "pre is given, but save is not")
    y = torch.empty(*lead, n, dtype=x.dtype, device=x.device) if out is None else out
    if save and pre is None:
        pre = torch.empty(*lead, n, dtype=x.dtype, device=x.device)
    a = B.tagc_linear(rows=m, in_=k, out=n, dtype=_TYPES[x.dtype], activation=act)
    a.x, a.ldx = _rows_of(x2, "x", (m, k), x)
    a.w, a.ldw = _rows_of(w, "w", (n, k), x)
    a.bias = _vector(bias, "bias", n, x)
    a.residual, a.ldr = _rows_of(_flat(residual, n), "residual", (m, n), x)
    a.y, a.ldy = _rows_of(_flat(y, n), "out", (m, n), x)
    a.pre, a.ldp = _rows_of(_flat(pre, n), "pre", (m, n), x)
    ws, at = _work(B.tagc_linear_forward_workspace(a), x, stream)
    B.tagc_linear_forward(a, at, _stream_ptr(stream))
    return y, pre


def linear_backward(dy, x, w, pre=None, activation=None, dx=None, dw=None, db=None, accumulate=False,
                    need_dx=True, stream=None):
    """dx (None without need_dx).  With `dw` ([out, in], a view into a bucket's gradient) and `db` ([out])
    given, the weight's and the bias's gradient are written there, or added to what is there
    (accumulate).  `pre`: what linear(save=True) gave; None without an activation."""
    _check_input(x, w)
    n, k = w.shape
    x2, dy2 = _flat(x, k), _flat(dy, n)
    m = x2.shape[0]
    act = _act(activation)
    _need((act != B.TAGC_ACT_NONE) == (pre is not None), "pre is wanted with an activation, and only then")
    _need(need_dx or dx is None, "dx is given, but need_dx is not")
    if need_dx and dx is None:
        dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    a = B.tagc_linear_grad(rows=m, in_=k, out=n, dtype=_TYPES[x.dtype], activation=act,
                           accumulate=int(bool(accumulate)))
    a.x, a.ldx = _rows_of(x2, "x", (m, k), x)
    a.w, a.ldw = _rows_of(w, "w", (n, k), x)
    a.pre, a.ldp = _rows_of(_flat(pre, n), "pre", (m, n), x)
    a.dy, a.lddy = _rows_of(dy2, "dy", (m, n), x)
    a.dx, a.lddx = _rows_of(_flat(dx, k), "dx", (m, k), x)
    a.dw, a.lddw = _rows_of(dw, "dw", (n, k), x)
    a.db = _vector(db, "db", n, x)
    ws, at = _work(B.tagc_linear_backward_workspace(a), x, stream)
    B.tagc_linear_backward(a, at, _stream_ptr(stream))
    return dx


class AdamW:
    """AdamW over a list of tensors, each contiguous: the library's plan, its table on the device, the
    moments (made here, zero, if they are not given) and the control block.

    `params`, `grads`: float32 or bfloat16, tensor by tensor.  `copies`: bfloat16 tensors that get
    the updated parameters, or None (for single ones too).  `bits`: 32, or 8 (m, v: uint8 of the tensor's
    length; bases: int32, one per 256 elements).  `groups`: (lr, weight_decay) pairs, `group_of`: each
    tensor's.  groups may be changed between steps.  Without params only grad_norm() can be
    called.  The tensors must stay where they are: a gradient is written into, not replaced."""

    def __init__(self, params=None, grads=(), m=None, v=None, bases=None, copies=None, groups=((1e-3, 0.01),),
                 group_of=None, betas=(0.9, 0.999), eps=1e-8, bits=32, grad_scale=1.0, max_norm=0.0, seed=0,
                 first_step=1):
        self.plan = None
        grads = list(grads)
        n = len(grads)
        _need(n > 0, "no gradients")
        self.device = grads[0].device
        _need(self.device.type == "cuda", "libtagc needs a GPU: no CPU path exists")
        group_of = [0] * n if group_of is None else list(group_of)
        self.groups = [tuple(g) for g in groups]
        self.bits, self.grads = bits, grads
        self.params = list(params) if params is not None else None
        lists = {"params": self.params, "copies": copies, "m": m, "v": v, "bases": bases, "group_of": group_of}
        for name, given in lists.items():
            _need(given is None or len(given) == n, "%s: %d for %d gradients" % (name, 0 if given is None else len(given), n))
        _need(all(0 <= g < len(self.groups) for g in group_of), "group_of: there are %d groups" % len(self.groups))
        _need(bits in (8, 32), "bits: 8 or 32")
        _need(first_step >= 1, "first_step: 1 or more")
        if self.params is not None and m is None:
            _need(v is None and bases is None, "m, v (and bases) are given together or not at all")
            state = torch.float32 if bits == 32 else torch.uint8
            m, v = ([torch.zeros(g.numel(), dtype=state, device=self.device) for g in grads] for _ in range(2))
            if bits == 8:
                bases = [torch.zeros(self._blocks(g), dtype=torch.int32, device=self.device) for g in grads]
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
        B.tagc_optim_upload(self.plan, self.table.data_ptr(), _stream_ptr())
        torch.cuda.current_stream().synchronize()

    @staticmethod
    def _blocks(g):
        return -(-g.numel() // B.TAGC_MOMENT_BLOCK)

    def _one(self, t, name, i, k, types):
        _need(t.dtype in types and t.device == self.device and t.numel() == k and (t.is_contiguous() or k <= 1),
              "%s[%d]: a contiguous tensor of %d, %s on %s, is wanted" % (name, i, k, " or ".join(map(str, types)), self.device))
        return t.data_ptr() if k else None

    def grad_norm(self, stream=None):
        """Begins a step; (norm, factor) as device scalars, views of the control block."""
        B.tagc_grad_norm(self.plan, self.table.data_ptr(), self.control.data_ptr(), _stream_ptr(stream))
        f = self.control.view(torch.float32)
        return f[3], f[4]

    def step(self, step=0, stream=None):
        """One step: the one that grad_norm() began, or, with `step` > 0, that one, unclipped."""
        B.tagc_adamw_step(self.plan, self.table.data_ptr(), self.groups, step,
                          self.control.data_ptr(), _stream_ptr(stream))

    @property
    def lr_scale(self):
        """Device scalar that the groups' learning rates are multiplied by in step(0)."""
        return self.control.view(torch.float32)[5]

    def unpack(self, stream=None):
        """(m, v): what 8-bit moments stand for, bfloat16, the tensors one behind the other."""
        m, v = (torch.empty(self.sizes.n_elems, dtype=torch.bfloat16, device=self.device) for _ in range(2))
        B.tagc_adamw_unpack(self.plan, self.table.data_ptr(), m.data_ptr() or None, v.data_ptr() or None,
                            _stream_ptr(stream))
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
