"""What the operators at a language model's ends are timed on, in plain torch and as the library's
kernels.

Around the blocks, whose linear layers `perf/operators.py` has, a model takes its tokens' vectors from
a table, is normalised in front of every layer, and ends in a loss over its vocabulary.  Their
gradients are segments of the same flat gradient:

  op = "norm"               y = (x - mean) / sqrt(variance + eps) * w + b ("layer"), or without mean and
                            b ("rms"); the statistics where a backward pass follows
  op = "norm_backward"      dx, with the gradient that came around the layer added; dw, db
  op = "embed"              y = scale * table[id], and what is added to it (positions)
  op = "embed_backward"     the table's gradient
  op = "loss"               softmax cross entropy of x w^T against a token each, without keeping the
                            scores x w^T; tokens outside the vocabulary are ignored
  op = "loss_backward"      dx and dw, from the rows' log-sums of exponentials
  op = "distill"            the divergence from a teacher's distribution over its `terms` largest scores,
                            renormalised, at a temperature; terms outside the vocabulary are none
  op = "distill_backward"   dx and dw of that

Sizes are those of this repository's GPT-2-like and Llama-like workloads (width 768 with 50257
tokens, width 4096 with 32000), and ragged ones.
"""
from __future__ import annotations

import math

import torch

own = False

_F = {"f32": torch.float32, "bf16": torch.bfloat16}
_EPS = 1e-5

_NORM = dict(op="norm", rows=0, width=0, dtype="bf16", kind="rms", bias=False, save=False, residual=False, add=False)
_EMBED = dict(op="embed", rows=0, width=0, vocab=0, dtype="bf16", scale=1.0, residual=False, add=False)
_LOSS = dict(op="loss", rows=0, width=0, vocab=0, dtype="bf16", ignored=0.0, terms=1, temperature=1.0, save=False, add=False)


def listed():
    return [
        # One token through a GPT-2-like model's norm: latency is all there is.
        dict(name="norm_token_f32", **{**_NORM, "rows": 1, "width": 768, "dtype": "f32", "kind": "layer", "bias": True}),
        # The norm in front of a Llama-like block's layers, in training.
        dict(name="norm_llama_bf16", **{**_NORM, "rows": 8192, "width": 4096, "save": True}),
        # A GPT-2-like norm backwards, in fp32 as the paper trains: weight, bias, and what came around.
        dict(name="norm_backward_gpt2_f32", **{**_NORM, "op": "norm_backward", "rows": 8192, "width": 768, "dtype": "f32", "kind": "layer", "bias": True, "residual": True}),
        # A Llama-like norm backwards, its weight's gradient added to earlier micro-batches'.
        dict(name="norm_backward_llama_bf16", **{**_NORM, "op": "norm_backward", "rows": 8192, "width": 4096, "residual": True, "add": True}),
        # A batch's tokens looked up.
        dict(name="embed_llama_bf16", **{**_EMBED, "rows": 8192, "width": 4096, "vocab": 32000}),
        # A short batch's gradient into a table with an odd number of rows: zeros are most of it.
        dict(name="embed_backward_gpt2_f32", **{**_EMBED, "op": "embed_backward", "rows": 1023, "width": 768, "vocab": 50257, "dtype": "f32", "scale": 768 ** 0.5}),
        # Several sequences' gradient, frequent tokens among them.
        dict(name="embed_backward_llama_bf16", **{**_EMBED, "op": "embed_backward", "rows": 16384, "width": 4096, "vocab": 32000}),
        # Odd sizes in fp32, a small vocabulary.
        dict(name="distill_odd_f32", **{**_LOSS, "op": "distill", "rows": 333, "width": 777, "vocab": 1001, "dtype": "f32", "terms": 17, "temperature": 2.0, "ignored": 0.1, "save": True}),
        # A Llama-like model's loss, evaluated, or the first half of a training step.
        dict(name="loss_llama_bf16", **{**_LOSS, "rows": 8192, "width": 4096, "vocab": 32000, "ignored": 0.1, "save": True}),
        # A GPT-2-like sequence's loss backwards in fp32.
        dict(name="loss_backward_gpt2_f32", **{**_LOSS, "op": "loss_backward", "rows": 1024, "width": 768, "vocab": 50257, "dtype": "f32"}),
        # The second half of a Llama-like training step.
        dict(name="loss_backward_llama_bf16", **{**_LOSS, "op": "loss_backward", "rows": 4096, "width": 4096, "vocab": 32000, "ignored": 0.1}),
        # A student's second half: 64 terms of a teacher at every token, added to what the bucket has.
        dict(name="distill_backward_llama_bf16", **{**_LOSS, "op": "distill_backward", "rows": 2048, "width": 4096, "vocab": 32000, "terms": 64, "temperature": 2.0,
                                                    "ignored": 0.05, "add": True}),
    ]


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    """One more case of the same ranges: 1 to 16384 rows, widths of 64 to 8192 (losses: to 4096), vocabularies of
    200 to 131072, 1 to 128 terms; a third of the widths odd."""
    op = rng.choice(["norm", "norm_backward", "embed", "embed_backward", "loss", "loss_backward", "distill", "distill_backward"])
    while True:
        rows = int(_log_uniform(rng, 1, 16384.9))
        width = 64 * int(_log_uniform(rng, 1, 128.9 if op in ("norm", "norm_backward") else 64.9))
        if rng.random() < 0.33:
            width -= rng.randrange(1, 64)
        vocab = int(_log_uniform(rng, 200, 131072.9))
        dtype = rng.choice(["bf16", "bf16", "f32"])
        if op in ("norm", "norm_backward"):
            kind = rng.choice(["layer", "rms"])
            c = dict(_NORM, op=op, rows=rows, width=width, dtype=dtype, kind=kind, bias=kind == "layer")
            c["save"] = op == "norm" and rng.random() < 0.5
            c["residual"], c["add"] = (rng.random() < 0.5, rng.random() < 0.4) if op == "norm_backward" else (False, False)
            return c
        if op in ("embed", "embed_backward"):
            c = dict(_EMBED, op=op, rows=rows, width=width, vocab=vocab, dtype=dtype, scale=rng.choice([1.0, width ** 0.5]))
            c["residual"], c["add"] = op == "embed" and rng.random() < 0.4, op == "embed_backward" and rng.random() < 0.4
            if work(c)["bytes"] <= 4e8:
                return c
            continue
        c = dict(_LOSS, op=op, rows=rows, width=width, vocab=vocab, dtype=dtype, ignored=rng.choice([0.0, 0.1, 0.5]))
        if op in ("distill", "distill_backward"):
            c["terms"], c["temperature"] = int(_log_uniform(rng, 1, 128.9)), rng.choice([1.0, 2.0, 4.0])
        c["save"], c["add"] = op in ("loss", "distill"), op.endswith("backward") and rng.random() < 0.4
        w = work(c)
        if w["flops"] * (6 if dtype == "f32" else 1) <= 2.5e12 and w["bytes"] <= 7e8:
            return c


# ------------------------------------------------------------------ inputs


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(n, gen, dtype=torch.float32, scale=1.0):
    return torch.randn(n, generator=gen, device="cuda").mul_(scale).to(dtype)


def _tokens(rows, vocab, gen):
    """Tokens as text has them: the k-th most frequent about 1 / k times as often as the first, frequent ones all over the table."""
    u = torch.rand(rows, generator=gen, device="cuda", dtype=torch.float64)
    k = torch.exp(u * math.log(vocab + 1.0)).long().clamp_(1, vocab) - 1
    return (k * 7919 + 13) % vocab


def prepare(case, seed):
    gen = _gen(seed)
    c, t = case, _F[case["dtype"]]
    M, D = c["rows"], c["width"]
    s = {"case": c}
    if c["op"] in ("norm", "norm_backward"):
        # a residual stream's rows: scales that differ from row to row, some features larger, a mean
        s["x"] = (_normal((M, D), gen) * torch.exp(_normal((M, 1), gen) * 0.5) * torch.exp(_normal(D, gen) * 0.3) + 0.3 * _normal((M, 1), gen)).to(t)
        s["w"] = (1 + 0.1 * _normal(D, gen)).to(t)
        s["b"] = _normal(D, gen, t, 0.1) if c["bias"] else None
        if c["op"] == "norm_backward":
            s["dy"] = _normal((M, D), gen, t, 1e-3)
            s["residual"] = _normal((M, D), gen, t, 1e-3) if c["residual"] else None
            # the bucket's flat gradient: the weight's segment, then the bias's
            n = D * (1 + c["bias"])
            s["bucket"] = _normal(n, gen, t, 1e-2) if c["add"] else torch.zeros(n, device="cuda", dtype=t)
            s["stats"] = _stats(s["x"].double(), c["kind"]).float()
        return s
    if c["op"] in ("embed", "embed_backward"):
        s["ids"] = _tokens(M, c["vocab"], gen)
        if c["op"] == "embed":
            s["table"] = _normal((c["vocab"], D), gen, t, 0.02)
            s["residual"] = _normal((M, D), gen, t, 0.02) if c["residual"] else None
        else:
            s["dy"] = _normal((M, D), gen, t, 1e-3)
            s["dtable"] = _normal((c["vocab"], D), gen, t, 1e-3) if c["add"] else torch.zeros((c["vocab"], D), device="cuda", dtype=t)
        return s
    V, K = c["vocab"], c["terms"]
    w = _normal((V, D), gen, scale=D ** -0.5)
    targets = _tokens(M, V, gen)
    # what training leaves: the right token's score above the others', more in some rows than in others
    s["x"] = (_normal((M, D), gen) + w[targets] * (14 * torch.rand((M, 1), generator=gen, device="cuda"))).to(t)
    s["w"] = w.to(t)
    del w
    ignored = torch.rand(M, generator=gen, device="cuda") < c["ignored"]
    if c["op"] in ("loss", "loss_backward"):
        s["ids"] = torch.where(ignored, -1, targets)
    else:
        # a teacher's largest scores, falling, the next token first; short lists end in terms that are none
        step = 1 + torch.randint(0, max(1, V // max(2, 2 * K)), (M, 1), generator=gen, device="cuda")
        ids = (targets[:, None] + step * torch.arange(K, device="cuda")) % V
        s["ids"] = torch.where(ignored[:, None] & (torch.arange(K, device="cuda") >= K // 2), -1, ids)
        s["logits"] = torch.sort(3 * _normal((M, K), gen), dim=1, descending=True).values
    if c["op"].endswith("backward"):
        s["dloss"] = torch.full((M,), 1.0 / M, device="cuda")
        s["dw"] = _normal((V, D), gen, t, 1e-4) if c["add"] else torch.zeros((V, D), device="cuda", dtype=t)
        s["saved"] = _saved(s["x"], s["w"], _terms(s["ids"]), c["temperature"], torch.float64).float()
    return s


# ------------------------------------------------------------------ plain forms


def _stats(x, kind):
    mean = x.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(x[:, :1])
    return torch.cat([mean, ((x - mean).square().mean(1, keepdim=True) + _EPS) ** -0.5], 1)


def _norm_plain(s):
    c, x = s["case"], s["x"].float()
    stats = _stats(x, c["kind"])
    y = (x - stats[:, :1]) * stats[:, 1:] * s["w"].float()
    if c["bias"]:
        y = y + s["b"].float()
    return {"y": y.to(_F[c["dtype"]]), "stats": stats if c["save"] else None}


def _norm_backward_plain(s):
    c = s["case"]
    x, dy, stats = s["x"].float(), s["dy"].float(), s["stats"]
    h = (x - stats[:, :1]) * stats[:, 1:]
    u = dy * s["w"].float()
    dx = u - h * (u * h).mean(1, keepdim=True)
    if c["kind"] == "layer":
        dx = dx - u.mean(1, keepdim=True)
    dx = dx * stats[:, 1:]
    if c["residual"]:
        dx = dx + s["residual"].float()
    grads = torch.cat([(dy * h).sum(0)] + ([dy.sum(0)] if c["bias"] else []))
    s["bucket"].copy_(grads + s["bucket"].float() if c["add"] else grads)
    return {"dx": dx.to(_F[c["dtype"]]), "bucket": s["bucket"]}


def _embed_plain(s):
    c = s["case"]
    y = s["table"][s["ids"]].float() * c["scale"]
    if c["residual"]:
        y = y + s["residual"].float()
    return {"y": y.to(_F[c["dtype"]])}


def _embed_backward_plain(s):
    c = s["case"]
    grad = torch.zeros((c["vocab"], c["width"]), device="cuda").index_add_(0, s["ids"], s["dy"].float()) * c["scale"]
    s["dtable"].copy_(grad + s["dtable"].float() if c["add"] else grad)
    return {"dtable": s["dtable"]}


def _terms(ids):
    return ids.view(len(ids), -1)


def _saved(x, w, ids, temperature, wide=torch.float32):
    """Of every row the log-sum of its scores' exponentials, and its terms' scores; 0 for what is no term, and for a row without one."""
    z = (x.to(wide) @ w.to(wide).T) / temperature
    top = z.amax(1, keepdim=True)
    lse = top + (z - top).exp().sum(1, keepdim=True).log()
    lse = torch.where((ids >= 0).any(1, keepdim=True), lse, 0.0)
    return torch.cat([lse, torch.where(ids >= 0, z.gather(1, ids.clamp(min=0)), 0.0)], 1)


def _weights(s):
    """What a row's terms weigh together: 1, shared as the teacher has it; 0 without a term."""
    ids = _terms(s["ids"])
    if "logits" not in s:
        return (ids >= 0).float()
    a = torch.where(ids >= 0, s["logits"] / s["case"]["temperature"], -math.inf)
    top = a.amax(1, keepdim=True)
    e = torch.where(ids >= 0, (a - top).exp(), 0.0)
    return torch.where(top > -math.inf, e / e.sum(1, keepdim=True), 0.0)


def _loss_plain(s):
    c, ids = s["case"], _terms(s["ids"])
    saved, q = _saved(s["x"], s["w"], ids, c["temperature"]), _weights(s)
    loss = torch.where(q > 0, q * (torch.where(q > 0, q, 1.0).log() + saved[:, :1] - saved[:, 1:]), 0.0).sum(1)
    return {"loss": loss, "saved": saved if c["save"] else None}


def _loss_backward_plain(s):
    c, ids, q = s["case"], _terms(s["ids"]), _weights(s)
    x, w = s["x"].float(), s["w"].float()
    g = torch.where((q > 0).any(1), s["dloss"], 0.0)[:, None] / c["temperature"]
    p = ((x @ w.T) / c["temperature"] - s["saved"][:, :1]).exp() * g
    p.scatter_add_(1, ids.clamp(min=0), -q * g)
    dw = p.T @ x
    s["dw"].copy_(dw + s["dw"].float() if c["add"] else dw)
    return {"dx": (p @ w).to(_F[c["dtype"]]), "dw": s["dw"]}


_PLAIN = {"norm": _norm_plain, "norm_backward": _norm_backward_plain, "embed": _embed_plain, "embed_backward": _embed_backward_plain,
          "loss": _loss_plain, "distill": _loss_plain, "loss_backward": _loss_backward_plain, "distill_backward": _loss_backward_plain}


def run(state):
    if own:
        return _own(state)
    return _PLAIN[state["case"]["op"]](state)


def _own(s):
    from paper_2504_05638_amd import train
    c = s["case"]
    if c["op"] == "norm":
        y, stats = train.norm(s["x"], s["w"], s["b"], kind=c["kind"], eps=_EPS, save=c["save"])
        return {"y": y, "stats": stats}
    if c["op"] == "norm_backward":
        D = c["width"]
        dx = train.norm_backward(s["dy"], s["x"], s["w"], s["stats"], kind=c["kind"], residual=s["residual"], dw=s["bucket"][:D],
                                 db=s["bucket"][D:] if c["bias"] else None, accumulate=c["add"])
        return {"dx": dx, "bucket": s["bucket"]}
    if c["op"] == "embed":
        return {"y": train.embedding(s["ids"], s["table"], scale=c["scale"], residual=s["residual"])}
    if c["op"] == "embed_backward":
        train.embedding_backward(s["dy"], s["ids"], s["dtable"], scale=c["scale"], accumulate=c["add"])
        return {"dtable": s["dtable"]}
    if c["op"] == "loss":
        loss, saved = train.cross_entropy(s["x"], s["w"], s["ids"], save=c["save"])
        return {"loss": loss, "saved": saved}
    if c["op"] == "distill":
        loss, saved = train.distill(s["x"], s["w"], s["ids"], s["logits"], temperature=c["temperature"], save=c["save"])
        return {"loss": loss, "saved": saved}
    if c["op"] == "loss_backward":
        dx = train.cross_entropy_backward(s["dloss"], s["x"], s["w"], s["ids"], s["saved"], dw=s["dw"], accumulate=c["add"])
    else:
        dx = train.distill_backward(s["dloss"], s["x"], s["w"], s["ids"], s["logits"], s["saved"], temperature=c["temperature"], dw=s["dw"], accumulate=c["add"])
    return {"dx": dx, "dw": s["dw"]}


# ------------------------------------------------------------------ what a pass cannot do without


def work(case):
    c, M, D, e = case, case["rows"], case["width"], 4 if case["dtype"] == "f32" else 2
    if c["op"] == "norm":
        return {"bytes": (2 * M * D + D * (1 + c["bias"])) * e + 8 * M * c["save"], "flops": 8.0 * M * D}
    if c["op"] == "norm_backward":
        return {"bytes": (M * D * (3 + c["residual"]) + D + D * (1 + c["bias"]) * (1 + c["add"])) * e + 8 * M, "flops": 15.0 * M * D}
    if c["op"] == "embed":  # (frequent tokens' vectors come from memory once)
        return {"bytes": ((2 + c["residual"]) * M * D) * e + 8 * M, "flops": 2.0 * M * D}
    V = c["vocab"]
    if c["op"] == "embed_backward":
        return {"bytes": (M * D + (2 * min(M, V) if c["add"] else V) * D) * e + 8 * M, "flops": 2.0 * M * D}
    K = c["terms"]
    M = max(1, round(M * (1 - c["ignored"]))) if K == 1 else M  # (rows that have a term)
    small = M * (K * (8 + (4 if c["op"].startswith("distill") else 0)) + 4 * (1 + K) + 4)
    if c["op"] in ("loss", "distill"):
        return {"bytes": (M + V) * D * e + small, "flops": 2.0 * M * V * D}
    return {"bytes": (2 * M + V * (2 + c["add"])) * D * e + small, "flops": 6.0 * M * V * D}


# ------------------------------------------------------------------ the definitions, in 64 bits


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"] == "norm":
        x = s["x"].double()
        mean = torch.sum(x, 1) / c["width"] * (c["kind"] == "layer")
        x = x - mean.unsqueeze(1)
        r = 1 / torch.sqrt(torch.sum(x * x, 1) / c["width"] + _EPS)
        y = x * torch.outer(r, s["w"].double())
        return {"y": y if s["b"] is None else y + s["b"].double(), "stats": torch.stack([mean, r], 1) if c["save"] else None}
    if c["op"] == "norm_backward":
        # through the definition itself: derivatives of sum(y dy), the statistics functions of x
        x, w = s["x"].double().requires_grad_(), s["w"].double().requires_grad_()
        b = torch.zeros(c["width"], device="cuda", dtype=torch.float64, requires_grad=True)
        off = x - x.mean(1, keepdim=True) if c["kind"] == "layer" else x
        y = off / torch.sqrt(torch.mean(off * off, 1, keepdim=True) + _EPS) * w + b
        dx, dw, db = torch.autograd.grad(y, (x, w, b), s["dy"].double())
        grads = torch.cat([dw, db]) if c["bias"] else dw
        return {"dx": dx if s["residual"] is None else dx + s["residual"].double(), "bucket": grads + s["bucket"].double() if c["add"] else grads}
    if c["op"] == "embed":
        y = torch.index_select(s["table"].double(), 0, s["ids"]) * c["scale"]
        return {"y": y if s["residual"] is None else y + s["residual"].double()}
    if c["op"] == "embed_backward":
        # sums of sorted tokens' rows, as differences of running sums
        order = torch.argsort(s["ids"], stable=True)
        run = torch.cumsum(s["dy"][order].double() * c["scale"], 0)
        tokens, counts = torch.unique_consecutive(s["ids"][order], return_counts=True)
        run = run[torch.cumsum(counts, 0) - 1]
        run[1:] -= run[:-1].clone()
        grad = s["dtable"].double() if c["add"] else torch.zeros(c["vocab"], c["width"], device="cuda", dtype=torch.float64)
        grad[tokens] += run
        return {"dtable": grad}
    x, w, T = s["x"].double(), s["w"].double(), c["temperature"]
    ids = s["ids"].reshape(c["rows"], c["terms"])
    there = ids >= 0
    a = s["logits"].double() / T if "logits" in s else torch.zeros_like(ids, dtype=torch.float64)
    log_q = torch.log_softmax(torch.where(there, a, -1e300), 1)
    q = torch.where(there, torch.exp(log_q), 0.0)
    score = torch.matmul(x, w.t()) / T
    log_p = torch.log_softmax(score, 1)
    if c["op"] in ("loss", "distill"):
        at = torch.where(there, ids, 0)
        loss = torch.sum(torch.where(there, q * (log_q - torch.gather(log_p, 1, at)), 0.0), 1)
        lse = torch.logsumexp(score, 1) * there.any(1)
        saved = torch.cat([lse.unsqueeze(1), torch.where(there, torch.gather(score, 1, at), 0.0)], 1)
        return {"loss": loss, "saved": saved if c["save"] else None}
    del score
    # ds = dloss (p - q) / T in the rows that have a term
    ds = torch.exp(log_p).mul_(there.any(1, keepdim=True))
    del log_p
    row = torch.arange(c["rows"], device="cuda").unsqueeze(1).expand_as(ids)
    ds.index_put_((row[there], ids[there]), -q[there], accumulate=True)
    ds.mul_(s["dloss"].double().unsqueeze(1) / T)
    dw = torch.matmul(ds.t(), x)
    return {"dx": torch.matmul(ds, w), "dw": dw + s["dw"].double() if c["add"] else dw}
