"""The operators at the ends of a model and between its blocks, one pass of each:
inputs, plain form, required work and results in 64 bits.

A case is a dict: ``kind`` (the operator), types and sizes.  The kinds:

embed       rows of the embedding table for a step's tokens, scaled.
embed_grad  the table's gradient: the rows of a token's places summed.
norm        layer or RMS norm of the residual stream, with the sum before it.
norm_grad   its gradients: the stream's, the weight's and the bias's.
distill     the loss of a student's logits against a teacher's largest ones, and its
            gradient, in one call.
sample      a token of each row of logits: temperature, top-k, top-p, min-p, from
            uniform numbers that are inputs.

``own`` false: elementary torch operations in 32 bits (64 where a border or a
difference asks for them), rounded once.  ``own`` true: this package's entry points.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
BYTES = {"fp16": 2, "bf16": 2, "fp32": 4}
EPS = 1e-5


def listed():
    return [
        # one token of a 7B model, called eagerly: the launch is what counts
        dict(name="embed_step_7b", kind="embed", tokens=1, vocab=32000, dim=4096, scale=1.0, pad=0.0, dtype="fp16"),
        # the prompts of one prefill step, 70B-shaped, a scaled embedding
        dict(name="embed_prompt_70b", kind="embed", tokens=8192, vocab=128256, dim=8192, scale=90.5, pad=0.0,
             dtype="bf16"),
        # a micro-batch of two sequences of 2048: the dense gradient of a 7B model's table
        dict(name="embed_grad_4096_7b", kind="embed_grad", tokens=4096, vocab=32000, dim=4096, scale=1.0, pad=0.0,
             dtype="fp16"),
        # ragged sequences, a third of the batch padding, 13B width, gradients kept in 32 bits
        dict(name="embed_grad_ragged_13b", kind="embed_grad", tokens=1999, vocab=32000, dim=5120, scale=71.5, pad=0.3,
             dtype="fp32"),
        # the residual sum and norm of one token of a 7B model
        dict(name="norm_step_7b", kind="norm", tokens=1, dim=4096, rms=True, weight=True, bias=False, residual=True,
             dtype="fp16"),
        # the same for a prefill step of a 70B-shaped model
        dict(name="norm_prompt_70b", kind="norm", tokens=4096, dim=8192, rms=True, weight=True, bias=False,
             residual=True, dtype="bf16"),
        # block-wise fine-tuning of a 7B model: one sequence
        dict(name="norm_grad_2048_7b", kind="norm_grad", tokens=2048, dim=4096, rms=True, weight=True, bias=False,
             residual=True, dtype="fp16"),
        # layer norm with a bias, a ragged micro-batch, 13B width, 32 bits
        dict(name="norm_grad_layer_13b", kind="norm_grad", tokens=1001, dim=5120, rms=False, weight=True, bias=True,
             residual=False, dtype="fp32"),
        # end-to-end fine-tuning of a quantised 7B model against the original's 64 largest logits
        dict(name="distill_2048_7b", kind="distill", tokens=2048, vocab=32000, listed=64, rest=False, tau=1.0,
             short=False, masked=0.1, dtype="fp16", teacher="fp16"),
        # a large vocabulary, an odd count of tokens, the mass outside the list as one outcome
        dict(name="distill_rest_333", kind="distill", tokens=333, vocab=128256, listed=200, rest=True, tau=2.0,
             short=True, masked=0.25, dtype="bf16", teacher="fp32"),
        # one sequence being decoded
        dict(name="sample_step_1", kind="sample", rows=1, vocab=32000, top_k=True, top_p=True, min_p=False,
             greedy=0, banned=0.0, logprob=False, dtype="fp16"),
        # a serving batch with a large vocabulary, the requests' own settings, constrained rows
        dict(name="sample_step_128", kind="sample", rows=128, vocab=128256, top_k=True, top_p=True, min_p=True,
             greedy=9, banned=0.3, logprob=True, dtype="fp32"),
    ]


def _log(rng, lo, hi):
    """An integer in [lo, hi], spread over the logarithm."""
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def _dim(rng):
    """A width: a usual one, or an odd one."""
    return rng.choice([64, 128, 256, 512, 768, 1024, 2048, 2560, 4096, 4096, 5120, 6656, 8192, _log(rng, 33, 8192)])


def draw(rng):
    kind = rng.choice(["embed", "embed_grad", "norm", "norm_grad", "distill", "sample"])
    dtype = rng.choice(["fp16", "bf16", "fp32"])
    size = BYTES[dtype]
    vocab = rng.choice([32000, 32000, 128256, _log(rng, 1000, 128256)])
    if kind in ("embed", "embed_grad"):
        dim = _dim(rng)
        scale, pad = rng.choice([1.0, 1.0, dim ** 0.5, 0.37]), rng.choice([0.0, 0.0, 0.2])
        if kind == "embed_grad":  # (the gradient has a row for every token of the vocabulary)
            vocab = max(100, min(vocab, 250_000_000 // (dim * size)))
        tokens = _log(rng, 1, max(1, min(8192, (250_000_000 if kind == "embed" else 80_000_000) // (2 * dim * size))))
        return dict(kind=kind, tokens=tokens, vocab=vocab, dim=dim, scale=scale, pad=pad, dtype=dtype)
    if kind in ("norm", "norm_grad"):
        dim = _dim(rng)
        rms = rng.random() < 0.6
        return dict(kind=kind, tokens=_log(rng, 1, min(8192, 250_000_000 // (4 * dim * size))), dim=dim, rms=rms,
                    weight=rng.random() < 0.85, bias=rng.random() < (0.1 if rms else 0.8),
                    residual=rng.random() < 0.5, dtype=dtype)
    if kind == "distill":
        return dict(kind=kind, tokens=_log(rng, 1, min(2048, 250_000_000 // (2 * vocab * size))), vocab=vocab,
                    listed=rng.choice([1, 8, 20, 50, 64, 100, 128, 256, _log(rng, 2, 999)]), rest=rng.random() < 0.5,
                    tau=rng.choice([1.0, 1.0, 2.0, 0.7, 4.0]), short=rng.random() < 0.4,
                    masked=rng.choice([0.0, 0.2]), dtype=dtype, teacher=rng.choice([dtype, "fp16", "bf16", "fp32"]))
    return dict(kind=kind, rows=_log(rng, 1, 128), vocab=vocab, top_k=rng.random() < 0.5, top_p=rng.random() < 0.6,
                min_p=rng.random() < 0.4, greedy=rng.choice([0, 0, 5]), banned=rng.choice([0.0, 0.0, 0.4]),
                logprob=rng.random() < 0.4, dtype=dtype)


# ---------------------------------------------------------------------------
# inputs

def _rand(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV, dtype=torch.float32)


def _uniform(gen, *shape):
    return torch.rand(*shape, generator=gen, device=DEV, dtype=torch.float32)


def _tokens(gen, n, vocab, pad):
    """Ids as text has them, the frequent ones with small numbers; a part of them padding (-1)."""
    ids = (float(vocab + 1) ** _uniform(gen, n).double() - 1).long().clamp(0, vocab - 1)
    out = _uniform(gen, n) < pad
    out[0] = False
    return torch.where(out, -1, ids).to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed) * 6271 + 29)
    dtype, kind = DTYPES[case["dtype"]], case["kind"]
    s = dict(case=case)
    if kind in ("embed", "embed_grad"):
        s["tokens"] = _tokens(gen, case["tokens"], case["vocab"], case["pad"])
        if kind == "embed":
            s["table"] = torch.empty(case["vocab"], case["dim"], dtype=dtype, device=DEV).normal_(generator=gen)
        else:
            s["dout"] = (_rand(gen, case["tokens"], case["dim"]) * 0.1).to(dtype)
        return s
    if kind in ("norm", "norm_grad"):
        t, dim = case["tokens"], case["dim"]
        # a residual stream: a few channels are much larger than the others, rows differ in size
        channel = torch.where(_uniform(gen, dim) < 0.01, 30.0, 1.0) * (0.5 + _uniform(gen, dim))
        stream = _rand(gen, t, dim) * channel * (0.3 + 3 * _uniform(gen, t, 1)) + 0.5 * _rand(gen, dim)
        s["x"] = stream.to(dtype)
        s["weight"] = (1 + 0.3 * _rand(gen, dim)).to(dtype) if case["weight"] else None
        s["bias"] = (0.3 * _rand(gen, dim)).to(dtype) if case["bias"] else None
        if kind == "norm":
            s["residual"] = _rand(gen, t, dim).to(dtype) if case["residual"] else None
        else:
            s["dy"] = (_rand(gen, t, dim) * 0.1).to(dtype)
            s["dsum"] = (_rand(gen, t, dim) * 0.1).to(dtype) if case["residual"] else None
        return s
    if kind == "distill":
        t, vocab, n = case["tokens"], case["vocab"], case["listed"]
        teacher = _rand(gen, t, vocab) * 2.5 + 3 * _rand(gen, t, 1)
        s["logits"] = (teacher + _rand(gen, t, vocab)).to(dtype)  # a student near its teacher
        top, ids = torch.topk(teacher, n, dim=1)
        s["teacher"] = top.to(DTYPES[case["teacher"]])
        if case["short"]:  # the lists end where the teacher's mass is nearly whole: entries of -1 behind
            keep = 1 + (_uniform(gen, t, 1) * n).long()
            if t > 3:
                keep[1] = 0  # a token of which nothing was kept
            ids = torch.where(torch.arange(n, device=DEV) < keep, ids, -1)
        s["ids"] = ids.to(torch.int32)
        s["lse"] = torch.logsumexp(teacher.double() / case["tau"], 1).float() if case["rest"] else None
        w = 0.5 + _uniform(gen, t)  # the loss scale's part, prompts and padding without
        s["weights"] = torch.where(_uniform(gen, t) < case["masked"], 0.0, w)
        s["weights"][0] = w[0]
        return s
    rows, vocab = case["rows"], case["vocab"]
    x = _rand(gen, rows, vocab) * (1.5 + 2 * _uniform(gen, rows, 1))
    # a model's likely next tokens stand out
    x.scatter_add_(1, torch.randint(0, vocab, (rows, 40), generator=gen, device=DEV), 6 * _uniform(gen, rows, 40))
    if case["banned"]:  # a grammar's masked tokens
        x = torch.where(_uniform(gen, rows, vocab) < case["banned"], -math.inf, x)
        x[:, vocab // 2] = 0.5
    s["logits"] = x.to(dtype)
    s["uniform"] = _uniform(gen, rows)
    temperature = 0.4 + _uniform(gen, rows)
    if case["greedy"]:
        temperature[case["greedy"] - 1::case["greedy"]] = 0
    s["temperature"] = temperature
    s["top_k"] = s["top_p"] = s["min_p"] = None
    if case["top_k"]:
        choice = torch.tensor([50, 40, 20, 0, 100, 1, 500, 50], device=DEV)  # (0: no limit)
        s["top_k"] = choice[(torch.arange(rows, device=DEV) * 5) % 8].to(torch.int32)
    if case["top_p"]:
        s["top_p"] = 0.5 + 0.55 * _uniform(gen, rows)  # (1 and above: all)
    if case["min_p"]:
        s["min_p"] = (0.2 * _uniform(gen, rows) - 0.05).clamp(min=0)
    return s


# ---------------------------------------------------------------------------
# plain forms

def _embed_plain(s, case):
    ids = s["tokens"].long()
    y = s["table"][ids.clamp(min=0)].float() * case["scale"]
    return torch.where(ids[:, None] >= 0, y, 0).to(s["table"].dtype)


def _embed_grad_plain(s, case):
    ids = s["tokens"].long()
    held = ids >= 0
    g = torch.zeros(case["vocab"], case["dim"], device=DEV)
    g.index_add_(0, ids[held], s["dout"][held].float())
    return (g * case["scale"]).to(s["dout"].dtype)


def _normed(x, rms):
    """Rows in 32 bits: centred (layer norm), and the factor that makes them of size one."""
    x = x.float()
    if not rms:
        x = x - x.mean(-1, keepdim=True)
    return x, torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)


def _norm_plain(s, case):
    h = s["x"]
    if s["residual"] is not None:
        h = (h.float() + s["residual"].float()).to(h.dtype)
    c, r = _normed(h, case["rms"])
    y = c * r
    if s["weight"] is not None:
        y = y * s["weight"].float()
    if s["bias"] is not None:
        y = y + s["bias"].float()
    y = y.to(h.dtype)
    return y if s["residual"] is None else [y, h]


def _norm_grad_plain(s, case):
    c, r = _normed(s["x"], case["rms"])
    xhat, dy = c * r, s["dy"].float()
    g = dy if s["weight"] is None else dy * s["weight"].float()
    d = g - xhat * (g * xhat).mean(-1, keepdim=True)
    if not case["rms"]:
        d = d - g.mean(-1, keepdim=True)
    d = d * r
    if s["dsum"] is not None:
        d = d + s["dsum"].float()
    return [d.to(s["dy"].dtype), None if s["weight"] is None else (dy * xhat).sum(0),
            dy.sum(0) if case["bias"] else None]


def _distill_plain(s, case):
    tau, ids = case["tau"], s["ids"].long()
    held, at = ids >= 0, ids.clamp(min=0)
    # statistics in 64 bits: the loss and the mass outside the list are differences
    z = s["logits"].double() / tau
    z = z - z.amax(1, keepdim=True)
    e = z.exp()
    total = e.sum(1, keepdim=True)
    q = (e / total).float()
    t = torch.where(held, s["teacher"].double() / tau, -math.inf)
    if case["rest"]:
        p = (t - s["lse"].double()[:, None]).exp()
    else:
        top = t.amax(1, keepdim=True)
        p = (t - torch.where(top == -math.inf, 0, top)).exp()
        mass = p.sum(1, keepdim=True)
        p = p / torch.where(mass == 0, 1, mass)
    log_q = z.gather(1, at) - total.log()
    loss = torch.where(p > 0, p * (torch.where(p > 0, p, 1).log() - log_q), 0).sum(1)
    pj = torch.zeros_like(q).scatter_add_(1, at, torch.where(held, p, 0).float())
    if case["rest"]:
        out = torch.zeros_like(q).scatter_add_(1, at, held.float()) == 0
        pr = (1 - p.sum(1, keepdim=True)).clamp(min=0)
        qr = torch.where(out, e, 0).sum(1, keepdim=True) / total
        loss = loss + torch.where(pr > 0, pr * (torch.where(pr > 0, pr, 1) / qr).log(), 0).squeeze(1)
        mass = p.sum(1, keepdim=True) + pr  # (1, or more where the list's roundings add up to more)
        grad = torch.where(out, q * (mass - pr / qr).float(), q * mass.float() - pj)
    else:
        grad = q * held.any(1, keepdim=True) - pj
    w = s["weights"][:, None]
    grad = torch.where(w != 0, grad * (w / tau), 0)
    return [torch.where(s["weights"] != 0, loss.float(), 0), grad.to(s["logits"].dtype)]


def _sample_plain(s, case):
    x = s["logits"].double()
    rows, vocab = x.shape
    top, first = x.max(1, keepdim=True)
    t = s["temperature"].double()[:, None]
    greedy = t <= 0
    t = torch.where(greedy, 1, t)
    w = torch.where(x == -math.inf, 0, ((x - top) / t).exp())
    rank = torch.arange(vocab, device=DEV)
    xs, order = torch.sort(x, dim=1, descending=True, stable=True)
    ws = w.gather(1, order)
    keep = torch.ones_like(ws, dtype=torch.bool)
    if s["top_k"] is not None:
        k = s["top_k"].long()[:, None]
        keep = (k <= 0) | (rank < k)
    if s["top_p"] is not None:
        p = s["top_p"].double()[:, None]
        held = torch.where(keep, ws, 0)
        upto = held.cumsum(1)
        keep = keep & ((p >= 1) | (upto - held < p * upto[:, -1:]))
    if s["min_p"] is not None:
        m = s["min_p"].double()[:, None]
        keep = keep & ((m <= 0) | (xs - top >= t * m.log()))
    keep[:, 0] = True
    held = torch.zeros_like(w).scatter_(1, order, torch.where(keep, ws, 0))
    upto = held.cumsum(1)
    total = upto[:, -1:]
    # the first token whose mass and those before it exceed the number's share
    token = (upto <= s["uniform"].double()[:, None] * total).sum(1, keepdim=True)
    lowest = (x == top).to(torch.int8).argmax(1, keepdim=True)  # (of equal ones)
    token = torch.where(greedy, lowest, token.clamp(max=vocab - 1))
    out = token.squeeze(1).to(torch.int32)
    if not case["logprob"]:
        return out
    lp = (x.gather(1, token) - top) / t - total.log()
    return [out, torch.where(greedy, 0, lp).squeeze(1).float()]


def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        return _run_own(s, case, kind)
    return {"embed": _embed_plain, "embed_grad": _embed_grad_plain, "norm": _norm_plain, "norm_grad": _norm_grad_plain,
            "distill": _distill_plain, "sample": _sample_plain}[kind](s, case)


def _run_own(s, case, kind):
    import paper_2401_06118_amd as aqlm

    if kind == "embed":
        return aqlm.embed(s["table"], s["tokens"], scale=case["scale"])
    if kind == "embed_grad":
        return aqlm.embed_backward(s["dout"], s["tokens"], case["vocab"], scale=case["scale"])
    if kind == "norm":
        return aqlm.layer_norm(s["x"], s["weight"], s["bias"], residual=s["residual"], eps=EPS, rms=case["rms"])
    if kind == "norm_grad":
        return aqlm.layer_norm_backward(s["dy"], s["x"], s["weight"], dsum=s["dsum"], eps=EPS, rms=case["rms"],
                                        bias=case["bias"])
    if kind == "distill":
        return aqlm.distill_loss(s["logits"], s["teacher"], s["ids"], teacher_lse=s["lse"], temperature=case["tau"],
                                 weights=s["weights"])
    return aqlm.sample(s["logits"], s["uniform"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                       min_p=s["min_p"], return_logprob=case["logprob"])


# ---------------------------------------------------------------------------
# what a pass cannot do without

def work(case):
    kind, size = case["kind"], BYTES[case["dtype"]]
    if kind in ("embed", "embed_grad"):
        t, vocab, dim = case["tokens"], case["vocab"], case["dim"]
        held = t * (1 - case["pad"])
        if kind == "embed":
            # rows that several tokens share are read once: how many differ, by the ids' distribution
            at = torch.arange(vocab + 1, dtype=torch.float64) + 1
            share = (at[1:] / at[:-1]).log() / math.log(vocab + 1)
            rows = float((1 - (1 - share) ** held).sum())
            return {"bytes": int((rows + t) * dim * size + 4 * t), "flops": int(held * dim)}
        return {"bytes": int((held + vocab) * dim * size + 4 * t), "flops": int(2 * held * dim)}
    if kind in ("norm", "norm_grad"):
        n, dim = case["tokens"] * case["dim"], case["dim"]
        if kind == "norm":
            b = n * size * (4 if case["residual"] else 2) + dim * size * (case["weight"] + case["bias"])
            return {"bytes": b, "flops": n * (5 if case["rms"] else 7)}
        b = n * size * (4 if case["residual"] else 3) + dim * (case["weight"] * (size + 4) + case["bias"] * 4)
        return {"bytes": b, "flops": n * (12 if case["rms"] else 15)}
    if kind == "distill":
        t, vocab, n = case["tokens"], case["vocab"], case["listed"]
        held = t * (1 - case["masked"])  # (logits of tokens without weight need not be read)
        b = (held + t) * vocab * size + held * n * (BYTES[case["teacher"]] + 4) + t * (12 if case["rest"] else 8)
        return {"bytes": int(b), "flops": int(held * vocab * 7)}
    rows, vocab = case["rows"], case["vocab"]
    b = rows * (vocab * size + 12 + 4 * (case["top_k"] + case["top_p"] + case["min_p"] + case["logprob"]))
    return {"bytes": b, "flops": 4 * rows * vocab}


# ---------------------------------------------------------------------------
# the definitions in 64 bits

def _norm_exact(x, w, b, rms):
    mu = 0 if rms else x.sum(-1, keepdim=True) / x.shape[-1]
    var = (x - mu).pow(2).sum(-1, keepdim=True) / x.shape[-1]
    y = (x - mu) / (var + EPS).sqrt()
    y = y if w is None else y * w
    return y if b is None else y + b


def _distill_row(z, t, ids, lse, weight, tau):
    """Loss of one token and its gradient, by automatic differentiation of the divergence."""
    if float(weight) == 0:
        return z.new_zeros(()), torch.zeros_like(z)
    z = z.detach().requires_grad_(True)
    held = ids >= 0
    at, t = ids[held].long(), t[held].double() / tau
    log_q = torch.log_softmax(z / tau, 0)
    log_p = t - (lse if lse is not None else torch.logsumexp(t, 0))
    loss = (log_p.exp() * (log_p - log_q[at])).sum()
    if lse is not None:
        rest = torch.ones_like(z, dtype=torch.bool)
        rest[at] = False
        pr = 1 - log_p.exp().sum()
        if float(pr) > 0:
            loss = loss + pr * (pr.log() - torch.logsumexp(log_q[rest], 0))
    (g,) = torch.autograd.grad(loss, z) if held.any() or lse is not None else (torch.zeros_like(z),)
    return loss.detach(), g * weight.double()


def _sample_row(x, u, t, k, p, m):
    """Token and its log-probability from the sorted list of one row's tokens."""
    if t <= 0:
        return int((x == x.max()).nonzero()[0, 0]), 0.0
    vals, ids = torch.sort(x, descending=True, stable=True)
    n = int((vals > -math.inf).sum())
    if k is not None and k > 0:
        n = min(n, k)
    w = torch.exp((vals[:n] - vals[0]) / t)
    if p is not None and p < 1:
        upto = torch.cumsum(w, 0)
        n = 1 + int((upto[:-1] < p * upto[-1]).sum())
    if m is not None and m > 0:
        n = min(n, max(1, int((vals[:n] - vals[0] >= t * math.log(m)).sum())))
    w, ids = w[:n], ids[:n]
    ids, by = torch.sort(ids)
    upto = torch.cumsum(w[by], 0)
    i = min(n - 1, int((upto <= u * upto[-1]).sum()))
    return int(ids[i]), float(torch.log(w[by][i] / upto[-1]))


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "embed":
        ids = s["tokens"].long()
        y = torch.zeros(case["tokens"], case["dim"], dtype=torch.float64, device=DEV)
        y[ids >= 0] = s["table"][ids[ids >= 0]].double() * case["scale"]
        return y
    if kind == "embed_grad":
        ids = s["tokens"].long()
        g = torch.zeros(case["vocab"], case["dim"], dtype=torch.float64, device=DEV)
        for i in ids.unique().tolist():
            if i >= 0:
                g[i] = s["dout"][ids == i].double().sum(0) * case["scale"]
        return g
    if kind == "norm":
        w, b = (None if s[n] is None else s[n].double() for n in ("weight", "bias"))
        if s["residual"] is None:
            return _norm_exact(s["x"].double(), w, b, case["rms"])
        h = s["x"].double() + s["residual"].double()
        # (the sum that the stream goes on with is what is normalised: rounded to its type)
        return [_norm_exact(h.to(s["x"].dtype).double(), w, b, case["rms"]), h]
    if kind == "norm_grad":
        x = s["x"].double().requires_grad_(True)
        w = None if s["weight"] is None else s["weight"].double().requires_grad_(True)
        b = None if s["bias"] is None else s["bias"].double().requires_grad_(True)
        leaves = [v for v in (x, w, b) if v is not None]
        g = dict(zip(map(id, leaves),
                     torch.autograd.grad(_norm_exact(x, w, b, case["rms"]), leaves, s["dy"].double())))
        dx = g[id(x)] if s["dsum"] is None else g[id(x)] + s["dsum"].double()
        return [dx, None if w is None else g[id(w)], None if b is None else g[id(b)]]
    if kind == "distill":
        loss = torch.zeros(case["tokens"], dtype=torch.float64, device=DEV)
        grad = torch.zeros(case["tokens"], case["vocab"], dtype=torch.float64, device=DEV)
        for i in range(case["tokens"]):
            lse = None if s["lse"] is None else s["lse"][i].double()
            loss[i], grad[i] = _distill_row(s["logits"][i].double(), s["teacher"][i], s["ids"][i], lse,
                                            s["weights"][i], case["tau"])
        return [loss, grad]
    got = []
    for i in range(case["rows"]):
        k, p, m = (None if s[n] is None else s[n][i].item() for n in ("top_k", "top_p", "min_p"))
        got.append(_sample_row(s["logits"][i].double(), s["uniform"][i].item(), s["temperature"][i].item(), k, p, m))
    out = torch.tensor([t for t, _ in got], dtype=torch.int32, device=DEV)
    return [out, torch.tensor([v for _, v in got], dtype=torch.float64, device=DEV)] if case["logprob"] else out
