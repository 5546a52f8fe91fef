"""The operators around the products of a transformer block and of a decode
step, one pass of each: inputs, plain form, required work and results in 64
bits.

A case is a dict: ``kind`` (the operator), types and sizes.  The kinds:

rope      rotary positions of queries and keys (half or interleaved layout, all
          of the head or its first part), with RMS norms of each head before
          the rotation where the model has them.
rope_grad the gradients of that through a fine-tuning step: queries, keys and
          the norms' weights.
append    the same rotation on the way into a paged key/value cache: queries
          come back rotated, keys and values go to the pages of their
          sequences.
attend    attention of each sequence's new tokens (one in a decode step, many in
          a chunk of a prompt) over its pages.
logits    penalties for repeated tokens, biases and grammar masks on the logits
          that a step ends with.

``own`` false: elementary torch operations in 32 bits, rounded once.  ``own``
true: this package's entry points.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
EPS = 1e-5


def listed():
    return [
        # one token of a 7B model, called eagerly: the launch is what counts
        dict(name="rope_step_7b", kind="rope", tokens=1, heads=32, kv=32, dim=128, rot=128, layout="half", norm=False,
             dtype="fp16", table=4096),
        # the prompts of one prefill step of a 70B-shaped model with head norms
        dict(name="rope_norm_prompt_70b", kind="rope", tokens=4096, heads=64, kv=8, dim=128, rot=128,
             layout="interleaved", norm=True, dtype="bf16", table=32768),
        # block-wise fine-tuning of a 7B block with head norms: one micro-batch of one sequence
        dict(name="rope_grad_norm_2048_7b", kind="rope_grad", tokens=2048, heads=32, kv=32, dim=128, rot=128,
             layout="half", norm=True, dtype="fp16", table=4096),
        # a ragged micro-batch, 13B heads, half of each head rotated
        dict(name="rope_grad_partial_1001_13b", kind="rope_grad", tokens=1001, heads=40, kv=40, dim=128, rot=64,
             layout="interleaved", norm=False, dtype="bf16", table=4096),
        # a decode step of 32 sequences
        dict(name="append_step32_70b", kind="append", seqs=32, new_max=1, ctx_min=40, ctx_max=4000, heads=64, kv=8,
             dim=128, rot=128, layout="half", norm=True, page=16, idle=0, dtype="fp16", table=8192),
        # five prompts of different lengths at once
        dict(name="append_prompts_7b", kind="append", seqs=5, new_max=1900, ctx_min=0, ctx_max=700, heads=32, kv=32,
             dim=128, rot=128, layout="half", norm=False, page=64, idle=0, dtype="bf16", table=4096),
        # one sequence of a 7B model being decoded: the smallest attention call
        dict(name="attend_step_7b", kind="attend", seqs=1, new_max=1, ctx_min=1023, ctx_max=1023, heads=32, kv=32,
             dim=128, page=16, window=0, causal=True, idle=0, lse=False, dtype="fp16"),
        # a decode step of a ragged batch with grouped heads, one slot in eight idle
        dict(name="attend_step64_70b", kind="attend", seqs=64, new_max=1, ctx_min=100, ctx_max=16000, heads=64, kv=8,
             dim=128, page=16, window=0, causal=True, idle=8, lse=False, dtype="bf16"),
        # a chunk of a long prompt over what is in the cache already
        dict(name="attend_chunk2048_70b", kind="attend", seqs=1, new_max=2048, ctx_min=6144, ctx_max=6144, heads=64,
             kv=8, dim=128, page=64, window=0, causal=True, idle=0, lse=False, dtype="bf16"),
        # single tokens, drafts and chunks in one step, a sliding window, shared heads
        dict(name="attend_mixed_window", kind="attend", seqs=14, new_max=300, ctx_min=3, ctx_max=4000, heads=32, kv=8,
             dim=128, page=32, window=1024, causal=True, idle=7, lse=True, dtype="fp16"),
        # greedy decoding of one sequence with penalties
        dict(name="logits_step_1", kind="logits", rows=1, vocab=32000, history=900, prompt=300, biases=16,
             grammar=False, dtype="fp16"),
        # a serving batch with a large vocabulary, constrained by grammars
        dict(name="logits_step_128", kind="logits", rows=128, vocab=128256, history=8000, prompt=5000, biases=300,
             grammar=True, dtype="fp32"),
    ]


def _log(rng, lo, hi):
    """An integer in [lo, hi], spread over the logarithm."""
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(max(lo, 0.5)), math.log(hi + 1))))))


HEADS = [(32, 32), (40, 40), (64, 8), (32, 8), (16, 2), (8, 1), (28, 4), (5, 5), (24, 8)]


def draw(rng):
    kind = rng.choice(["rope", "rope_grad", "append", "attend", "attend", "attend", "logits"])
    if kind == "logits":
        rows = _log(rng, 1, 128)
        history = _log(rng, 1, 8000)
        return dict(kind=kind, rows=rows, vocab=_log(rng, 1000, 128256), history=history,
                    prompt=rng.randint(0, history), biases=rng.choice([0, 1, 7, 64, 300]),
                    grammar=rng.random() < 0.5, dtype=rng.choice(["fp16", "bf16", "fp32"]))
    heads, kv = rng.choice(HEADS)
    dtype = rng.choice(["fp16", "bf16"])
    if kind in ("rope", "rope_grad"):
        dim = rng.choice([64, 80, 96, 128, 128, 128, 256])
        most = 4096 * 72 * 128 if kind == "rope" else 2048 * 64 * 128
        return dict(kind=kind, tokens=_log(rng, 1, max(1, min(8192, most // ((heads + kv) * dim)))), heads=heads, kv=kv,
                    dim=dim, rot=rng.choice([dim, dim, dim // 2, dim // 4, 2 * rng.randint(1, dim // 2)]),
                    layout=rng.choice(["half", "interleaved"]), norm=rng.random() < 0.5,
                    dtype=rng.choice([dtype, dtype, "fp32"]), table=16384)
    if kind == "append":
        dim = rng.choice([64, 80, 96, 128, 128, 256])
        seqs = _log(rng, 1, 128)
        new = 1 if rng.random() < 0.4 else _log(rng, 2, max(2, min(2000, 8000 // seqs)))
        return dict(kind=kind, seqs=seqs, new_max=new, ctx_min=0, ctx_max=_log(rng, 1, 3000), heads=heads, kv=kv,
                    dim=dim, rot=rng.choice([dim, dim, dim // 2]), layout=rng.choice(["half", "interleaved"]),
                    norm=rng.random() < 0.5, page=rng.choice([8, 16, 32, 64, 128]), idle=rng.choice([0, 0, 5]),
                    dtype=dtype, table=8192)
    dim = rng.choice([64, 80, 96, 128, 128, 128, 256])
    form = rng.choice(["step", "draft", "chunk"])
    seqs = _log(rng, 1, 96 if form == "step" else 24 if form == "draft" else 4)
    new = 1 if form == "step" else rng.randint(2, 12) if form == "draft" else _log(rng, 16, 2048)
    # keys in the cache, scores and products stay below those of the largest listed cases
    new = min(new, int((4.5e11 / (4 * heads * dim * seqs)) ** 0.5))
    most = min(300000 * 8 // (seqs * kv) * 128 // dim, (1 << 30) // (seqs * heads * new), 65536,
               int(4.5e11 / (4 * heads * dim * seqs * new)) - new)
    most = max(64, most)
    hi = _log(rng, 1, most)
    return dict(kind="attend", seqs=seqs, new_max=new, ctx_min=_log(rng, 1, hi), ctx_max=hi, heads=heads, kv=kv,
                dim=dim, page=rng.choice([1, 8, 16, 16, 32, 64, 128]), window=rng.choice([0, 0, 0, _log(rng, 1, hi)]),
                causal=rng.random() < 0.85, idle=rng.choice([0, 0, 6]), lse=rng.random() < 0.3, dtype=dtype)


# ---------------------------------------------------------------------------
# inputs

def _spread(lo, hi, n):
    """n integers from lo to hi, spread over the logarithm, in a mixed order."""
    if n == 1:
        return [hi]
    v = [int(round(math.exp(math.log(lo + 1) + (math.log(hi + 1) - math.log(lo + 1)) * i / (n - 1)))) - 1
         for i in range(n)]
    step = next(s for s in range(max(1, int(n * 0.618)), 2 * n + 2) if math.gcd(s, n) == 1)
    return [max(lo, min(hi, v[i * step % n])) for i in range(n)]


def _lengths(case):
    """(new tokens, keys with the new ones) of each sequence, as the step's scheduler made them."""
    n = case["seqs"]
    new = _spread(1, case["new_max"], n)
    ctx = _spread(case["ctx_min"], case["ctx_max"], n)[::-1]
    lens = [a + b for a, b in zip(new, ctx)]
    if case["idle"]:
        for i in range(case["idle"] - 1, n, case["idle"]):  # a slot without a sequence, kept by the fixed step
            new[i], lens[i] = 1, 0
    return new, lens


def _rand(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV, dtype=torch.float32)


def _table(positions, rot):
    """cos and sin of position * frequency, in 64 bits, rounded once."""
    f = 10000.0 ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / rot)
    a = torch.arange(positions, device=DEV, dtype=torch.float64)[:, None] * f
    return torch.stack([a.cos(), a.sin()], -1).float().contiguous()


def _weight(case, gen, dtype):
    """A norm's weight as a trained model has it, or none."""
    return (1 + 0.2 * _rand(gen, case["dim"])).to(dtype) if case["norm"] else None


def _qkv(case, gen, tokens, dtype, parts):
    """Queries, keys (and values) as views of the one activation that the fused projection writes."""
    heads, kv, dim = case["heads"], case["kv"], case["dim"]
    a = _rand(gen, tokens, heads + parts * kv, dim)
    a *= 0.5 + 2 * torch.rand(tokens, heads + parts * kv, 1, generator=gen, device=DEV)
    a = a.to(dtype)
    return [a[:, :heads]] + [a[:, heads + i * kv:heads + (i + 1) * kv] for i in range(parts)]


def _pages(case, gen, lens, capacity):
    """A block table over a cache of somewhat more pages than are in use, in the order in which they were freed."""
    page = case["page"]
    width = max(1, -(-capacity // page))
    count = sum(-(-n // page) for n in lens) + case["seqs"] + 3
    order = torch.randperm(count, generator=gen, device=DEV).to(torch.int32)
    used = torch.tensor([-(-n // page) for n in lens], device=DEV)
    first = torch.cumsum(used, 0) - used
    at = first[:, None] + torch.arange(width, device=DEV)
    held = torch.arange(width, device=DEV) < used[:, None]
    return torch.where(held, order[at.clamp(max=count - 1)], 0).to(torch.int32).contiguous(), count


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed) * 7919 + 17)
    dtype = DTYPES[case["dtype"]]
    s = dict(case=case)
    if case["kind"] in ("rope", "rope_grad"):
        t = case["tokens"]
        s["q"], s["k"] = _qkv(case, gen, t, dtype, 1)
        s["table"] = _table(case["table"], case["rot"])
        # several sequences packed one after another, each from a position of its own
        start = torch.randint(0, case["table"] - min(t, 1024), (max(1, -(-t // 1024)),), generator=gen, device=DEV)
        at = torch.arange(t, device=DEV)
        s["positions"] = (start[at // 1024] + at % 1024).to(torch.int32)
        s["q_weight"], s["k_weight"] = _weight(case, gen, dtype), _weight(case, gen, dtype)
        if case["kind"] == "rope_grad":
            s["dq"] = (_rand(gen, t, case["heads"], case["dim"]) * 0.1).to(dtype)
            s["dk"] = (_rand(gen, t, case["kv"], case["dim"]) * 0.1).to(dtype)
        return s
    if case["kind"] == "logits":
        rows, vocab, history = case["rows"], case["vocab"], case["history"]
        s["logits"] = (_rand(gen, rows, vocab) * 3 - 2).to(dtype)
        # frequent tokens are drawn more often, as in text
        u = torch.rand(rows, history, generator=gen, device=DEV)
        s["tokens"] = ((vocab ** u - 1) * vocab / max(1, vocab - 1)).to(torch.int32).clamp(0, vocab - 1)
        lens = _spread(max(1, history // 8), history, rows)
        s["lens"] = _ints(lens)
        s["prompt"] = _ints([min(n, case["prompt"] * n // history) for n in lens])
        s["repetition"] = 1 + 0.3 * torch.rand(rows, generator=gen, device=DEV)
        s["frequency"] = 0.6 * torch.rand(rows, generator=gen, device=DEV) - 0.1
        s["presence"] = 0.6 * torch.rand(rows, generator=gen, device=DEV) - 0.1
        s["bias_ids"] = s["bias_values"] = s["mask"] = None
        if case["biases"]:
            n = case["biases"]
            ids = torch.randint(0, vocab, (rows, n), generator=gen, device=DEV)
            ids = torch.where(torch.arange(n, device=DEV) < 1 + torch.arange(rows, device=DEV)[:, None] * 37 % n, ids, -1)
            s["bias_ids"] = ids.to(torch.int32)
            s["bias_values"] = _rand(gen, rows, n) * 4
            s["bias_values"][:, 0] = -math.inf  # a token that is banned
        if case["grammar"]:
            words = -(-vocab // 32)
            bits = torch.randint(-(1 << 31), 1 << 31, (3, rows, words), generator=gen, device=DEV)
            few = bits[0] & bits[1] & bits[2]
            kind = torch.arange(rows, device=DEV)[:, None] % 4  # unconstrained, half, an eighth, a few words
            near = torch.arange(words, device=DEV) % 97 == 5
            m = torch.where(kind == 0, -1, torch.where(kind == 1, bits[0], torch.where(kind == 2, few, few * near)))
            if rows > 8:
                m[-2] = 0  # a grammar at its end: nothing may follow
            s["mask"] = m.to(torch.int32)
        return s
    new, lens = _lengths(case)
    total = sum(new)
    s["total"], s["max_new"], s["max_len"] = total, max(new), max(1, max(lens))
    s["block_table"], pages = _pages(case, gen, lens, max(lens))
    s["cu"] = _ints([sum(new[:i]) for i in range(len(new) + 1)])
    s["lens"] = _ints(lens)
    shape = (pages, case["page"], case["kv"], case["dim"])
    if case["kind"] == "append":
        s["q"], s["k"], s["v"] = _qkv(case, gen, total, dtype, 2)
        s["k_cache"], s["v_cache"] = (_rand(gen, *shape).to(dtype) for _ in range(2))
        s["table"] = _table(case["table"], case["rot"])
        s["q_weight"], s["k_weight"] = _weight(case, gen, dtype), _weight(case, gen, dtype)
        return s
    s["q"] = _qkv(case, gen, total, dtype, 0)[0]
    s["k_cache"], s["v_cache"] = (torch.empty(shape, dtype=dtype, device=DEV).normal_(generator=gen) for _ in range(2))
    return s


# ---------------------------------------------------------------------------
# plain forms

def _norm(x, weight):
    """x in 32 bits and the factor of each head's root mean square (None without a norm)."""
    x = x.float()
    return (x, None) if weight is None else (x, torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS))


def _rotate(x, table, positions, layout, sign=1.0):
    """The first 2 * table.shape[1] elements of each head rotated; x in 32 bits."""
    half = table.shape[1]
    cos, sin = (table[positions.long()][:, None, :, i] for i in (0, 1))
    sin = sin * sign
    if layout == "half":
        a, b = x[..., :half], x[..., half:2 * half]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([y, x[..., 2 * half:]], -1)


def _rope_plain(x, weight, table, positions, layout):
    y, r = _norm(x, weight)
    if r is not None:
        y = y * r * weight.float()
    return _rotate(y, table, positions, layout).to(x.dtype)


def _rope_grad_plain(dy, x, weight, table, positions, layout):
    g = _rotate(dy.float(), table, positions, layout, -1.0)
    if weight is None:
        return g.to(dy.dtype), None
    f, r = _norm(x, weight)
    xhat = f * r
    h = g * weight.float()
    dx = r * (h - xhat * (h * xhat).mean(-1, keepdim=True))
    return dx.to(dy.dtype), (g * xhat).sum((0, 1))


def _places(s):
    """Sequence and position of each new token."""
    t = torch.arange(s["total"], device=DEV)
    seq = torch.searchsorted(s["cu"][1:].long(), t, right=True)
    pos = s["lens"][seq].long() - s["cu"][seq + 1].long() + t
    return seq, pos


def _append_plain(s, layout, page):
    seq, pos = _places(s)
    held = pos >= 0  # an idle slot has no place
    at = pos.clamp(min=0)
    q = _rope_plain(s["q"], s["q_weight"], s["table"], at, layout)
    k = _rope_plain(s["k"], s["k_weight"], s["table"], at, layout)
    q = torch.where(held[:, None, None], q, 0)
    where = s["block_table"][seq, at // page].long() * page + at % page
    for cache, x in (("k_cache", k), ("v_cache", s["v"])):
        rows = s[cache].view(-1, *s[cache].shape[2:])
        rows[where[held]] = x[held]
    return {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _attend_plain(s, case):
    page, kv, dim = case["page"], case["kv"], case["dim"]
    group = case["heads"] // kv
    n, length, width = case["seqs"], s["max_len"], s["max_new"]
    at = torch.arange(length, device=DEV)
    where = s["block_table"][:, at // page].long() * page + at % page
    k, v = (s[c].view(-1, kv, dim)[where].permute(0, 2, 1, 3).float().contiguous() for c in ("k_cache", "v_cache"))
    new = (s["cu"][1:] - s["cu"][:-1]).long()
    i = torch.arange(width, device=DEV)
    token = (s["cu"][:-1, None].long() + i).clamp(max=s["total"] - 1)
    q = s["q"][token].float().view(n, width, kv, group, dim).permute(0, 2, 3, 1, 4).reshape(n, kv, group * width, dim)
    score = torch.matmul(q, k.transpose(-1, -2)).mul_(dim ** -0.5).view(n, kv, group, width, length)
    lens = s["lens"].long()[:, None, None]
    pos = lens - new[:, None, None] + i[:, None]
    seen = at < lens
    if case["causal"]:
        seen = seen & (at <= pos)
    if case["window"]:
        seen = seen & (at > pos - case["window"])
    score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(torch.where(top == -math.inf, 0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(n, kv, group * width, length), v).view(n, kv, group, width, dim)
    out = out / torch.where(total == 0, 1, total)
    seq, pos = _places(s)
    row = torch.arange(s["total"], device=DEV) - s["cu"][seq].long()
    out = out.permute(0, 3, 1, 2, 4)[seq, row].flatten(1, 2).to(s["q"].dtype)
    if not case["lse"]:
        return out
    lse = (top + total.log()).squeeze(-1).permute(0, 3, 1, 2)[seq, row].flatten(1, 2)
    return [out, lse]


def _logits_plain(s):
    x = s["logits"].float()
    rows, vocab = x.shape
    at = torch.arange(s["tokens"].shape[1], device=DEV)
    ids = s["tokens"].long()
    held = at < s["lens"][:, None]
    written = held & (at >= s["prompt"][:, None])
    seen = torch.zeros(rows, vocab, device=DEV).scatter_add_(1, ids, held.float()) > 0
    count = torch.zeros(rows, vocab, device=DEV).scatter_add_(1, ids, written.float())
    r = s["repetition"][:, None]
    x = torch.where(seen, torch.where(x > 0, x / r, x * r), x)
    x = x - s["frequency"][:, None] * count - s["presence"][:, None] * (count > 0)
    if s["bias_ids"] is not None:
        ids = s["bias_ids"].long()
        x = x + torch.zeros(rows, vocab, device=DEV).scatter_add_(
            1, ids.clamp(min=0), torch.where(ids >= 0, s["bias_values"], 0))
    if s["mask"] is not None:
        at = torch.arange(vocab, device=DEV)
        x = torch.where((s["mask"][:, at // 32] >> (at % 32) & 1).bool(), x, -math.inf)
    return x.to(s["logits"].dtype)


def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        return _run_own(s, case, kind)
    if kind == "logits":
        return _logits_plain(s)
    if kind == "append":
        return _append_plain(s, case["layout"], case["page"])
    if kind == "attend":
        return _attend_plain(s, case)
    table, positions, layout = s["table"], s["positions"], case["layout"]
    if kind == "rope":
        return [_rope_plain(s["q"], s["q_weight"], table, positions, layout),
                _rope_plain(s["k"], s["k_weight"], table, positions, layout)]
    gq, gqw = _rope_grad_plain(s["dq"], s["q"], s["q_weight"], table, positions, layout)
    gk, gkw = _rope_grad_plain(s["dk"], s["k"], s["k_weight"], table, positions, layout)
    return [gq, gk, gqw, gkw]


def _run_own(s, case, kind):
    import paper_2401_06118_amd as aqlm

    if kind == "logits":
        return aqlm.process_logits(s["logits"], tokens=s["tokens"], token_lens=s["lens"], prompt_lens=s["prompt"],
                                   repetition=s["repetition"], frequency=s["frequency"], presence=s["presence"],
                                   bias_ids=s["bias_ids"], bias_values=s["bias_values"], mask=s["mask"])
    if kind == "attend":
        return aqlm.paged_attention(s["q"], s["k_cache"], s["v_cache"], s["block_table"], s["lens"], s["cu"],
                                    causal=case["causal"], window=case["window"], max_new=s["max_new"],
                                    return_lse=case["lse"])
    norm = dict(q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS, interleaved=case["layout"] == "interleaved")
    if kind == "append":
        q = aqlm.paged_append(s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["block_table"], s["lens"], s["cu"],
                              table=s["table"], **norm)
        return {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    if kind == "rope":
        return aqlm.rope(s["q"], s["k"], s["table"], s["positions"], **norm)
    return aqlm.rope_backward(s["dq"], s["dk"], s["table"], s["positions"], q=s["q"], k=s["k"], **norm)


# ---------------------------------------------------------------------------
# what a pass cannot do without

def work(case):
    kind = case["kind"]
    size = {"fp16": 2, "bf16": 2, "fp32": 4}[case["dtype"]]
    if kind == "logits":
        rows, vocab = case["rows"], case["vocab"]
        held = sum(_spread(max(1, case["history"] // 8), case["history"], rows))
        b = 2 * rows * vocab * size + 4 * held + 20 * rows + 8 * rows * case["biases"]
        if case["grammar"]:
            b += rows * -(-vocab // 32) * 4
        return {"bytes": b, "flops": rows * vocab + 8 * held}
    heads, kv, dim = case["heads"], case["kv"], case["dim"]
    if kind in ("rope", "rope_grad"):
        n = case["tokens"] * (heads + kv) * dim
        b = 2 * n * size + case["tokens"] * (4 * case["rot"] + 4)
        if case["norm"]:
            b += 2 * dim * size + (n * size + 8 * dim if kind == "rope_grad" else 0)
        return {"bytes": b, "flops": n * (3 + (0 if not case["norm"] else 4 if kind == "rope" else 10))}
    new, lens = _lengths(case)
    if kind == "append":
        t = sum(n for n, m in zip(new, lens) if m)
        b = t * (2 * (heads + 2 * kv) * dim * size + 4 * case["rot"] + 4) + 12 * case["seqs"]
        return {"bytes": b, "flops": t * (heads + kv) * dim * (7 if case["norm"] else 3)}
    keys = pairs = 0
    for n, m in zip(new, lens):
        if not m:
            continue
        low = m
        for i in range(n):
            pos = m - n + i
            last = pos + 1 if case["causal"] else m
            first = max(0, pos - case["window"] + 1) if case["window"] else 0
            pairs += max(0, last - first)
            low = min(low, first)
        keys += m - low
    b = 2 * keys * kv * dim * size + 2 * sum(new) * heads * dim * size + 4 * -(-keys // case["page"]) + 8 * case["seqs"]
    if case["lse"]:
        b += 4 * sum(new) * heads
    return {"bytes": b, "flops": 4 * pairs * heads * dim}


# ---------------------------------------------------------------------------
# the definitions in 64 bits

def _angles(s, positions):
    c = s["table"].double()[positions.long()]
    return c[..., 0], c[..., 1]


def _rope_exact(x, weight, c, sn, layout):
    """Head by head as complex numbers: normalise, then multiply by cos + i sin."""
    x = x.double() if x.dtype != torch.float64 else x
    half = c.shape[-1]
    if weight is not None:
        x = x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt() * weight.double()
    turn = torch.complex(c, sn)[:, None]
    head, rest = x[..., :2 * half], x[..., 2 * half:]
    pairs = head.unflatten(-1, (2, half)).transpose(-1, -2) if layout == "half" else head.unflatten(-1, (half, 2))
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    z = z.transpose(-1, -2).flatten(-2) if layout == "half" else z.flatten(-2)
    return torch.cat([z, rest], -1)


def _rope_grad_exact(dy, x, weight, c, sn, layout):
    x = x.detach().double().requires_grad_(True)
    w = None if weight is None else weight.detach().double().requires_grad_(True)
    y = _rope_exact(x, w, c, sn, layout)
    g = torch.autograd.grad(y, [x] if w is None else [x, w], dy.double())
    return g[0], (g[1] if w is not None else None)


def _attend_exact(s, case):
    new, lens = _lengths(case)
    page, group, dim = case["page"], case["heads"] // case["kv"], case["dim"]
    out = torch.zeros(s["total"], case["heads"], dim, dtype=torch.float64, device=DEV)
    lse = torch.full((s["total"], case["heads"]), -math.inf, dtype=torch.float64, device=DEV)
    first = 0
    for b, (n, m) in enumerate(zip(new, lens)):
        pos = torch.arange(m - n, m, device=DEV)[:, None]
        j = torch.arange(m, device=DEV)[None]
        ok = torch.ones(n, m, dtype=torch.bool, device=DEV)
        if case["causal"]:
            ok &= j <= pos
        if case["window"]:
            ok &= pos - j < case["window"]
        ids = s["block_table"][b, :-(-m // page)].long()
        for h in range(case["kv"] if m else 0):
            k, v = (s[c][ids, :, h].reshape(-1, dim)[:m].double() for c in ("k_cache", "v_cache"))
            for g in range(group):
                e = h * group + g
                score = (s["q"][first:first + n, e].double() @ k.t()) / math.sqrt(dim)
                score = torch.where(ok, score, -math.inf)
                some = ok.any(-1)
                out[first:first + n, e] = torch.where(some[:, None], torch.softmax(score, -1).nan_to_num(0.0) @ v, 0)
                lse[first:first + n, e] = torch.logsumexp(score, -1)
        first += n
    return [out, lse] if case["lse"] else out


def _logits_exact(s):
    x = s["logits"].double()
    for b in range(x.shape[0]):
        n, p = int(s["lens"][b]), int(s["prompt"][b])
        ids = s["tokens"][b, :n].long()
        known = ids.unique()
        r = s["repetition"][b].double()
        x[b, known] = torch.where(x[b, known] < 0, x[b, known] * r, x[b, known] / r)
        which, times = ids[p:].unique(return_counts=True)
        x[b, which] -= times.double() * s["frequency"][b].double() + s["presence"][b].double()
        if s["bias_ids"] is not None:
            keep = s["bias_ids"][b] >= 0
            x[b].index_add_(0, s["bias_ids"][b][keep].long(), s["bias_values"][b][keep].double())
        if s["mask"] is not None:
            word = s["mask"][b].long() & 0xFFFFFFFF
            bit = (word[:, None] >> torch.arange(32, device=DEV)) & 1
            x[b, bit.flatten()[:x.shape[1]] == 0] = -math.inf
    return x


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "logits":
        return _logits_exact(s)
    if kind == "attend":
        return _attend_exact(s, case)
    layout = case["layout"]
    if kind in ("rope", "rope_grad"):
        c, sn = _angles(s, s["positions"])
        if kind == "rope":
            return [_rope_exact(s[x], s[x + "_weight"], c, sn, layout) for x in "qk"]
        (gq, gqw), (gk, gkw) = (_rope_grad_exact(s["d" + x], s[x], s[x + "_weight"], c, sn, layout) for x in "qk")
        return [gq, gk, gqw, gkw]
    new, lens = _lengths(case)
    q = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
    first = 0
    for b, (n, m) in enumerate(zip(new, lens)):
        if m:
            pos = torch.arange(m - n, m, device=DEV)
            c, sn = _angles(s, pos)
            at = slice(first, first + n)
            q[at] = _rope_exact(s["q"][at], s["q_weight"], c, sn, layout)
            ids = s["block_table"][b].long()[pos // case["page"]]
            k_cache[ids, pos % case["page"]] = _rope_exact(s["k"][at], s["k_weight"], c, sn, layout)
            v_cache[ids, pos % case["page"]] = s["v"][at].double()
        first += n
    return {"q": q, "k_cache": k_cache, "v_cache": v_cache}
