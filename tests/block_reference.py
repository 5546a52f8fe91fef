"""The operators of ``block.py`` from their definitions in 64 bits, on the CPU, with
what the error bounds of the tests need beside the results."""
import math

import torch

UNIT = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
TINY = {torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -126, torch.float32: 2.0 ** -126}


def table64(positions, rot, base=10000.0):
    f = base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    a = torch.arange(positions, dtype=torch.float64)[:, None] * f
    return torch.stack([a.cos(), a.sin()], -1)


def pairs_of(rot, interleaved):
    i = torch.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def rope64(x, weight, table, positions, interleaved, eps):
    """(result, magnitude of what was added up) for x [tokens, heads, dim] in 64 bits."""
    y = x
    if weight is not None:
        y = x / (x.pow(2).mean(-1, keepdim=True) + eps).sqrt() * weight
    rot = 2 * table.shape[1]
    a, b = pairs_of(rot, interleaved)
    c, s = (table[positions][:, None, :, k] for k in (0, 1))
    out, size = y.clone(), y.abs()
    out[..., a] = y[..., a] * c - y[..., b] * s
    out[..., b] = y[..., b] * c + y[..., a] * s
    size[..., a] = size[..., b] = y[..., a].abs() + y[..., b].abs()
    return out, size


def unrotate64(g, table, positions, interleaved):
    a, b = pairs_of(2 * table.shape[1], interleaved)
    c, s = (table[positions][:, None, :, k] for k in (0, 1))
    out = g.clone()
    out[..., a] = g[..., a] * c + g[..., b] * s
    out[..., b] = g[..., b] * c - g[..., a] * s
    return out


def rope_grad64(dy, x, weight, table, positions, interleaved, eps):
    """(dx, magnitude, dweight, magnitude) by the formulas."""
    g = unrotate64(dy, table, positions, interleaved)
    mag_g = unrotate64(dy.abs(), torch.stack([table[..., 0].abs(), -table[..., 1].abs()], -1), positions,
                       interleaved).abs()
    # (|a c| + |b s| for both elements of a pair, an upper bound of the rotated gradient)
    a, b = pairs_of(2 * table.shape[1], interleaved)
    mag_g[..., a] = dy[..., a].abs() + dy[..., b].abs()
    mag_g[..., b] = mag_g[..., a]
    if weight is None:
        return g, mag_g, None, None
    r = 1 / (x.pow(2).mean(-1, keepdim=True) + eps).sqrt()
    n = x * r
    gw = g * weight
    dx = r * (gw - n * (gw * n).mean(-1, keepdim=True))
    mag = r * (mag_g * weight.abs() + n.abs() * (mag_g * weight.abs() * n.abs()).mean(-1, keepdim=True))
    return dx, mag, (g * n).sum((0, 1)), (mag_g * n.abs()).sum((0, 1))


def gather(cache, row, n):
    """Keys 0 .. n of one sequence [n, kv heads, dim] in 64 bits."""
    page = cache.shape[1]
    j = torch.arange(n)
    return cache[row[j // page].long(), j % page].double()


def visible(n, keys, causal, window):
    pos = torch.arange(keys - n, keys)[:, None]
    j = torch.arange(keys)[None]
    ok = torch.ones(n, keys, dtype=torch.bool)
    if causal:
        ok &= j <= pos
    if window:
        ok &= j > pos - window
    return ok


def attend64(q, k_cache, v_cache, table, lens, cu, scale, causal, window):
    """(out, bound of the rounding of weights and scores, lse) [tokens, heads, ...].
    The bound is in units of the type's rounding unit for the weights; the scores'
    part is added by the caller from ``score`` (largest |q| . |k| of a row)."""
    tokens, heads, dim = q.shape
    kv = k_cache.shape[2]
    group = heads // kv
    out = torch.zeros(tokens, heads, dim, dtype=torch.float64)
    size = torch.zeros_like(out)
    score = torch.zeros(tokens, heads, 1, dtype=torch.float64)
    lse = torch.full((tokens, heads), -math.inf, dtype=torch.float64)
    for b in range(len(lens)):
        n, m = int(cu[b + 1] - cu[b]), int(lens[b])
        if n == 0 or m == 0:
            continue
        ok = visible(n, m, causal, window)
        k, v = gather(k_cache, table[b], m), gather(v_cache, table[b], m)
        rows = slice(int(cu[b]), int(cu[b + 1]))
        for e in range(heads):
            h = e // group
            qe = q[rows, e].double()
            kh, vh = k[:, h], v[:, h]
            s = torch.where(ok, qe @ kh.t() * scale, -math.inf)
            mag = torch.where(ok, qe.abs() @ kh.abs().t() * abs(scale), 0.0)
            some = ok.any(-1)
            p = torch.softmax(s, -1)
            p = torch.where(some[:, None], p, 0.0)
            # keys that a row does not see take no part in it, whatever they hold
            o = torch.stack([(p[i][ok[i]][:, None] * vh[ok[i]]).sum(0) for i in range(n)]) \
                if not torch.isfinite(vh).all() else p @ vh
            out[rows, e] = o
            size[rows, e] = p @ vh.abs().nan_to_num(0.0, 0.0, 0.0)
            score[rows, e] = mag.amax(-1, keepdim=True).nan_to_num(0.0)
            lse[rows, e] = torch.where(some, torch.logsumexp(s, -1), -math.inf)
    return out, size, score, lse


def attend_bound(dtype, out, size, score):
    """How far a result may be: the weights are rounded once to the type (relative
    error of a unit each), the scores' sums of up to 256 products in fp32 are off by 2^-20 of
    their magnitude (which moves weights by that much, twice: weight and denominator), exp2
    and the sums by 2^-20 more, and the result is rounded once."""
    u = UNIT[dtype]
    e = 2.0 ** -19 * (score + 2)
    return (u + e) * size * (1 + 4 * u) + u * out.abs() + TINY[dtype]


def logits64(x, tokens, lens, prompts, repetition, frequency, presence, ids, values, mask):
    """(result, magnitude) in 64 bits."""
    y = x.double().clone()
    size = y.abs()
    rows, vocab = y.shape
    for b in range(rows):
        if tokens is not None:
            n = int(lens[b])
            p = 0 if prompts is None else int(prompts[b])
            seq = [int(t) for t in tokens[b, :n]]
            known = sorted({t for t in seq if 0 <= t < vocab})
            if repetition is not None and known:
                r = float(repetition[b])
                for t in known:
                    y[b, t] = y[b, t] / r if y[b, t] > 0 else y[b, t] * r
                    size[b, t] = y[b, t].abs()
            counts = {}
            for t in seq[p:]:
                if 0 <= t < vocab:
                    counts[t] = counts.get(t, 0) + 1
            for t, c in counts.items():
                d = (float(frequency[b]) * c if frequency is not None else 0.0)
                e = (float(presence[b]) if presence is not None else 0.0)
                y[b, t] = y[b, t] - d - e
                size[b, t] += abs(d) + abs(e)
        if ids is not None:
            for t, v in zip(ids[b].tolist(), values[b].tolist()):
                if 0 <= t < vocab:
                    y[b, t] += v
                    size[b, t] += abs(v)
        if mask is not None:
            for t in range(vocab):
                if not (int(mask[b, t // 32]) >> (t % 32)) & 1:
                    y[b, t] = -math.inf
    return y, size
