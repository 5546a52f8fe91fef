"""The operators of ``ends.py`` from their definitions, in 64 bits, with bounds on how far
results in 32 bits, rounded once, can be from them.

A rounding to a type is off by half a step: ``HALF`` of the value, or half the smallest
subnormal.  A sum of n terms in 32 bits is off by at most n 2^-24 of the sum of their sizes.
"""
import math

import torch

E32 = 2.0 ** -24
HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -150}


def rounded(exact, dtype):
    """Bound of one rounding to dtype."""
    return exact.abs() * HALF[dtype] * (1 + 2.0 ** -8) + TINY[dtype] * 2


def check(got, exact, bound, what=""):
    got, bound = got.double(), bound.expand_as(exact)
    same = (got == exact) | (torch.isnan(got) & torch.isnan(exact))
    bad = ~same & ~((got - exact).abs() <= bound)
    if bad.any():
        i = tuple(int(v) for v in bad.nonzero()[0])
        raise AssertionError(f"{what} {int(bad.sum())} of {bad.numel()} outside; at {i}: got {got[i].item()!r}, exact "
                             f"{exact[i].item()!r}, bound {bound[i].item():.3g}")


def embed(table, tokens, scale):
    ids = tokens.long()
    held = (ids >= 0) & (ids < table.shape[0])
    y = table.double()[ids.clamp(0, table.shape[0] - 1)] * scale
    return torch.where(held[:, None], y, 0.0)


def embed_grad(dout, tokens, vocab, scale):
    """The gradient, and the bound of its sum in 32 bits."""
    ids = tokens.long()
    held = (ids >= 0) & (ids < vocab)
    zero = torch.zeros(vocab, dout.shape[1], dtype=torch.float64, device=dout.device)
    d = dout[held].double()
    g, size = zero.index_add(0, ids[held], d), zero.index_add(0, ids[held], d.abs())
    n = torch.bincount(ids[held], minlength=vocab)[:, None].double()
    # n - 1 additions, the scale's product (and fp32's rounding of the scale itself)
    return g * scale, size * abs(scale) * (n + 2) * E32


def norm(h, weight, bias, eps, rms):
    """y, and what the gradient needs: xhat, r, the bound of xhat."""
    h = h.double()
    mu = torch.zeros_like(h[:, :1]) if rms else h.mean(1, keepdim=True)
    r = ((h - mu).square().mean(1, keepdim=True) + eps).rsqrt()
    xhat = (h - mu) * r
    # Sums pass 32 elements of a thread, 6 steps in the wave and 16 waves: 54 additions, and a
    # few roundings of products, quotients and the root; mu and eps are rounded to 32 bits
    off = 64 * E32 * (xhat.abs() + 1) + 2 * E32 * mu.abs() * r
    y = xhat if weight is None else xhat * weight.double()
    bound = off if weight is None else off * weight.double().abs()
    if bias is not None:
        y = y + bias.double()
    return y, bound + 3 * E32 * y.abs() + (0 if bias is None else 2 * E32 * bias.double().abs()), xhat, r, off


def norm_grad(dy, h, weight, dsum, eps, rms):
    """(dx, bound), (dweight, bound), (dbias, bound)."""
    _, _, xhat, r, off = norm(h, weight, None, eps, rms)
    dy = dy.double()
    g = dy if weight is None else dy * weight.double()
    by = (g * xhat).mean(1, keepdim=True)
    d = g - xhat * by
    size = g.abs() + xhat.abs() * (g * xhat).abs().mean(1, keepdim=True)
    slip = off * by.abs() + xhat.abs() * (g.abs() * off).mean(1, keepdim=True)
    if not rms:
        d = d - g.mean(1, keepdim=True)
        size = size + g.abs().mean(1, keepdim=True)
    d = d * r
    bound = r * (128 * E32 * size + slip)
    if dsum is not None:
        d = d + dsum.double()
        bound = bound + 2 * E32 * dsum.double().abs()
    n = len(dy) + 64  # (rows of a slot, slots of a wave, waves)
    return ((d, bound), ((dy * xhat).sum(0), ((dy * xhat).abs() * (n + 4) * E32 + dy.abs() * off).sum(0)),
            (dy.sum(0), dy.abs().sum(0) * n * E32))


def distill(logits, teacher, ids, lse, weights, tau):
    """loss, gradient and their bounds, row by row (automatic differentiation)."""
    rows, vocab = logits.shape
    f64 = dict(dtype=torch.float64, device=logits.device)
    loss, loss_off = torch.zeros(rows, **f64), torch.zeros(rows, **f64)
    grad, grad_off = torch.zeros(rows, vocab, **f64), torch.zeros(rows, vocab, **f64)
    for b in range(rows):
        w = 1.0 if weights is None else float(weights[b])
        if w == 0:
            continue
        held = (ids[b] >= 0) & (ids[b] < vocab)
        if not held.any():
            continue
        z = logits[b].double().requires_grad_(True)
        at, t = ids[b][held].long(), teacher[b][held].double() / tau
        log_q = torch.log_softmax(z / tau, 0)
        log_p = t - (torch.logsumexp(t, 0) if lse is None else lse[b].double())
        p = log_p.exp()
        value = (p * torch.where(p > 0, log_p - log_q[at], 0)).sum()
        pr = torch.zeros((), **f64)
        outside = torch.ones(vocab, dtype=torch.bool, device=z.device)
        outside[at] = False
        q = log_q.detach().exp()
        if lse is not None:
            pr = (1 - p.sum()).clamp(min=0) * outside.any()
            if float(pr) > 0:
                value = value + pr * (pr.log() - torch.logsumexp(log_q[outside], 0))
        (g,) = torch.autograd.grad(value, z)
        loss[b], grad[b] = value.detach(), g * w
        # The sum outside the list: up to 128 additions of a thread and 17 changes of its maximum,
        # each term's argument rounded three times and its exponential to 2^-23
        d = (logits[b].double() - logits[b].double().max()) / tau
        d = torch.where(torch.isfinite(d), d, 0).abs()
        delta = float(128 + 2 * 17 + 8 + 3 * (q * d).sum() / max(float((q * outside).sum()), 1e-30)) * E32
        loss_off[b] = delta + 2 * E32 * abs(value.item()) + 1e-14
        qr = float((q * outside).sum())
        many = p.sum() + pr
        size = torch.where(outside, q / max(qr, 1e-300) * (qr * many + pr), q * many)
        size[at] += p  # (duplicates: any of their masses)
        grad_off[b] = abs(w) / tau * size * (delta + (3 * d + 8) * E32)
    return loss, loss_off, grad, grad_off


def sample(x, u, t=1.0, k=0, p=1.0, m=0.0):
    """(token, log-probability) of one row, by the sorted list of its tokens."""
    x = x.double()
    if torch.isnan(x).any() or float(x.max()) == -math.inf:
        return -1, math.nan
    if not t > 0:
        return int((x == x.max()).nonzero()[0, 0]), 0.0
    vals, ids = torch.sort(x, descending=True, stable=True)
    n = int((vals > -math.inf).sum())
    if k > 0:
        n = min(n, k)
    d = torch.where(vals[:n] == vals[0], 0.0, vals[:n] - vals[0])
    w = torch.exp(d / t)
    if p < 1:
        before = torch.cumsum(w, 0) - w
        n = max(1, int((before < p * w.sum()).sum()))
    if m > 0:
        n = min(n, max(1, int((d[:n] >= t * math.log(min(m, 1.0))).sum())))
    ids, by = torch.sort(ids[:n])
    w = w[:n][by]
    upto = torch.cumsum(w, 0)
    some = (w > 0).nonzero()[-1, 0]
    i = min(int(some), int((upto <= u * upto[-1]).sum()))
    return int(ids[i]), float(torch.log(w[i] / upto[-1]))
