"""Token generation with an AQLM-quantised transformer: prompts of different
lengths go through the blocks in chunks, then all sequences are decoded together,
one token a step.

    python3 examples/generate.py [--layers 2] [--tokens 16] [--chunk 64] [--temperature 0.8] [--top-p 0.9]

The model is a small Llama-shaped one with random 2x8 codes and head norms (there
are no checkpoints here); what it shows is how the calls fit together:

    embed                        -> the residual stream
    layer_norm (RMS form, with the sum before it)
    q, k, v products (gemm)      -> paged_append  (head norms, rotation, cache)
                                 -> paged_attention over the cache
    o, gate, up, down products   (gemm)
    LM head, then process_logits (penalties, biases, a grammar mask), then sample
    (temperature 0, the default: the largest logit).

The gate's activation is plain torch.  The training forms: ``head_gradients``, the q and k
codebooks of a block through rope and its backward; ``end_gradients``, a step against a
teacher's largest logits through the loss, the last norm and the embedding.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2401_06118_amd as aqlm  # noqa: E402

EPS = 1e-5


class Linear:
    """A 2x8 layer with random codes: [d_out, d_in], about 1 / sqrt(d_in) large."""

    def __init__(self, gen, d_out, d_in, device):
        self.codes = torch.randint(0, 256, (d_out, d_in // 8, 2), generator=gen, device=device, dtype=torch.uint8)
        self.codebooks = (torch.randn(2, 256, 8, generator=gen, device=device) * (0.5 / d_in) ** 0.5).half()
        self.scales = torch.ones(d_out, dtype=torch.float16, device=device)

    @property
    def parts(self):
        return self.codes, self.codebooks, self.scales

    def __call__(self, x):
        return aqlm.gemm(*self.parts, x)


class Model:
    def __init__(self, layers=2, hidden=512, heads=8, kv=2, dim=64, ffn=1408, vocab=2000, positions=4096, device="cuda",
                 seed=0):
        gen = torch.Generator(device=device).manual_seed(seed)
        self.heads, self.kv, self.dim, self.hidden, self.vocab, self.device = heads, kv, dim, hidden, vocab, device
        self.embedding = torch.randn(vocab, hidden, generator=gen, device=device).half()
        self.head = torch.randn(vocab, hidden, generator=gen, device=device).half()
        self.table = aqlm.rotary_table(positions, dim, scaling={"kind": "llama3", "factor": 4.0, "original": 1024},
                                       device=device)
        self.blocks = [dict(qkv=Linear(gen, (heads + 2 * kv) * dim, hidden, device),
                            o=Linear(gen, hidden, heads * dim, device), gate=Linear(gen, ffn, hidden, device),
                            up=Linear(gen, ffn, hidden, device), down=Linear(gen, hidden, ffn, device),
                            q_weight=torch.ones(dim, dtype=torch.float16, device=device),
                            k_weight=torch.ones(dim, dtype=torch.float16, device=device))
                       for _ in range(layers)]

    def new_cache(self, pages, page_size=16):
        shape = (pages, page_size, self.kv, self.dim)
        return [tuple(torch.empty(shape, dtype=torch.float16, device=self.device) for _ in range(2))
                for _ in self.blocks]

    def forward(self, tokens, cache, block_table, kv_lens, cu_new, max_new):
        """Logits after each sequence's last new token.  ``tokens`` int64 [n], one sequence after
        another; ``kv_lens`` and ``cu_new`` as for aqlm.paged_append."""
        x, more = aqlm.embed(self.embedding, tokens.int()), None
        for b, (k_cache, v_cache) in zip(self.blocks, cache):
            h, x = rms(x, more)
            qkv = b["qkv"](h).view(len(tokens), self.heads + 2 * self.kv, self.dim)
            q, k, v = qkv.split((self.heads, self.kv, self.kv), 1)
            where = (k_cache, v_cache, block_table, kv_lens, cu_new)
            q = aqlm.paged_append(q, k, v, *where, table=self.table, q_weight=b["q_weight"], k_weight=b["k_weight"],
                                  eps=EPS, out=q)
            h, x = rms(x, b["o"](aqlm.paged_attention(q, *where, max_new=max_new).flatten(1)))
            more = b["down"]((torch.nn.functional.silu(b["gate"](h).float()) * b["up"](h).float()).half())
        at = cu_new[1:].long() - 1
        last, _ = rms(x[at], more[at])
        return last @ self.head.t() / self.hidden ** 0.5


def rms(x, more):
    """The norm of the residual stream after ``more`` is added to it, and the stream."""
    if more is None:
        return aqlm.layer_norm(x, rms=True, eps=EPS), x
    return aqlm.layer_norm(x, residual=more, rms=True, eps=EPS)


def head_gradients(model, block, x, dq, dk, positions):
    """Gradients of a block's q and k codebooks (and scales and norm weights) for upstream
    gradients of the rotated heads: what a fine-tuning step of the block needs of its
    first product."""
    b, n = model.blocks[block], model.heads + model.kv
    qkv = b["qkv"](x).view(len(x), n + model.kv, model.dim)
    gq, gk, gq_weight, gk_weight = aqlm.rope_backward(
        dq, dk, model.table, positions, q=qkv[:, :model.heads], k=qkv[:, model.heads:n], q_weight=b["q_weight"],
        k_weight=b["k_weight"], eps=EPS)
    dy = torch.cat([gq, gk, torch.zeros_like(gk)], 1).flatten(1)
    return (*aqlm.backward(*b["qkv"].parts, x, dy), gq_weight, gk_weight)


def end_gradients(model, tokens, weight, teacher_logits, teacher_ids, teacher_lse, loss_scale=1.0):
    """A step of the model's two ends alone, embedding, norm (``weight``) and head, against a
    teacher of whom each token's largest logits are known: the mean loss, and loss_scale times its
    gradients of the embedding (fp32), the norm's weight and the head."""
    n, scale = len(tokens), model.hidden ** -0.5
    x = aqlm.embed(model.embedding, tokens)
    h = aqlm.layer_norm(x, weight, rms=True, eps=EPS)
    logits = h @ model.head.t() * scale
    share = torch.full((n,), loss_scale / n, device=logits.device)
    loss, dlogits = aqlm.distill_loss(logits, teacher_logits, teacher_ids, teacher_lse=teacher_lse, weights=share,
                                      out=logits)
    dh = dlogits @ model.head * scale
    dx, dweight, _ = aqlm.layer_norm_backward(dh, x, weight, rms=True, eps=EPS)
    return loss.mean(), aqlm.embed_backward(dx, tokens, model.vocab, fp32=True), dweight, dlogits.t() @ h * scale


def generate(model, prompts, new_tokens, *, chunk=64, page_size=16, repetition=1.3, presence=0.2, banned=(), allowed=None,
             temperature=0.0, top_p=1.0, seed=0):
    """Continuations of the prompts (lists of ids), greedy at temperature 0: int64
    [sequences, new_tokens]."""
    dev, seqs = model.device, len(prompts)
    most = max(len(p) for p in prompts) + new_tokens
    width = -(-most // page_size)
    cache = model.new_cache(seqs * width, page_size)
    table = torch.randperm(seqs * width, device=dev).to(torch.int32).view(seqs, width)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731

    done = [0] * seqs
    while any(d < len(p) for d, p in zip(done, prompts)):  # a chunk of every prompt that has more
        new = [min(chunk, len(p) - d) for d, p in zip(done, prompts)]
        if min(new) <= 0:  # (a sequence may have no new tokens; its logits are kept from before)
            keep, ids = logits, [i for i, n in enumerate(new) if n > 0]
        else:
            keep, ids = None, list(range(seqs))
        tokens = [t for i in ids for t in prompts[i][done[i]:done[i] + new[i]]]
        done = [d + max(0, n) for d, n in zip(done, new)]
        cu = [sum(new[i] for i in ids[:j]) for j in range(len(ids) + 1)]
        logits = model.forward(torch.tensor(tokens, device=dev), cache, table[ids], ints([done[i] for i in ids]),
                               ints(cu), max(new))
        if keep is not None:
            keep[ids] = logits
            logits = keep

    history = torch.zeros(seqs, most, dtype=torch.int32, device=dev)
    for i, p in enumerate(prompts):
        history[i, :len(p)] = ints(p)
    prompt_lens = ints([len(p) for p in prompts])
    lens = prompt_lens.clone()
    rules = dict(repetition=torch.full((seqs,), repetition, device=dev),
                 presence=torch.full((seqs,), presence, device=dev))
    if banned:
        rules["bias_ids"] = ints(list(banned)).repeat(seqs, 1)
        rules["bias_values"] = torch.full((seqs, len(banned)), -torch.inf, device=dev)
    if allowed is not None:
        rules["mask"] = allowed.repeat(seqs, 1)
    cu = torch.arange(seqs + 1, dtype=torch.int32, device=dev)
    draw = dict(temperature=torch.full((seqs,), temperature, device=dev), top_p=torch.full((seqs,), top_p, device=dev))
    gen = torch.Generator(device=dev).manual_seed(seed)
    out = []
    for step in range(new_tokens):
        scored = aqlm.process_logits(logits, tokens=history, token_lens=lens, prompt_lens=prompt_lens, **rules)
        token = aqlm.sample(scored, torch.rand(seqs, generator=gen, device=dev), **draw)
        out.append(token)
        history.scatter_(1, lens[:, None].long(), token[:, None])
        lens += 1
        if step + 1 < new_tokens:
            logits = model.forward(token, cache, table, lens, cu, 1)
    return torch.stack(out, 1).long()


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--tokens", type=int, default=16)
    ap.add_argument("--chunk", type=int, default=64)
    ap.add_argument("--temperature", type=float, default=0.0)
    ap.add_argument("--top-p", type=float, default=1.0)
    a = ap.parse_args()
    model = Model(layers=a.layers)
    gen = torch.Generator().manual_seed(1)
    prompts = [torch.randint(0, model.vocab, (n,), generator=gen).tolist() for n in (5, 130, 77, 1)]
    for p, t in zip(prompts, generate(model, prompts, a.tokens, chunk=a.chunk, temperature=a.temperature,
                                          top_p=a.top_p).tolist()):
        print(f"prompt of {len(p)} tokens ->", t)


if __name__ == "__main__":
    main()
