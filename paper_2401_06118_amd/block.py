"""The operators between the products of a transformer block and at the end of
a decode step, on torch tensors that live on the GPU:

- :func:`rotary_table` - cos and sin of rotary positions, scaled for long
  contexts or not;
- :func:`rope` / :func:`rope_backward` - rotary positions of queries and keys with
  the RMS norm of each head before them, and the gradients;
- :func:`paged_append` - the same on the way into a paged key/value cache;
- :func:`paged_attention` - attention of each sequence's new tokens over its pages;
- :func:`process_logits` - penalties for repeated tokens, biases, grammar masks.

Activations are [tokens, heads, head_dim] with any token and head strides (views
of a fused projection's output), the elements of a head contiguous.  ``stream``: where
the launches go, the current stream if not given; another one has to wait for the
current one first (``stream.wait_stream``), whose work may still use the inputs and the
memory that outputs are made of.  Every
computation runs in the library's kernels (``include/aqlm.h`` states their
rules); this module only marshals arguments and makes output tensors.  As
elsewhere in this package no autograd graph is recorded: gradients are calls of
their own.  Tensors that a call writes (``out``, caches) count as modified in place, so
autograd refuses to use what it saved of them.
"""
from __future__ import annotations

import math
import os
import threading

import torch

from . import _check, _lib, _stream_handle

_COUNTER_BYTES = 16384  # AQLM_ATTENTION_COUNTER_BYTES
_lock = threading.Lock()
_ext = None


def _binding():
    """The C++ binding (raises if it has not been built)."""
    global _ext
    if _ext is None:
        with _lock:
            if _ext is None:
                if not os.path.exists(os.path.join(_lib.HERE, "_block.so")):
                    raise RuntimeError("_block.so is missing: build it with `python -m paper_2401_06118_amd.build` "
                                       "(hipcc, gfx950). There is no CPU fallback.")
                _lib.load()
                from . import _block
                _block.set_check(_check)
                _ext = _block
    return _ext


def _made(stream, *tensors):
    """Tensors made here are the current stream's; tells the allocator where ``stream`` is another one."""
    if stream is not None and stream != torch.cuda.current_stream():
        for t in tensors:
            if t is not None:
                t.record_stream(stream)


def rotary_table(positions: int, rot: int, *, base: float = 10000.0, scaling=None, device="cuda",
                 stream=None) -> torch.Tensor:
    """cos and sin of ``positions`` rotary positions for heads of which ``rot``
    elements are rotated: fp32 [positions, rot / 2, 2], for :func:`rope` and
    :func:`paged_append`.  Pair i turns by position * base^(-2i / rot), changed by
    ``scaling`` (None or a dict), with n the context length that the model was trained for:

    - ``{"kind": "linear", "factor": f}``: positions divided by f;
    - ``{"kind": "ntk", "factor": f}``: base multiplied by f^(rot / (rot - 2));
    - ``{"kind": "yarn", "factor": f, "original": n}`` (``fast`` 32, ``slow`` 1): pairs
      that turn less than ``slow`` times in n positions are divided by f, those of more
      than ``fast`` turns kept, linearly between by the pair's number; cos and sin
      multiplied by ``attention`` (default 0.1 ln f + 1);
    - ``{"kind": "llama3", "factor": f, "original": n}`` (``low`` 1, ``high`` 4): the same
      idea, linear between in the number of turns.
    """
    rot, positions = int(rot), int(positions)
    if positions <= 0 or rot <= 0 or rot % 2:
        raise ValueError("positions must be positive, rot positive and even")
    half = rot // 2
    freq = [float(base) ** (-2.0 * i / rot) for i in range(half)]
    scale = 1.0
    if scaling is not None:
        kind, f = scaling.get("kind"), float(scaling.get("factor", 1.0))
        if f <= 0:
            raise ValueError("scaling's factor must be positive")
        if kind == "linear":
            freq = [w / f for w in freq]
        elif kind == "ntk":
            if rot <= 2:
                raise ValueError("ntk scaling needs rot of more than 2")
            b = float(base) * f ** (rot / (rot - 2))
            freq = [b ** (-2.0 * i / rot) for i in range(half)]
        elif kind == "yarn":
            n = float(scaling["original"])
            # the pair that turns t times in n positions
            pair = lambda t: rot * math.log(n / (t * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
            lo = max(0.0, math.floor(pair(float(scaling.get("fast", 32.0)))))
            hi = min(rot - 1.0, math.ceil(pair(float(scaling.get("slow", 1.0)))))
            part = [min(1.0, max(0.0, (i - lo) / max(hi - lo, 1e-3))) for i in range(half)]
            freq = [w * (1 - p) + w / f * p for w, p in zip(freq, part)]
            scale = float(scaling.get("attention", 0.1 * math.log(f) + 1.0 if f > 1 else 1.0))
        elif kind == "llama3":
            n, low, high = float(scaling["original"]), float(scaling.get("low", 1.0)), float(scaling.get("high", 4.0))
            if not high > low:
                raise ValueError("llama3 scaling needs high above low")
            keep = [min(1.0, max(0.0, (n * w / (2 * math.pi) - low) / (high - low))) for w in freq]
            freq = [w * k + w / f * (1 - k) for w, k in zip(freq, keep)]
        else:
            raise ValueError("scaling's kind must be linear, ntk, yarn or llama3")
    inv = torch.tensor(freq, dtype=torch.float64).to(device)
    out = torch.empty((positions, half, 2), dtype=torch.float32, device=inv.device)
    _made(stream, inv, out)
    st = _lib.load().aqlm_rotary_table(inv.data_ptr(), positions, half, scale, out.data_ptr(), _stream_handle(stream))
    _check(st, "aqlm_rotary_table")
    return out


def rope(q, k, table, positions, *, q_weight=None, k_weight=None, eps: float = 1e-6, interleaved: bool = False,
         out=None, stream=None):
    """Queries [tokens, heads, head_dim] and keys [tokens, kv heads, head_dim] with
    rotary positions: returns (q', k').  Where there is a weight [head_dim], each
    head is normalised first (x rsqrt(mean x^2 + eps) weight).  ``table`` as
    :func:`rotary_table` makes it (it may rotate the first part of the head only);
    ``positions`` int32 [tokens].  Pairs are (i, i + rot / 2), or (2i, 2i + 1) with
    ``interleaved``.  ``out``: a (q', k') to write, which may be (q, k) itself."""
    oq, ok = (None, None) if out is None else out
    r = (_ext or _binding()).rope(q, k, table, positions, q_weight, k_weight, eps, interleaved, oq, ok,
                                  _stream_handle(stream))
    if stream is not None and out is None:
        _made(stream, *r)
    return r


def rope_backward(dq, dk, table, positions, *, q=None, k=None, q_weight=None, k_weight=None, eps: float = 1e-6,
                  interleaved: bool = False, out=None, stream=None):
    """Gradients of :func:`rope`: ``dq``, ``dk`` are those of its outputs; returns
    those of q, k and (fp32 [head_dim], or None) of the two weights.  ``q`` and
    ``k``, what the forward read, are needed where there is a weight."""
    oq, ok = (None, None) if out is None else out
    r = (_ext or _binding()).rope_backward(dq, dk, table, positions, q, k, q_weight, k_weight, eps, interleaved, oq,
                                           ok, _stream_handle(stream))
    if stream is not None:
        if dq.shape[0] == 0:  # (the weights' gradients are zeros, written on the current stream)
            stream.wait_stream(torch.cuda.current_stream())
        _made(stream, *(r if out is None else r[2:]))
    return r[:4]


def paged_append(q, k, v, k_cache, v_cache, block_table, kv_lens, cu_new, *, table=None, q_weight=None, k_weight=None,
                 eps: float = 1e-6, interleaved: bool = False, out=None, stream=None):
    """Writes the new tokens' keys (normalised and rotated as by :func:`rope`) and
    values to their pages and returns the queries, normalised and rotated (None for
    ``q`` None).  ``k_cache``, ``v_cache``: [pages, page_size, kv heads, head_dim], any
    strides but the last; ``block_table`` int32 [sequences, pages of a sequence];
    ``kv_lens`` int32 [sequences], the keys of each sequence with the new ones;
    ``cu_new`` int32 [sequences + 1], where each sequence's new tokens begin among
    the activations.  Positions follow from these.  Without ``table`` nothing is
    rotated."""
    r = (_ext or _binding()).paged_append(q, k, v, k_cache, v_cache, block_table, kv_lens, cu_new, table, q_weight,
                                          k_weight, eps, interleaved, out, _stream_handle(stream))
    if stream is not None and out is None:
        _made(stream, r)
    return r


def attention_workspace(head_dim: int, device="cuda") -> torch.Tensor:
    """A workspace for :func:`paged_attention` with heads of up to ``head_dim``
    elements, ready for use (heads of up to 64, 128 and 256 elements: 35, 68 and 68 MB).  One
    serves any calls on one stream, one after another."""
    need = int(_lib.load().aqlm_paged_attention_workspace_bytes(int(head_dim)))
    if need <= 0:
        raise ValueError("head_dim must be a multiple of 8 up to 256")
    ws = torch.empty((need,), dtype=torch.uint8, device=device)
    ws[:_COUNTER_BYTES].zero_()
    return ws


# Workspaces of calls that bring none, one per device, stream and padded head
# size: calls on one stream run one after another.  Kept for good, as a stream's
# later calls may come at any time.
_workspaces = {}
_workspaces_lock = threading.Lock()


def _workspace(device, head_dim, stream, handle):
    if head_dim % 8 or not 0 < head_dim <= 256 or device.type != "cuda":
        raise ValueError("paged_attention takes GPU tensors and a head_dim that is a multiple of 8 up to 256")
    if (_ext or _binding()).capturing(handle):
        # a graph's launches may run beside this stream's later ones: it gets its own
        return _workspace_on(stream, device, head_dim)
    key = (device, handle, 64 if head_dim <= 64 else 128 if head_dim <= 128 else 256)
    ws = _workspaces.get(key)
    if ws is None:
        with _workspaces_lock:  # (of threads that come together, one makes it)
            ws = _workspaces.get(key)
            if ws is None:
                ws = _workspaces[key] = _workspace_on(stream, device, key[2])
    return ws


def _workspace_on(stream, device, head_dim):
    """Made and zeroed on the stream that launches: in its order, its graph and its memory."""
    if stream is None:
        return attention_workspace(head_dim, device)
    with torch.cuda.stream(stream):
        return attention_workspace(head_dim, device)


def paged_attention(q, k_cache, v_cache, block_table, kv_lens, cu_new, *, scale=None, causal: bool = True,
                    window: int = 0, max_new: int = 0, return_lse: bool = False, out=None, workspace=None,
                    stream=None):
    """Attention of the new tokens' queries [tokens, heads, head_dim] over their
    sequences' pages (cache, lengths and table as for :func:`paged_append`, after
    it): returns [tokens, heads, head_dim], or with ``return_lse`` also the logarithm
    of each row's softmax denominator (fp32 [tokens, heads]).  Query head e reads kv
    head e // (heads / kv heads).  ``scale``: 1 / sqrt(head_dim) if not given.
    ``causal``: a token sees keys up to its own position; ``window`` above 0: only that
    many positions up to its own.  A row that sees no key, or whose token no sequence holds, is 0, its lse -inf.
    ``max_new``: the most new tokens of a sequence, if known.  It chooses the kernel, any
    value is right; without it a call of more than 16 rows (tokens times heads per kv
    head) takes the kernel for many rows, which is up to twice as slow for single tokens
    and rounds the weights once more.  ``workspace``: as :func:`attention_workspace` makes it;
    without one, one per stream and size of heads is kept for good."""
    handle = _stream_handle(stream)
    if workspace is None:
        workspace = _workspace(q.device, q.shape[-1], stream, handle)
    r = (_ext or _binding()).paged_attention(q, k_cache, v_cache, block_table, kv_lens, cu_new, scale, causal, window,
                                             max_new, return_lse, out, workspace, handle)
    if stream is not None:
        _made(stream, *(r if return_lse else (r,)))
    return r


def process_logits(logits, *, tokens=None, token_lens=None, prompt_lens=None, repetition=None, frequency=None,
                   presence=None, bias_ids=None, bias_values=None, mask=None, out=None, stream=None) -> torch.Tensor:
    """Logits [rows, vocab] (fp16, bf16, fp32) after, in this order: a repetition
    penalty (divide positive, multiply negative ones) for every token among a row's
    ``tokens`` so far; frequency (times its count) and presence penalties for those of
    its output; biases; and -inf where the ``mask`` does not allow a token.

    ``tokens`` int32 [rows, n] of which ``token_lens`` int32 [rows] are in use, the first
    ``prompt_lens`` (int32 [rows], none if not given) of them the prompt; penalties fp32
    [rows]; ``bias_ids`` int32 [rows, n] (negative: no entry) with ``bias_values`` fp32
    [rows, n]; ``mask`` int32 [rows, ceil(vocab / 32)], bit token % 32 of word token //
    32 set where the token is allowed.  ``out`` may be ``logits`` itself."""
    r = (_ext or _binding()).process_logits(logits, tokens, token_lens, prompt_lens, repetition, frequency, presence,
                                            bias_ids, bias_values, mask, out, _stream_handle(stream))
    if stream is not None and out is None:
        _made(stream, r)
    return r
