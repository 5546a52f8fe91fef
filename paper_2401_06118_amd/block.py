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
of a fused projection's output), the elements of a head contiguous.  Every
computation runs in the library's kernels (``include/aqlm.h`` states their
rules); this module only marshals arguments and makes output tensors.
"""
from __future__ import annotations

import ctypes
import math

import torch

from . import _check, _lib, _stream_handle

_DTYPES = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}
_byref = ctypes.byref


def _heads(name, t, tokens=None, heads=None, like=None):
    """``aqlm_heads`` of a [tokens, heads, head_dim] tensor."""
    if t.dim() != 3 or not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor [tokens, heads, head_dim]")
    shape = t.shape
    st = t.stride()
    if st[2] != 1 and shape[2] > 1:
        raise ValueError(f"the elements of a head of {name} must be contiguous")
    if (tokens is not None and shape[0] != tokens) or (heads is not None and shape[1] != heads):
        raise ValueError(f"{name} must be [{tokens}, {heads}, head_dim], got {tuple(shape)}")
    if like is not None and (t.dtype != like.dtype or shape[2] != like.shape[2] or t.device != like.device):
        raise ValueError(f"{name} must have the type, head size and device of the other activations")
    if t.dtype not in _DTYPES:
        raise ValueError(f"{name} must be fp16, bf16 or fp32")
    # (the stride of a dimension of one is never used, whatever it says)
    return _lib.Heads(t.data_ptr(), st[0] if shape[0] > 1 else 0, st[1] if shape[1] > 1 else 0, shape[1])


def _vector(name, t, like, n, dtype):
    if t.dtype != dtype or t.numel() != n or not t.is_cuda or t.device != like.device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} GPU tensor of {n} elements")
    return t.data_ptr()


def _rotation(like, table, q_weight, k_weight, eps, interleaved):
    dim = like.shape[2]
    r = _lib.Rotation()
    if table is not None:
        if table.dtype != torch.float32 or table.dim() != 3 or table.shape[2] != 2 or not table.is_cuda \
                or table.device != like.device or not table.is_contiguous():
            raise ValueError("table must be a contiguous fp32 GPU tensor [positions, rot / 2, 2]")
        rot = 2 * table.shape[1]
        if rot > dim:
            raise ValueError(f"the table rotates {rot} elements of heads of {dim}")
        r.rot = rot
        if rot:
            r.table, r.rows = table.data_ptr(), table.shape[0]
    r.interleaved, r.eps = bool(interleaved), eps
    if q_weight is not None:
        r.q_weight = _vector("q_weight", q_weight, like, dim, like.dtype)
    if k_weight is not None:
        r.k_weight = _vector("k_weight", k_weight, like, dim, like.dtype)
    return r


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


def _like(t, out, name):
    """A caller's output, checked, or a new contiguous one of t's shape."""
    if out is None:
        return torch.empty(t.shape, dtype=t.dtype, device=t.device), True
    if out.shape != t.shape or out.dtype != t.dtype or out.device != t.device:
        raise ValueError(f"{name} must have the shape, type and device of its input")
    return out, False


def rope(q, k, table, positions, *, q_weight=None, k_weight=None, eps: float = 1e-6, interleaved: bool = False,
         out=None, stream=None):
    """Queries [tokens, heads, head_dim] and keys [tokens, kv heads, head_dim] with
    rotary positions: returns (q', k').  Where there is a weight [head_dim], each
    head is normalised first (x rsqrt(mean x^2 + eps) weight).  ``table`` as
    :func:`rotary_table` makes it (it may rotate the first part of the head only);
    ``positions`` int32 [tokens].  Pairs are (i, i + rot / 2), or (2i, 2i + 1) with
    ``interleaved``.  ``out``: a (q', k') to write, which may be (q, k) itself."""
    tokens = q.shape[0]
    hq, hk = _heads("q", q), _heads("k", k, tokens, None, q)
    r = _rotation(q, table, q_weight, k_weight, eps, interleaved)
    oq, oq_new = _like(q, None if out is None else out[0], "out")
    ok, ok_new = _like(k, None if out is None else out[1], "out")
    if stream is not None:
        _made(stream, oq if oq_new else None, ok if ok_new else None)
    pos = _vector("positions", positions, q, tokens, torch.int32)
    st = _lib.load().aqlm_rope(_byref(hq), _byref(hk), _byref(_heads("out", oq)), _byref(_heads("out", ok)),
                               _DTYPES[q.dtype], tokens, q.shape[2], pos, _byref(r), _stream_handle(stream))
    _check(st, "aqlm_rope")
    return oq, ok


def rope_backward(dq, dk, table, positions, *, q=None, k=None, q_weight=None, k_weight=None, eps: float = 1e-6,
                  interleaved: bool = False, out=None, stream=None):
    """Gradients of :func:`rope`: ``dq``, ``dk`` are those of its outputs; returns
    those of q, k and (fp32 [head_dim], or None) of the two weights.  ``q`` and
    ``k``, what the forward read, are needed where there is a weight."""
    tokens, dim = dq.shape[0], dq.shape[2] if dq.dim() == 3 else 0
    hdq, hdk = _heads("dq", dq), _heads("dk", dk, tokens, None, dq)
    r = _rotation(dq, table, q_weight, k_weight, eps, interleaved)
    pos = _vector("positions", positions, dq, tokens, torch.int32)
    gq, gq_new = _like(dq, None if out is None else out[0], "out")
    gk, gk_new = _like(dk, None if out is None else out[1], "out")
    if (q_weight is not None and q is None) or (k_weight is not None and k is None):
        raise ValueError("q and k are needed where their norm has a weight")
    hq = _byref(_heads("q", q, tokens, dq.shape[1], dq)) if q_weight is not None else None
    hk = _byref(_heads("k", k, tokens, dk.shape[1], dq)) if k_weight is not None else None
    wq = wk = ws = None
    ws_bytes = 0
    lib = _lib.load()
    if hq or hk:
        ws_bytes = int(lib.aqlm_rope_backward_workspace_bytes(dim))
        both = torch.empty((2, dim), dtype=torch.float32, device=dq.device)
        ws = torch.empty((ws_bytes,), dtype=torch.uint8, device=dq.device)
        wq = both[0] if hq else None
        wk = both[1] if hk else None
        if stream is not None:
            _made(stream, both, ws)
    if stream is not None:
        _made(stream, gq if gq_new else None, gk if gk_new else None)
    if tokens == 0:  # (nothing to sum over)
        for w in (wq, wk):
            if w is not None:
                w.zero_()
        return gq, gk, wq, wk
    st = lib.aqlm_rope_backward(
        _byref(hdq), _byref(hdk), hq, hk, _byref(_heads("out", gq)), _byref(_heads("out", gk)),
        wq.data_ptr() if wq is not None else None, wk.data_ptr() if wk is not None else None, _DTYPES[dq.dtype],
        tokens, dim, pos, _byref(r), ws.data_ptr() if ws is not None else None, ws_bytes, _stream_handle(stream))
    _check(st, "aqlm_rope_backward")
    return gq, gk, wq, wk


def _cache(k_cache, v_cache, block_table, kv_lens, cu_new):
    """``aqlm_paged_cache`` of the cache's tensors and the batch's integers."""
    for name, t in (("k_cache", k_cache), ("v_cache", v_cache)):
        if t.dim() != 4 or not t.is_cuda or t.dtype not in _DTYPES:
            raise ValueError(f"{name} must be a GPU tensor [pages, page_size, kv heads, head_dim]")
        if t.stride(3) != 1 and t.shape[3] > 1:
            raise ValueError(f"the elements of a head of {name} must be contiguous")
    if k_cache.shape != v_cache.shape or k_cache.dtype != v_cache.dtype or k_cache.device != v_cache.device:
        raise ValueError("k_cache and v_cache must have one shape, type and device")
    pages, page_size, kv_heads, dim = k_cache.shape
    if block_table.dtype != torch.int32 or block_table.dim() != 2 or block_table.device != k_cache.device \
            or (block_table.stride(1) != 1 and block_table.shape[1] > 1):
        raise ValueError("block_table must be an int32 tensor [sequences, pages] on the cache's device")
    seqs, width = block_table.shape
    ks, vs = k_cache.stride(), v_cache.stride()
    if pages == 1 or page_size == 1 or kv_heads == 1:  # (such strides are never used, whatever they say)
        ks, vs = ([s if n > 1 else 0 for s, n in zip(st, k_cache.shape)] for st in (ks, vs))
    return _lib.PagedCache(
        k_cache.data_ptr(), v_cache.data_ptr(), ks[0], ks[1], ks[2], vs[0], vs[1], vs[2], pages,
        block_table.data_ptr(), block_table.stride(0), _vector("kv_lens", kv_lens, k_cache, seqs, torch.int32),
        _vector("cu_new", cu_new, k_cache, seqs + 1, torch.int32), width, seqs, page_size, kv_heads, dim,
        _DTYPES[k_cache.dtype])


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
    c = _cache(k_cache, v_cache, block_table, kv_lens, cu_new)
    tokens = k.shape[0]
    hk, hv = _heads("k", k, tokens, c.kv_heads, k), _heads("v", v, tokens, c.kv_heads, k)
    if k.dtype != k_cache.dtype or k.shape[2] != c.head_dim or k.device != k_cache.device:
        raise ValueError("the activations must have the cache's type, head size and device")
    r = _rotation(k, table, q_weight, k_weight, eps, interleaved)
    hq = ho = oq = None
    if q is not None:
        hq = _byref(_heads("q", q, tokens, None, k))
        oq, new = _like(q, out, "out")
        ho = _byref(_heads("out", oq))
        if new and stream is not None:
            _made(stream, oq)
    st = _lib.load().aqlm_paged_append(hq, _byref(hk), _byref(hv), ho, _byref(c), tokens, _byref(r),
                                       _stream_handle(stream))
    _check(st, "aqlm_paged_append")
    return oq


def attention_workspace(head_dim: int, device="cuda") -> torch.Tensor:
    """A workspace for :func:`paged_attention` with heads of up to ``head_dim``
    elements, ready for use.  One serves any calls on one stream, one after another."""
    need = int(_lib.load().aqlm_paged_attention_workspace_bytes(int(head_dim)))
    if need <= 0:
        raise ValueError("head_dim must be a multiple of 8 up to 256")
    return torch.zeros((need,), dtype=torch.uint8, device=device)


# Workspaces of calls that bring none, one per device, stream and padded head
# size: calls on one stream run one after another.
_workspaces = {}


def _workspace(device, head_dim, stream_handle):
    if torch.cuda.is_current_stream_capturing():
        # a graph's launches may run beside this stream's later ones: it gets its own
        return attention_workspace(head_dim, device)
    key = (device, stream_handle, 64 if head_dim <= 64 else 128 if head_dim <= 128 else 256)
    ws = _workspaces.get(key)
    if ws is None:
        ws = attention_workspace(key[2], device)
        if stream_handle != _stream_handle(None):
            torch.cuda.current_stream(device).synchronize()  # (zeroed on the current stream, used on another)
        _workspaces[key] = ws
    return ws


def paged_attention(q, k_cache, v_cache, block_table, kv_lens, cu_new, *, scale=None, causal: bool = True,
                    window: int = 0, max_new: int = 0, return_lse: bool = False, out=None, workspace=None,
                    stream=None):
    """Attention of the new tokens' queries [tokens, heads, head_dim] over their
    sequences' pages (cache, lengths and table as for :func:`paged_append`, after
    it): returns [tokens, heads, head_dim], or with ``return_lse`` also the logarithm
    of each row's softmax denominator (fp32 [tokens, heads]).  Query head e reads kv
    head e // (heads / kv heads).  ``scale``: 1 / sqrt(head_dim) if not given.
    ``causal``: a token sees keys up to its own position; ``window`` above 0: only that
    many positions up to its own.  A row that sees no key is 0, its lse -inf.
    ``max_new``: the most new tokens of a sequence, if known (it chooses the kernel,
    not the result).  ``workspace``: as :func:`attention_workspace` makes it;
    without one, one per stream is kept."""
    c = _cache(k_cache, v_cache, block_table, kv_lens, cu_new)
    hq = _heads("q", q)
    tokens, heads, dim = q.shape
    if q.dtype != k_cache.dtype or dim != c.head_dim or q.device != k_cache.device:
        raise ValueError("q must have the cache's type, head size and device")
    if heads % c.kv_heads:
        raise ValueError("the query heads must be a multiple of the kv heads")
    handle = _stream_handle(stream)
    out, new = _like(q, out, "out")
    lse = torch.empty((tokens, heads), dtype=torch.float32, device=q.device) if return_lse else None
    if workspace is None:
        if dim % 8 or dim > 256:
            raise ValueError("head_dim must be a multiple of 8 up to 256")
        workspace = _workspace(q.device, dim, handle)
    elif not workspace.is_cuda or workspace.device != q.device or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous GPU tensor on q's device")
    if stream is not None:
        _made(stream, out if new else None, lse)
    st = _lib.load().aqlm_paged_attention(
        _byref(hq), _byref(_heads("out", out)), lse.data_ptr() if return_lse else None, _byref(c), tokens,
        int(max_new), dim ** -0.5 if scale is None else scale, bool(causal), int(window), workspace.data_ptr(),
        workspace.numel() * workspace.element_size(), handle)
    _check(st, "aqlm_paged_attention")
    return (out, lse) if return_lse else out


def _table2(name, t, rows, dtype, like):
    if t.dtype != dtype or t.dim() != 2 or t.shape[0] != rows or not t.is_cuda or t.device != like.device \
            or (t.stride(1) != 1 and t.shape[1] > 1):
        raise ValueError(f"{name} must be a {dtype} GPU tensor [{rows}, n], its rows contiguous")
    return t.data_ptr()


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
    if logits.dim() != 2 or not logits.is_cuda or logits.dtype not in _DTYPES \
            or (logits.stride(1) != 1 and logits.shape[1] > 1):
        raise ValueError("logits must be an fp16, bf16 or fp32 GPU tensor [rows, vocab], its rows contiguous")
    rows, vocab = logits.shape
    r = _lib.LogitRules()
    if tokens is not None:
        if token_lens is None:
            raise ValueError("tokens need token_lens")
        r.tokens = _table2("tokens", tokens, rows, torch.int32, logits)
        r.history, r.token_stride = tokens.shape[1], tokens.stride(0)
        r.token_lens = _vector("token_lens", token_lens, logits, rows, torch.int32)
        if prompt_lens is not None:
            r.prompt_lens = _vector("prompt_lens", prompt_lens, logits, rows, torch.int32)
    elif repetition is not None or frequency is not None or presence is not None:
        raise ValueError("penalties need tokens")
    if tokens is not None and tokens.shape[1] == 0:  # (nothing to penalise)
        tokens = repetition = frequency = presence = None
        r.tokens = r.token_lens = r.prompt_lens = None
    if repetition is not None:
        r.repetition = _vector("repetition", repetition, logits, rows, torch.float32)
    if frequency is not None:
        r.frequency = _vector("frequency", frequency, logits, rows, torch.float32)
    if presence is not None:
        r.presence = _vector("presence", presence, logits, rows, torch.float32)
    if (bias_ids is None) != (bias_values is None):
        raise ValueError("bias_ids and bias_values go together")
    if bias_ids is not None:
        if bias_ids.shape != bias_values.shape or bias_ids.stride() != bias_values.stride():
            raise ValueError("bias_ids and bias_values must have one shape and layout")
        r.bias_ids = _table2("bias_ids", bias_ids, rows, torch.int32, logits)
        r.bias_values = _table2("bias_values", bias_values, rows, torch.float32, logits)
        r.biases, r.bias_stride = bias_ids.shape[1], bias_ids.stride(0)
    if mask is not None:
        r.mask = _table2("mask", mask, rows, torch.int32, logits)
        r.mask_stride = mask.stride(0)
        if mask.shape[1] < (vocab + 31) // 32:
            raise ValueError(f"mask must have {(vocab + 31) // 32} words per row")
    if out is None:
        out = torch.empty((rows, vocab), dtype=logits.dtype, device=logits.device)
        if stream is not None:
            _made(stream, out)
    elif out.shape != logits.shape or out.dtype != logits.dtype or out.device != logits.device \
            or (out.stride(1) != 1 and vocab > 1):
        raise ValueError("out must have the shape, type and device of logits, its rows contiguous")
    in_row, out_row = (logits.stride(0), out.stride(0)) if rows > 1 else (0, 0)
    st = _lib.load().aqlm_process_logits(logits.data_ptr(), in_row, out.data_ptr(), out_row, _DTYPES[logits.dtype],
                                         rows, vocab, _byref(r), _stream_handle(stream))
    _check(st, "aqlm_process_logits")
    return out
