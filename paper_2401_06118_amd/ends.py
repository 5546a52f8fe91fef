"""The ends of a model and the norms of its residual stream, on torch tensors that
live on the GPU:

- :func:`embed` / :func:`embed_backward` - rows of the embedding table, scaled, and the
  table's gradient;
- :func:`layer_norm` / :func:`layer_norm_backward` - layer or RMS norm with the residual
  sum before it, and the gradients;
- :func:`distill_loss` - the loss of logits against a teacher's largest ones and its
  gradient;
- :func:`sample` - a token of each row of logits by temperature, top-k, top-p and min-p.

Activations are [rows, n] (fp16, bf16 or fp32) with any row stride, the elements of a row
contiguous.  ``stream``: where the launches go, the current stream of the tensors' device if
not given; another one has to wait for the current one first (``stream.wait_stream``), whose
work may still use the inputs and the memory that outputs are made of.  Every computation
runs in the library's kernels (``include/aqlm.h`` states their rules); this module
only marshals arguments and makes output tensors.  No autograd graph is recorded:
gradients are calls of their own.  Tensors that a call writes (``out``) count as modified in
place, so autograd refuses to use what it saved of them.
"""
from __future__ import annotations

import torch

from . import _stream_handle, block
from .block import _binding, _made


def _handle(t, stream) -> int:
    """The stream's handle; a launch on another device than the tensors' is refused."""
    if stream is None:
        if t.is_cuda and t.get_device() != torch.cuda.current_device():
            return int(torch.cuda.current_stream(t.device).cuda_stream)
        return _stream_handle(None) if t.is_cuda else 0
    if t.is_cuda and stream.device != t.device:
        raise ValueError(f"stream is one of {stream.device}, the tensors are on {t.device}")
    return _stream_handle(stream)


def embed(table, tokens, *, scale: float = 1.0, out=None, stream=None) -> torch.Tensor:
    """scale * table[token] for each of ``tokens`` (int32 [tokens]): [tokens, dim] of the
    type of ``table`` [vocab, dim].  A token outside the table (padding) gives zeros."""
    r = (block._ext or _binding()).embed(table, tokens, scale, out, _handle(table, stream))
    if stream is not None and out is None:
        _made(stream, r)
    return r


def embed_backward(dout, tokens, vocab: int, *, scale: float = 1.0, fp32: bool = False, out=None,
                   stream=None) -> torch.Tensor:
    """Gradient of :func:`embed`'s table: [vocab, dim], for each token the sum of ``dout``
    [tokens, dim] over its places, times ``scale``; zeros for tokens that do not occur.  Summed in
    fp32 in a fixed order; of the type of ``dout``, or fp32 with ``fp32`` or an fp32 ``out``."""
    r, ws = (block._ext or _binding()).embed_backward(dout, tokens, vocab, scale, fp32, out, _handle(dout, stream))
    if stream is not None:
        _made(stream, ws, r if out is None else None)
    return r


def layer_norm(x, weight=None, bias=None, *, residual=None, eps: float = 1e-5, rms: bool = False, out=None,
               sum_out=None, stream=None):
    """(x - mean) / sqrt(variance + eps) * weight + bias over each row of ``x`` [rows, dim];
    with ``rms`` x / sqrt(mean x^2 + eps) * weight + bias.  With ``residual`` [rows, dim] the
    norm is that of h = x + residual, rounded to its type, and the result (y, h).  ``weight``,
    ``bias``: [dim] of the type of ``x``, or None.  ``out`` and ``sum_out`` (for h) may each be
    ``x`` or ``residual`` itself, not one another.  dim up to 16384."""
    r = (block._ext or _binding()).layer_norm(x, weight, bias, residual, eps, rms, out, sum_out, _handle(x, stream))
    if stream is not None:
        y, h = r if residual is not None else (r, None)
        _made(stream, y if out is None else None, h if sum_out is None else None)
    return r


def layer_norm_backward(dy, x, weight=None, *, dsum=None, eps: float = 1e-5, rms: bool = False, bias: bool = False,
                        out=None, stream=None):
    """Gradients of :func:`layer_norm`: ``dy`` is that of its output, ``x`` what it
    normalised (h, where there was a residual), ``dsum`` the gradient that h gets from elsewhere.
    Returns (dx, dweight, dbias): dx = dsum + the norm's, the gradient of x and of the residual
    alike; dweight (fp32 [dim]) where there is a weight, dbias (fp32 [dim]) with ``bias``, else
    None.  ``out`` (for dx) may be ``dy``, ``x`` or ``dsum`` itself."""
    r = (block._ext or _binding()).layer_norm_backward(dy, x, weight, dsum, eps, rms, bias, out, _handle(dy, stream))
    if stream is not None:
        _made(stream, *(r if out is None else r[1:]))
    return r[:3]


def distill_loss(logits, teacher_logits, teacher_ids, *, teacher_lse=None, temperature: float = 1.0, weights=None,
                 grad: bool = True, out=None, stream=None):
    """Divergence of softmax(logits / temperature) from a teacher of whom each row's
    largest logits are known: ``teacher_logits`` [rows, n] (any of the types) of the tokens
    ``teacher_ids`` (int32 [rows, n]; ids outside the vocabulary: no entry).  The teacher's
    probabilities are the softmax of the listed ones, or with ``teacher_lse`` (fp32 [rows],
    logsumexp of all its logits / temperature, which is held in 32 bits) their true ones, the rest of
    the mass being one outcome.  Returns (loss, gradient): fp32 [rows], and ``weights`` (fp32
    [rows]; 1 if not given) times the loss's gradient of ``logits``, of their type (None without
    ``grad``).  A row of weight 0 has loss and gradient 0, whatever it holds.  ``out`` (the gradient's) may be
    ``logits`` itself."""
    r = (block._ext or _binding()).distill_loss(logits, teacher_logits, teacher_ids, teacher_lse, weights, temperature,
                                                grad, out, _handle(logits, stream))
    if stream is not None:
        _made(stream, *(r if out is None else r[::2]))
    return r[:2]


def sample(logits, uniform, *, temperature=None, top_k=None, top_p=None, min_p=None, return_logprob: bool = False,
           stream=None):
    """A token of each row of ``logits`` [rows, vocab] by the numbers ``uniform`` (fp32
    [rows], in [0, 1)): int32 [rows].  Each rule is a tensor [rows] or None: ``temperature``
    fp32 (1; 0: the largest logit), ``top_k`` int32 (0: all), ``top_p`` fp32 (1: all),
    ``min_p`` fp32 (0: all), applied in this order; equal logits count in the order of their
    numbers.  The token is the first one, by number, at which the kept mass exceeds uniform
    times all of it.  -inf masks a token; a row with NaN or with nothing but masked
    tokens gives -1.  With ``return_logprob`` also the logarithm of the token's share of
    the kept mass (fp32 [rows])."""
    r = (block._ext or _binding()).sample(logits, uniform, temperature, top_k, top_p, min_p, return_logprob,
                                          _handle(logits, stream))
    if stream is not None:
        _made(stream, *r)
    return r[:2] if return_logprob else r[0]
