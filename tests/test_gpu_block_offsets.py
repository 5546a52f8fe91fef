"""Offsets of new tokens (``cu_new``) that do not ascend, or leave tokens to no sequence."""
import random

import pytest

torch = pytest.importorskip("torch")

import block_reference as ref  # noqa: E402
from test_gpu_block import DEV, Batch, aq, rand, within  # noqa: E402,F401

pytestmark = pytest.mark.gpu


def claims(cu, tokens):
    """(first, count) of each sequence: a token is the first sequence's that claims it."""
    out, end = [], 0
    for a, b in zip(cu, cu[1:]):
        a = min(max(a, 0), tokens)
        b = min(max(b, a), tokens)
        first = max(a, end)
        out.append((first, max(b - first, 0)))
        end = max(end, b)
    return out


def call_with(aq, cu, lens, tokens, heads=4, kv=2, dim=64, dtype=torch.float16):
    """Outputs through both kernels, those of the definition, and which tokens a sequence holds."""
    bt = Batch(lens, [0] * len(lens), kv, dim, 16, dtype)
    bt.cu = torch.tensor(cu, dtype=torch.int32)
    q = rand(2, tokens, heads, dim, dtype=dtype, scale=1.5)
    want, size = (torch.zeros(tokens, heads, dim, dtype=torch.float64) for _ in range(2))
    score = torch.zeros(tokens, heads, 1, dtype=torch.float64)
    lse = torch.full((tokens, heads), -float("inf"), dtype=torch.float64)
    held = torch.zeros(tokens, dtype=torch.bool)
    for b, (first, count) in enumerate(claims(cu, tokens)):
        at = slice(first, first + count)
        assert not held[at].any()
        held[at] = True
        want[at], size[at], score[at], lse[at] = ref.attend64(
            q[at], bt.k, bt.v, bt.table[b:b + 1], lens[b:b + 1], torch.tensor([0, count]), dim ** -0.5, True, 0)
    gots = [aq.paged_attention(q.to(DEV), *bt.gpu(), max_new=most, return_lse=True) for most in (1, 0)]
    return gots, want, ref.attend_bound(dtype, want, size, score), lse, score, held


def some_offsets(seed, seqs, tokens):
    r = random.Random(seed)
    return [r.randint(-3, tokens + 3) for _ in range(seqs + 1)]


FALLING = [
    ([0, 6, 0, 6], [40, 90, 33], 6),
    ([0, 1, 2, 3, 0, 0, 0], [70, 20, 300, 0, 0, 0], 3),     # empty slots at the end, their offsets never written
    ([5, 2, 9, 1, 12], [60, 50, 40, 30], 12),
    ([0, 200, 0, 200, 7, 90], [250, 300, 210, 100, 64], 200),
    (some_offsets(1, 150, 90), [30 + 7 * i % 120 for i in range(150)], 90),
    (some_offsets(2, 70, 600), [90 + 7 * i % 200 for i in range(70)], 600),
]


@pytest.mark.parametrize("cu,lens,tokens", FALLING)
def test_attention_falling_offsets(aq, cu, lens, tokens):
    """A token that several sequences claim is the first one's; every held token's row is right."""
    gots, want, bound, lse, score, held = call_with(aq, cu, lens, tokens)
    for got, got_lse in gots:
        within(got[held.to(DEV)], want[held], bound[held], "out")
        within(got_lse[held.to(DEV)], lse[held],
               (2.0 ** -19 * (score[..., 0] + lse.abs().nan_to_num(0.0, 0.0, 0.0) + 2))[held], "lse")


UNHELD = [
    ([0, 3, 5], [40, 90], 9),              # a padded batch: tokens behind the last sequence's
    ([2, 6, 8], [40, 90], 10),             # and before the first one's
    ([0, 0], [50], 4),                     # none held
    ([9, 9, 9], [50, 20], 20),
    ([0, 60, 100], [300, 90], 131),
    ([5, 1, -7], [50, 20], 12),
]


@pytest.mark.parametrize("cu,lens,tokens,dim", [(*c, 64) for c in UNHELD + FALLING] + [(*c, 200) for c in UNHELD])
def test_attention_tokens_of_no_sequence(aq, cu, lens, tokens, dim):
    """Rows that no sequence holds are zeros, their lse -inf, whatever was there before."""
    # (freed memory that new outputs may come from holds NaN)
    junk = [torch.full((tokens, 4, dim), float("nan"), dtype=torch.float16, device=DEV) for _ in range(4)]
    del junk
    gots, want, bound, lse, score, held = call_with(aq, cu, lens, tokens, dim=dim)
    tol = 2.0 ** -19 * (score[..., 0] + lse.abs().nan_to_num(0.0, 0.0, 0.0) + 2)
    for got, got_lse in gots:
        assert (got[~held.to(DEV)] == 0).all() and (got_lse[~held.to(DEV)] == -float("inf")).all()
        within(got, want, bound, "out")
        within(got_lse, lse, tol, "lse")


def test_padded_batch_in_a_graph(aq):
    """One captured call for up to 6 tokens serves fewer: the others' rows are zeros in every replay."""
    bt = Batch([40, 90, 33], [1, 1, 4], 2, 64, 16, torch.float16)
    q = rand(2, 6, 4, 64).to(DEV)
    k, v, table, lens, cu = bt.gpu()
    out = torch.empty(6, 4, 64, dtype=torch.float16, device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        aq.paged_attention(q, k, v, table, lens, cu, out=out)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        aq.paged_attention(q, k, v, table, lens, cu, out=out)
    for ends in ((1, 2, 6), (1, 2, 3), (0, 0, 0), (2, 2, 5)):
        cu.copy_(torch.tensor((0,) + ends, dtype=torch.int32))
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert (out[ends[-1]:] == 0).all() and torch.isfinite(out).all()
        assert torch.equal(out, aq.paged_attention(q, k, v, table, lens, cu))
