"""The example that runs the operators together: examples/generate.py."""
import importlib.util
import math
import os

import pytest

torch = pytest.importorskip("torch")

import block_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "generate.py")
    spec = importlib.util.spec_from_file_location("generate_example", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def plain_logits(example, model, tokens):
    """Logits after the last token of one sequence, by its whole length at once, in 64 bits
    but for the layers' products, whose weights are the dequantised ones."""
    import paper_2401_06118_amd as aqlm

    weights = [{n: aqlm.dequantize(*b[n].parts).double().cpu() for n in ("qkv", "o", "gate", "up", "down")}
               for b in model.blocks]
    emb, head, table = (t.double().cpu() for t in (model.embedding, model.head, model.table))
    n, pos = len(tokens), torch.arange(len(tokens))
    norm = lambda x: x / (x.pow(2).mean(-1, keepdim=True) + example.EPS).sqrt()  # noqa: E731
    x = emb[tokens]
    one = torch.ones(model.dim, dtype=torch.float64)
    for w in weights:
        qkv = (norm(x) @ w["qkv"].t()).view(n, -1, model.dim)
        q, k, v = qkv.split((model.heads, model.kv, model.kv), 1)
        q, k = (ref.rope64(t, one, table, pos, False, example.EPS)[0] for t in (q, k))
        group = model.heads // model.kv
        s = torch.einsum("ihd,jhd->hij", q, k.repeat_interleave(group, 1)) / model.dim ** 0.5
        s = torch.where(pos[None, :] <= pos[:, None], s, -math.inf)
        a = torch.einsum("hij,jhd->ihd", torch.softmax(s, -1), v.repeat_interleave(group, 1)).flatten(1)
        x = x + a @ w["o"].t()
        h = norm(x)
        x = x + (torch.nn.functional.silu(h @ w["gate"].t()) * (h @ w["up"].t())) @ w["down"].t()
    return norm(x[-1]) @ head.t() / model.hidden ** 0.5


def test_prompt_in_chunks(example):
    """The logits after a prompt do not depend on how it was cut, and are those of a plain model."""
    model = example.Model()
    gen = torch.Generator().manual_seed(3)
    tokens = torch.randint(0, model.vocab, (150,), generator=gen).tolist()
    want = plain_logits(example, model, tokens)
    table = torch.randperm(10, device=DEV).to(torch.int32).view(1, 10)
    for cuts in ((150,), (64, 64, 22), (149, 1), (1, 2, 3, 100, 44)):
        cache, done = model.new_cache(10), 0
        for n in cuts:
            new, done = tokens[done:done + n], done + n
            logits = model.forward(torch.tensor(new, device=DEV), cache, table,
                                   torch.tensor([done], dtype=torch.int32, device=DEV),
                                   torch.tensor([0, n], dtype=torch.int32, device=DEV), n)
        # about twenty roundings to fp16 on the way, of values of the logits' own relative size
        err = (logits[0].double().cpu() - want).norm() / want.norm()
        assert err <= 20 * 2.0 ** -11, (cuts, float(err))


def test_generate(example):
    """Sequences decoded together give what each gives alone; banned and masked tokens do not come."""
    model = example.Model()
    gen = torch.Generator().manual_seed(5)
    prompts = [torch.randint(0, model.vocab, (n,), generator=gen).tolist() for n in (5, 130, 1)]
    free = example.generate(model, prompts, 6, chunk=50)
    assert free.shape == (3, 6) and (free >= 0).all() and (free < model.vocab).all()
    banned = free[:, 0].tolist()
    out = example.generate(model, prompts, 6, chunk=50, banned=banned)
    assert not set(banned) & set(out.flatten().tolist())
    words = -(-model.vocab // 32)
    allowed = torch.zeros(1, words, dtype=torch.int32, device=DEV)
    allowed[0, 3] = 0x0F0F
    out = example.generate(model, prompts, 4, allowed=allowed)
    assert all(96 <= t < 112 and (0x0F0F >> (t - 96)) & 1 for t in out.flatten().tolist())


def test_head_gradients(example):
    """Codebook gradients through rope_backward and backward against differences of the whole in 64 bits."""
    import paper_2401_06118_amd as aqlm

    model = example.Model(layers=1, hidden=128, heads=2, kv=1)
    gen = torch.Generator().manual_seed(2)
    x = torch.randn(9, 128, generator=gen).half().to(DEV)
    dq, dk = (torch.randn(9, n, 64, generator=gen).half().to(DEV) for n in (2, 1))
    pos = torch.arange(9, dtype=torch.int32, device=DEV) * 7
    dcb, ds, gqw, gkw = example.head_gradients(model, 0, x, dq, dk, pos)
    lin = model.blocks[0]["qkv"]
    codes, cb = lin.codes.long().cpu(), lin.codebooks.double().cpu()
    table, one = model.table.double().cpu(), torch.ones(64, dtype=torch.float64)

    def loss(cb):
        w = sum(cb[m][codes[:, :, m]] for m in range(2)).flatten(1)
        y = (x.double().cpu() @ w.t()).view(9, 4, 64)
        q, k = (ref.rope64(t, one, table, pos.long().cpu(), False, example.EPS)[0] for t in (y[:, :2], y[:, 2:3]))
        return float((q * dq.double().cpu()).sum() + (k * dk.double().cpu()).sum())

    big = dcb.abs().max().item()
    for m, e, j in ((0, 3, 1), (1, 200, 7), (0, 77, 4)):
        d = torch.zeros_like(cb)
        d[m, e, j] = 1e-4
        slope = (loss(cb + d) - loss(cb - d)) / 2e-4
        # the heads and their gradients are rounded to fp16 on the way
        assert abs(slope - float(dcb[m, e, j])) <= 4 * 2.0 ** -11 * big
    assert gqw.shape == gkw.shape == (64,) and torch.isfinite(ds).all()
