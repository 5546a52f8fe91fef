"""The operators of ``ends.py`` as a program uses them: refused tensors, streams, graphs,
versions, offsets that 32 bits do not hold, and a step of all of them together."""
import pytest

torch = pytest.importorskip("torch")

import ends_reference as ref  # noqa: E402
from test_gpu_ends import BF16, DEV, F16, F32, aq, distill_case, ids_of, ints, rand, rules, uniform  # noqa: E402,F401

pytestmark = pytest.mark.gpu


def test_refused_tensors(aq):
    x, w, i, u = rand(1, 4, 64), rand(2, 64), ints([0] * 4), uniform(3, 4)
    t, ids = rand(4, 4, 8), torch.zeros(4, 8, dtype=torch.int32, device=DEV)
    bad = [lambda: aq.embed(x.double(), i), lambda: aq.embed(x, i.long()), lambda: aq.embed(x.t(), i),
           lambda: aq.embed(x, i.cpu()), lambda: aq.embed(x[0], i), lambda: aq.embed(x, i.view(2, 2)),
           lambda: aq.embed(x, i, out=x.half()), lambda: aq.embed(x, i, out=x[:3]),
           lambda: aq.embed(x, i, out=x[:, :63]), lambda: aq.embed_backward(x, i[:3], 9),
           lambda: aq.embed_backward(x, i, 0), lambda: aq.embed_backward(x.half(), i, 9, out=rand(1, 9, 64).bfloat16()),
           lambda: aq.embed_backward(x, i, 9, out=rand(1, 8, 64)), lambda: aq.layer_norm(x, w.half()),
           lambda: aq.layer_norm(x, w[:63]), lambda: aq.layer_norm(x, w, w.cpu()), lambda: aq.layer_norm(x[None]),
           lambda: aq.layer_norm(x, residual=x[:3]), lambda: aq.layer_norm(x, residual=x.half()),
           lambda: aq.layer_norm(x, sum_out=x), lambda: aq.layer_norm(x.int()),
           lambda: aq.layer_norm_backward(x, x.half()), lambda: aq.layer_norm_backward(x, x[:, :63]),
           lambda: aq.layer_norm_backward(x, x, dsum=x[:2]), lambda: aq.layer_norm_backward(x, x, w, out=x.t()),
           lambda: aq.distill_loss(x, t, ids.long()), lambda: aq.distill_loss(x, t, ids[:, :7]),
           lambda: aq.distill_loss(x, t[:3], ids[:3]), lambda: aq.distill_loss(x, t.cpu(), ids),
           lambda: aq.distill_loss(x, t, ids, weights=u[:3]), lambda: aq.distill_loss(x, t, ids, teacher_lse=u.double()),
           lambda: aq.distill_loss(x, t, ids, grad=False, out=x), lambda: aq.distill_loss(x, t, ids, out=x.half()),
           lambda: aq.sample(x, u[:3]), lambda: aq.sample(x, u.double()), lambda: aq.sample(x, u, top_k=u),
           lambda: aq.sample(x, u, temperature=i), lambda: aq.sample(x[0], u)]
    for n, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
    shared = torch.empty(1, 64, device=DEV).expand(4, 64)  # rows that share addresses
    refused = [lambda: aq.embed(x, i, out=shared), lambda: aq.embed_backward(x, i, 4, out=shared),
               lambda: aq.layer_norm(x, out=shared), lambda: aq.layer_norm_backward(x, x, out=shared),
               lambda: aq.layer_norm(x, residual=x, out=x, sum_out=x), lambda: aq.layer_norm(rand(1, 1, 16385)),
               lambda: aq.layer_norm(x, eps=-1.0), lambda: aq.distill_loss(x, t, ids, out=shared),
               lambda: aq.distill_loss(x, t, ids, temperature=0.0), lambda: aq.distill_loss(x, t[:, :0], ids[:, :0]),
               lambda: aq.embed_backward(x, i, (1 << 30) + 1)]
    for call in refused:
        with pytest.raises((aq.AqlmError, ValueError)):
            call()


def calls(aq, seed=0, dtype=F16):
    """Each operator with its inputs and the tensors that it may write."""
    rows, dim, vocab = 37, 1032, 5003
    ids = ids_of(seed + 60, rows, vocab)
    table, x, r = rand(seed + 61, vocab, dim, dtype=dtype), rand(seed + 62, rows, dim, dtype=dtype), rand(seed + 63, rows, dim, dtype=dtype)
    w, b = rand(seed + 64, dim, dtype=dtype), rand(seed + 65, dim, dtype=dtype)
    z, t, tid, lse = distill_case(seed + 67, rows, vocab, 20, dtype, F32)
    u, s = uniform(seed + 70, rows), rules(seed + 71, rows)
    flat = lambda *v: [e for e in v if e is not None]  # noqa: E731
    return {"embed": lambda **k: flat(aq.embed(table, ids, scale=3.0, **k)),
            "embed_backward": lambda **k: flat(aq.embed_backward(x, ids, vocab, **k)),
            "layer_norm": lambda **k: flat(*aq.layer_norm(x, w, b, residual=r, **k)),
            "layer_norm_backward": lambda **k: flat(*aq.layer_norm_backward(x, r, w, dsum=r, bias=True, **k)),
            "distill_loss": lambda **k: flat(*aq.distill_loss(z, t, tid, teacher_lse=lse, temperature=1.5, **k)),
            "sample": lambda **k: flat(*aq.sample(z, u, return_logprob=True, **s, **k))}


NAMES = ["embed", "embed_backward", "layer_norm", "layer_norm_backward", "distill_loss", "sample"]


def same(a, b):
    return all(torch.equal(p.nan_to_num(7.0), q.nan_to_num(7.0)) for p, q in zip(a, b))


@pytest.mark.parametrize("name", NAMES)
def test_another_stream(aq, name):
    call = calls(aq)[name]
    want = call()
    side = torch.cuda.Stream()
    for _ in range(3):
        side.wait_stream(torch.cuda.current_stream())
        got = call(stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert same(got, want)
    with torch.cuda.stream(side):
        got = call()
    side.synchronize()
    assert same(got, want)


@pytest.mark.parametrize("name", NAMES)
def test_two_graphs_and_eager_calls(aq, name):
    """Two captured graphs of one operator and eager calls between their replays, on one stream and
    beside one another."""
    a, b = calls(aq, 0)[name], calls(aq, 100)[name]
    want = a(), b()
    torch.cuda.synchronize()
    graphs, outs = [], []
    for call in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(call())
        graphs.append(g)
    side = torch.cuda.Stream()
    for turn in range(6):
        for o in outs[0] + outs[1]:
            o.zero_()
        if turn % 2:
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                graphs[1].replay()
            graphs[0].replay()
            eager = a()
            torch.cuda.current_stream().wait_stream(side)
        else:
            graphs[0].replay()
            eager = a()
            graphs[1].replay()
        torch.cuda.synchronize()
        assert same(outs[0], want[0]) and same(outs[1], want[1]) and same(eager, want[0])


def test_many_calls_at_once(aq):
    """Calls of several sizes on several streams, without waiting between them."""
    streams = [torch.cuda.Stream() for _ in range(3)]
    sets = [calls(aq, 200 + i) for i in range(3)]
    want = [{n: c() for n, c in s.items()} for s in sets]
    torch.cuda.synchronize()
    got = []
    for turn in range(4):
        for i, st in enumerate(streams):
            for n in NAMES:
                with torch.cuda.stream(st):
                    got.append((i, n, sets[i][n]()))
    torch.cuda.synchronize()
    for i, n, v in got:
        assert same(v, want[i][n]), (i, n)


def test_written_tensors_count_as_modified(aq):
    x, w, ids, u = rand(1, 3, 64), rand(2, 64), ints([0, 1, 2]), uniform(3, 3)
    t, tid = rand(4, 3, 8), ints([[0, 1, 2, 3, 4, 5, 6, 7]] * 3)
    o, s, v = torch.empty_like(x), torch.empty_like(x), torch.empty(5, 64, device=DEV)
    for call, changed, kept in (
            (lambda: aq.embed(x, ids, out=o), (o,), (x, ids)),
            (lambda: aq.embed_backward(x, ids, 5, out=v), (v,), (x, ids)),
            (lambda: aq.layer_norm(x, w, residual=x, out=o, sum_out=s), (o, s), (x, w)),
            (lambda: aq.layer_norm_backward(x, x, w, out=o), (o,), (x, w)),
            (lambda: aq.distill_loss(x, t, tid, out=o), (o,), (x, t, tid)),
            (lambda: aq.sample(x, u), (), (x, u))):
        before = [[e._version for e in es] for es in (changed, kept)]
        call()
        assert all(e._version > n for e, n in zip(changed, before[0]))
        assert all(e._version == n for e, n in zip(kept, before[1]))
    with torch.inference_mode():
        y = torch.empty(3, 64, device=DEV)
        aq.layer_norm(x, w, out=y)
        assert torch.equal(y, aq.layer_norm(x, w))


def test_offsets_past_32_bits(aq):
    """Rows whose offsets in elements, and in bytes, 32 bits do not hold."""
    far, n = (1 << 32) + 8, 2000
    big = torch.empty(2 * far + n, dtype=F16, device=DEV)
    rows = big.as_strided((3, n), (far, 1))
    x = rand(80, 3, n, dtype=F16)
    rows.copy_(x)
    ids, u = ints([2, 0, 1]), uniform(81, 3)
    assert torch.equal(aq.embed(rows, ids), x[ids.long()])
    assert torch.equal(aq.layer_norm(rows), aq.layer_norm(x))
    a, b = aq.layer_norm_backward(rows, rows, x[0], bias=True), aq.layer_norm_backward(x, x, x[0], bias=True)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    assert torch.equal(aq.sample(rows, u), aq.sample(x, u))
    t, tid = torch.topk(x, 9)
    a, b = aq.distill_loss(rows, t, tid.int()), aq.distill_loss(x, t, tid.int())
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert torch.equal(aq.embed_backward(rows, ids, 5), aq.embed_backward(x, ids, 5))
    for call in (lambda o: aq.embed(x, ids, out=o), lambda o: aq.layer_norm(x, out=o),
                 lambda o: aq.layer_norm_backward(x, x, out=o)[0], lambda o: aq.distill_loss(x, t, tid.int(), out=o)[1],
                 lambda o: aq.embed_backward(x, ids, 3, out=o)):
        want = call(None)
        rows.zero_()
        call(rows)
        assert torch.equal(rows, want)


def test_many_rows(aq):
    """More rows than a launch has workgroups of one row."""
    n = (1 << 20) + 77
    x = rand(82, n, 8, dtype=F16)
    y = aq.layer_norm(x, rms=True)
    assert torch.equal(y[-100:], aq.layer_norm(x[-100:].clone(), rms=True))
    dx, _, db = aq.layer_norm_backward(x, x, rms=True, bias=True)
    assert torch.equal(dx[-100:], aq.layer_norm_backward(x[-100:].clone(), x[-100:].clone(), rms=True)[0])
    wide = rand(83, n // 4, 32)
    assert torch.equal(aq.sample(wide, uniform(84, n // 4))[-50:], aq.sample(wide[-50:].clone(), uniform(84, n // 4)[-50:].clone()))
    ids = (torch.arange(n, device=DEV) % 1000).int()
    assert torch.equal(aq.embed(x[:1000], ids)[-2000:], x[ids[-2000:].long()])
    want, off = ref.embed_grad(x, ids, 1000, 1.0)
    ref.check(aq.embed_backward(x, ids, 1000, fp32=True), want, off + ref.rounded(want.abs() + off, F32))


def test_step_and_gradients_together(aq):
    """Token ids to drawn tokens, and the gradients back to the table, as one model's ends: against
    automatic differentiation in 64 bits."""
    g = torch.Generator(device=DEV).manual_seed(90)
    vocab, dim, rows = 300, 128, 21
    table = torch.randn(vocab, dim, generator=g, device=DEV) * 0.05
    head = torch.randn(vocab, dim, generator=g, device=DEV) * 0.2
    w = 1 + 0.1 * torch.randn(dim, generator=g, device=DEV)
    ids = ids_of(91, rows, vocab)
    teacher = torch.randn(rows, vocab, generator=g, device=DEV) * 2
    top, tid = torch.topk(teacher, 16)
    lse = torch.logsumexp(teacher, 1)
    weights = torch.full((rows,), 1.0 / rows, device=DEV)
    weights[ids < 0] = 0

    e = aq.embed(table, ids, scale=8.0)
    a, h = aq.layer_norm(e, w, residual=e.flip(0).contiguous(), rms=True)
    z = a @ head.t()
    loss, dz = aq.distill_loss(z, top, tid.int(), teacher_lse=lse, weights=weights)
    dh, dw, _ = aq.layer_norm_backward(dz @ head, h, w, rms=True)
    de = dh + dh.flip(0)
    dt = aq.embed_backward(de.contiguous(), ids, vocab, scale=8.0)
    token = aq.sample(z, uniform(92, rows), top_k=ints([10] * rows))

    T, W = table.double().requires_grad_(), w.double().requires_grad_()
    held = ((ids >= 0) & (ids < vocab))[:, None]
    E = torch.where(held, T[ids.long().clamp(0, vocab - 1)] * 8.0, 0.0)
    H = E + E.flip(0)
    Z = (H * (H.square().mean(1, keepdim=True) + 1e-5).rsqrt() * W) @ head.double().t()
    lq, lp = torch.log_softmax(Z, 1), top.double() - lse.double()[:, None]
    outside = torch.ones(rows, vocab, device=DEV).scatter_(1, tid, 0.0).bool()
    pr = 1 - lp.exp().sum(1)
    L = (lp.exp() * (lp - lq.gather(1, tid))).sum(1) + pr * (pr.log() - lq.masked_fill(~outside, -torch.inf).logsumexp(1))
    (L * weights.double()).sum().backward()
    # (products of 128 and of 300 terms in 32 bits between: 1e-5 of the largest)
    live = weights != 0
    for got, want in ((loss[live], L.detach()[live]), (dt, T.grad), (dw, W.grad)):
        assert (got.double() - want).abs().max() <= 1e-5 * want.abs().max()
    for i in range(rows):
        assert int(token[i]) in torch.topk(z[i], 10).indices.tolist()


@pytest.fixture(scope="module")
def example():
    import importlib.util
    import os

    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "generate.py")
    spec = importlib.util.spec_from_file_location("generate_example_ends", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_example_draws(aq, example):
    """Drawn continuations: the same for the same seed, allowed tokens only, the greedy one at a temperature of 0."""
    model = example.Model()
    prompts = [[5, 7, 11], [13], [1] * 40]
    a, b = (example.generate(model, prompts, 6, temperature=0.9, top_p=0.95, seed=4) for _ in range(2))
    assert torch.equal(a, b) and (a >= 0).all() and (a < model.vocab).all()
    allowed = torch.zeros(1, -(-model.vocab // 32), dtype=torch.int32, device=DEV)
    allowed[0, 3] = 0x0F0F
    out = example.generate(model, prompts, 4, allowed=allowed, temperature=1.5)
    assert all(96 <= t < 112 and (0x0F0F >> (t - 96)) & 1 for t in out.flatten().tolist())
    assert torch.equal(example.generate(model, prompts, 3), example.generate(model, prompts, 3, seed=9))


def test_example_end_gradients(aq, example):
    """The gradients of the example's step against automatic differentiation in 64 bits."""
    model = example.Model(layers=1, hidden=128, vocab=500)
    ids = ids_of(95, 33, 500)
    w = (1 + 0.1 * rand(96, 128)).half()
    teacher = rand(97, 33, 500) * 2
    top, tid = torch.topk(teacher, 12)
    lse = torch.logsumexp(teacher, 1)
    loss, de, dw, dhead = example.end_gradients(model, ids, w, top, tid.int(), lse, loss_scale=1024.0)
    E, W, H = (t.double().requires_grad_() for t in (model.embedding, w, model.head))
    held = ((ids >= 0) & (ids < 500))[:, None]
    x = torch.where(held, E[ids.long().clamp(0, 499)], 0.0)
    z = (x * (x.square().mean(1, keepdim=True) + example.EPS).rsqrt() * W) @ H.t() / 128 ** 0.5
    lq, lp = torch.log_softmax(z, 1), top.double() - lse.double()[:, None]
    outside = torch.ones(33, 500, device=DEV).scatter_(1, tid, 0.0).bool()
    pr = 1 - lp.exp().sum(1)
    L = (lp.exp() * (lp - lq.gather(1, tid))).sum(1) + pr * (pr.log() - lq.masked_fill(~outside, -torch.inf).logsumexp(1))
    L.mean().backward()
    # about six roundings to fp16 on the way, each of 2^-11 of values of the result's size
    want = L.mean().item()
    assert abs(float(loss) - want) <= 6 * 2.0 ** -11 * want
    for got, want in ((de, E.grad), (dw, W.grad), (dhead, H.grad)):
        assert (got.double() / 1024 - want).norm() <= 6 * 2.0 ** -11 * want.norm()


def test_example_ids_are_indices(aq, example):
    """Continuations are int64, as ids that torch takes as indices."""
    model = example.Model(layers=1)
    out = example.generate(model, [[5, 7], [13]], 2)
    assert out.dtype == torch.int64 and out.shape == (2, 2)
    assert model.embedding.gather(0, out).shape == (2, 2)
