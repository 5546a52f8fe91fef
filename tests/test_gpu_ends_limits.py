"""The operators of ``ends.py`` where a quantity of theirs reaches a limit."""
import math

import pytest

torch = pytest.importorskip("torch")

import ends_reference as ref  # noqa: E402
from test_gpu_ends import DEV, F32, TYPES, aq, check_sample, distill_case, rand, uniform  # noqa: E402,F401

pytestmark = pytest.mark.gpu


# --------------------------------------------------------------------------- norms

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [8, 64, 250, 500, 512, 1000, 1024, 2050])
@pytest.mark.parametrize("rms", [True, False])
def test_norm_without_epsilon(aq, dtype, dim, rms):
    """eps = 0, which rows that are not constant allow, for every count of rows in a workgroup."""
    for rows in (1, 2, 3, 4, 5, 6, 7, 8, 9, 1101):
        x = (rand(1, rows, dim) * (0.5 + uniform(2, rows, 1)) + 0.5).to(dtype)
        dy, w, b = rand(3, rows, dim, dtype=dtype), rand(4, dim, dtype=dtype), rand(5, dim, dtype=dtype)
        y, off, *_ = ref.norm(x, w, b, 0.0, rms)
        ref.check(aq.layer_norm(x, w, b, eps=0.0, rms=rms), y, off + ref.rounded(y.abs() + off, dtype), f"y, {rows} rows")
        (dx, dx_off), (dw, dw_off), (db, db_off) = ref.norm_grad(dy, x, w, None, 0.0, rms)
        got = aq.layer_norm_backward(dy, x, w, eps=0.0, rms=rms, bias=True)
        ref.check(got[0], dx, dx_off + ref.rounded(dx.abs() + dx_off, dtype), f"dx, {rows} rows")
        ref.check(got[1], dw, dw_off + ref.rounded(dw, F32), f"dweight, {rows} rows")
        ref.check(got[2], db, db_off + ref.rounded(db, F32), f"dbias, {rows} rows")


# --------------------------------------------------------------------------- sampling

@pytest.mark.parametrize("vocab", [8000, 30000, 128256])
@pytest.mark.parametrize("many", [200, 2000])
@pytest.mark.parametrize("level,temperature", [(100.0, 1e-5), (-100.0, 1e-5), (100.0, 4e-5), (3.0, 1e-6), (1000.0, 1e-4)])
def test_sample_clusters_at_a_low_temperature(aq, vocab, many, level, temperature):
    """Hundreds of equal logits at each of neighbouring 32-bit numbers, many units of the temperature's
    size away from 0: tokens by sixteenths of the temperature are no longer told apart in 32 bits."""
    rows = 4
    step = float(torch.finfo(F32).eps) * 2.0 ** math.floor(math.log2(abs(level)))
    at = torch.stack([torch.randperm(vocab, generator=torch.Generator(device=DEV).manual_seed(i), device=DEV)
                      for i in range(rows)])
    x = torch.full((rows, vocab), level - 1.0, device=DEV)
    for j in range(min(8, vocab // many - 1)):
        x.scatter_(1, at[:, j * many:(j + 1) * many], level - j * step)
    assert (x.unique().numel()) == min(8, vocab // many - 1) + 1
    x[3] = torch.where(x[3] == level, -math.inf, x[3])
    u, full = uniform(6, rows), lambda v, t=F32: torch.full((rows,), v, dtype=t, device=DEV)  # noqa: E731
    for r in (dict(), dict(top_p=full(0.3)), dict(top_p=full(0.9)), dict(top_p=full(0.999)), dict(min_p=full(0.3)),
              dict(min_p=full(0.001)), dict(top_k=full(150, torch.int32)), dict(top_k=full(300, torch.int32)),
              dict(top_k=full(300, torch.int32), top_p=full(0.9)), dict(top_k=full(2500, torch.int32)),
              dict(top_k=full(2500, torch.int32), top_p=full(0.9), min_p=full(0.2))):
        check_sample(aq, x, u, temperature=full(temperature), **r)


@pytest.mark.parametrize("level", [0.0, -1.0 / 512, 3.0, -250.0])
def test_sample_parts_of_a_bin(aq, level):
    """A bin of thousands of tokens that is divided into 512 parts, many of the tokens just below a part's end; also
    where that is 0, and 32 bits are finer than next to the bin's other end."""
    vocab, t = 40000, 16.0  # (bins of one unit)
    gen = torch.Generator(device=DEV).manual_seed(8)
    at = torch.randperm(vocab, generator=gen, device=DEV)
    below = torch.tensor([-1e-9 * 2.0 ** j for j in range(8)], device=DEV)
    x = torch.full((vocab,), -math.inf, device=DEV)
    x[at[:100]] = level + 0.5
    x[at[100:1700]] = torch.minimum(level + below.repeat(200), torch.tensor(level, device=DEV).nextafter(torch.tensor(-math.inf, device=DEV)))
    x[at[1700:3300]] = level - 0.25 + below.repeat(200)
    x[at[3300:5000]] = level - 0.9 + 0.8 * torch.rand(1700, generator=gen, device=DEV)
    rows = 16
    u, full = uniform(9, rows), lambda v, t=F32: torch.full((rows,), v, dtype=t, device=DEV)  # noqa: E731
    for r in (dict(top_p=full(0.1)), dict(top_p=full(0.2)), dict(top_p=full(0.335)), dict(top_p=full(0.5)),
              dict(top_p=full(0.9)), dict(top_k=full(1000, torch.int32)), dict(top_k=full(1701, torch.int32)),
              dict(top_k=full(4000, torch.int32), top_p=full(0.5)), dict(min_p=full(0.955)), dict(min_p=full(0.96))):
        check_sample(aq, x.expand(rows, vocab), u, temperature=full(t), **r)


def test_sample_bin_of_more_tokens_than_its_place_holds(aq):
    """A bin of 9400 tokens of which the slices' masses show fewer: each weighs 1.4 units of 2^-44 of
    the largest, which the slice with the largest logit counts as 1."""
    vocab, tail_last, tail_first = 32768, 7600, 1800
    gen = torch.Generator(device=DEV).manual_seed(7)
    x = torch.full((vocab,), -math.inf, device=DEV)
    last = 24576 + torch.randperm(8191, generator=gen, device=DEV)[:tail_last]
    first = torch.randperm(24576, generator=gen, device=DEV)[:tail_first]
    tail = torch.cat([first, last])
    # l in (-30.1875, -30.125): exp(l) 2^44 lies between 1.36 and 1.45
    x[tail] = -30.1874 + 0.0623 * torch.rand(len(tail), generator=gen, device=DEV)
    x[vocab - 1] = 0.0
    least = torch.tensor(math.exp(-30.15), dtype=F32, device=DEV)
    kept = tail[x[tail].double() >= math.log(float(least))].sort().values
    assert 3600 < len(kept) < 3900
    w = torch.exp(x[kept].double()) * 2.0 ** 44
    assert 1.3 < float(w.min()) and float(w.max()) < 1.5  # (so each is one unit)
    j = torch.tensor([0, 1, 500, 700, 1000, 1100, 2000, 3000, 3500, len(kept) - 1], device=DEV)
    # the number of unit j, half a unit on: total is 2^44 (1 + 2^-31)
    u = ((j.double() + 0.5) * 2.0 ** -44).float()
    rows = x.expand(len(j), vocab)
    full = least.expand(len(j)).contiguous()
    for _ in range(3):
        assert torch.equal(aq.sample(rows, u, min_p=full), kept[j].int())


@pytest.mark.parametrize("vocab", [8192, 8193, 32000, 32768, 50001])
def test_sample_a_top_k_of_others(aq, vocab):
    """Rows without top-k among requests of which some bring one: summed up differently, drawn alike."""
    x, u = rand(10, 12, vocab) * 2.5, uniform(11, 12)
    zeros = torch.zeros(12, dtype=torch.int32, device=DEV)
    for r in (dict(), dict(top_p=torch.full((12,), 0.9, device=DEV)), dict(min_p=torch.full((12,), 0.05, device=DEV))):
        assert torch.equal(check_sample(aq, x, u, **r), check_sample(aq, x, u, top_k=zeros, **r))


# --------------------------------------------------------------------------- distillation

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("copies", [1, 300])  # (rows that are cut, and not)
@pytest.mark.parametrize("vocab", [40, 5000])
def test_distill_rest_far_below_the_list(aq, dtype, copies, vocab):
    """What is not listed masked with finite numbers, so low that its mass is no number of 64 bits: the
    loss is that mass's logarithm all the same."""
    n, tau = 30, 1.5
    lows = [-1e4, float(torch.finfo(dtype).min), -2000.0, -1100.0]
    z, t, ids, lse = distill_case(37, len(lows), vocab, n, dtype, F32, short=False)
    at = ids.long()
    listed = torch.zeros_like(z, dtype=torch.bool).scatter_(1, at, True)
    z = torch.where(listed, z, torch.tensor(lows, dtype=dtype, device=DEV)[:, None])
    lse = lse + 0.1
    many = [v.repeat(copies, *[1] * (v.dim() - 1)) for v in (z, t, ids, lse)]
    loss, g = (v[-len(lows):] for v in aq.distill_loss(*many[:3], teacher_lse=many[3], temperature=tau))
    p = (t.double() / tau - lse.double()[:, None]).exp()
    rest = 1 - p.sum(1)
    assert (rest > 0.05).all()
    zl = z.double().gather(1, at) / tau
    log_all = torch.logsumexp(zl, 1)  # (the rest adds nothing to it)
    low = z[~listed].double().view(len(lows), -1)[:, 0] / tau
    log_rest = low + math.log(vocab - n) - log_all
    want = (p * (p.log() - zl + log_all[:, None])).sum(1) + rest * (rest.log() - log_rest)
    # the rest's sum in 32 bits: 128 additions of a thread, 17 waves' parts; then one rounding
    ref.check(loss, want, want.abs() * 2 * ref.E32 + (128 + 17 + 8) * ref.E32)
    assert torch.isfinite(g).all()
    grad = torch.where(listed, 0.0, (-rest / (vocab - n))[:, None])
    grad.scatter_(1, at, (zl - log_all[:, None]).exp() - p)
    size = torch.where(listed, 0.0, (rest / (vocab - n))[:, None]).scatter_(1, at, (zl - log_all[:, None]).exp() + p)
    bound = size / tau * (128 + 17 + 8) * ref.E32
    ref.check(g, grad / tau, bound + ref.rounded(grad.abs() / tau + bound, dtype))


@pytest.mark.parametrize("copies", [1, 600])
@pytest.mark.parametrize("rest", [False, True])
def test_distill_all_masked(aq, copies, rest):
    """A student's row of nothing but -inf has no softmax: loss and gradient are NaN, all of it."""
    z, t, ids, lse = distill_case(38, 3, 700, 20, F32, F32, short=False)
    z[1] = -math.inf
    many = [v.repeat(copies, *[1] * (v.dim() - 1)) for v in (z, t, ids, lse)]
    loss, g = aq.distill_loss(*many[:3], teacher_lse=many[3] if rest else None, temperature=1.5)
    assert torch.isnan(loss[1::3]).all() and torch.isnan(g[1::3]).all()
    assert torch.isfinite(loss[0::3]).all() and torch.isfinite(g[0::3]).all()
    assert torch.isfinite(loss[2::3]).all() and torch.isfinite(g[2::3]).all()
    got, none = aq.distill_loss(z[1:2], t[1:2], ids[1:2], weights=torch.zeros(1, device=DEV))
    assert float(got[0]) == 0 and not none.any()


def test_distill_long_lists_after_short_ones(aq):
    """Lists of 2048, which need more of the processors' memory than a kernel has by itself, before and after
    short ones."""
    for rows, vocab in ((2, 9000), (600, 9000)):
        z, t, ids, lse = distill_case(39, rows, vocab, 2048, F32, F32, short=False)
        want, want_off, grad, grad_off = ref.distill(z[:2], t[:2], ids[:2], None, None, 1.5)
        for n in (2048, 64, 2048, 1, 2048):
            loss, g = aq.distill_loss(z, t[:, :n].contiguous(), ids[:, :n].contiguous(), temperature=1.5)
            if n == 2048:
                ref.check(loss[:2], want, want_off, "loss")
                ref.check(g[:2], grad, grad_off + ref.rounded(grad.abs() + grad_off, F32), "gradient")
