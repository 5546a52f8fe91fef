"""The operators of ``ends.py`` on the GPU against their definitions in 64 bits."""
import math

import pytest

torch = pytest.importorskip("torch")

import ends_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda"
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
TYPES = [F16, BF16, F32]


@pytest.fixture(scope="module")
def aq():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    import paper_2401_06118_amd as aq

    return aq


def rand(seed, *shape, dtype=F32):
    return torch.randn(*shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(dtype)


def uniform(seed, *shape):
    return torch.rand(*shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV)


def ints(v):
    return torch.as_tensor(v, dtype=torch.int32, device=DEV)


def spaced(x, extra=3, first=1):
    """The same rows, `extra` elements apart, from an odd element's address on."""
    rows, n = x.shape
    big = torch.full((rows * (n + extra) + first,), float("nan"), dtype=x.dtype, device=x.device)
    view = big[first:].as_strided((rows, n), (n + extra, 1), first)
    view.copy_(x)
    return view


def around(view):
    """Elements of a spaced() tensor's memory outside its rows."""
    rows, n = view.shape
    s = view.stride(0)
    whole = torch.empty(0, dtype=view.dtype, device=view.device).set_(view.untyped_storage())
    mark = torch.ones_like(whole, dtype=torch.bool)
    for r in range(rows):
        mark[view.storage_offset() + r * s:view.storage_offset() + r * s + n] = False
    return whole[mark]


# --------------------------------------------------------------------------- embedding

def ids_of(seed, n, vocab, pad=0.2):
    u = uniform(seed, n)
    ids = (vocab ** u - 1).to(torch.int32).clamp(0, vocab - 1)
    out = uniform(seed + 1, n)
    ids = torch.where(out < pad / 2, -1, ids)
    return torch.where(out > 1 - pad / 2, vocab, ids)  # (both ends of the table)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,vocab,dim", [(1, 1, 1), (1, 300, 4096), (7, 50, 33), (130, 1000, 2056), (65, 70, 5120)])
def test_embed(aq, dtype, tokens, vocab, dim):
    table, ids = rand(1, vocab, dim, dtype=dtype), ids_of(2, tokens, vocab)
    for scale in (1.0, 71.5, -0.3):
        want = ref.embed(table, ids, scale)
        got = aq.embed(table, ids, scale=scale)
        assert got.dtype == dtype and got.shape == (tokens, dim)
        ref.check(got, want, ref.rounded(want, dtype) + 2 * ref.E32 * want.abs())
        out = spaced(torch.zeros(tokens, dim, dtype=dtype, device=DEV))
        assert aq.embed(spaced(table), ids, scale=scale, out=out) is not None
        assert torch.equal(out, got) and torch.isnan(around(out)).all()
    assert torch.equal(aq.embed(table, ids), ref.embed(table, ids, 1.0).to(dtype))


def test_embed_no_tokens(aq):
    assert aq.embed(rand(1, 5, 8), ints([])).shape == (0, 8)
    for dtype, fp32 in ((F16, False), (F32, False), (BF16, True)):
        g = aq.embed_backward(rand(1, 0, 9, dtype=dtype), ints([]), 13, fp32=fp32)
        assert g.shape == (13, 9) and not g.any() and g.dtype == (F32 if fp32 else dtype)


@pytest.mark.parametrize("dtype,fp32", [(F16, False), (BF16, False), (F32, False), (F16, True), (BF16, True)])
@pytest.mark.parametrize("tokens,vocab,dim", [(1, 1, 1), (3, 700, 40), (16, 5, 33), (17, 5, 4100), (400, 1000, 264),
                                             (1999, 130000, 8), (5000, 37, 70)])
def test_embed_backward(aq, dtype, fp32, tokens, vocab, dim):
    dout, ids = rand(3, tokens, dim, dtype=dtype), ids_of(4, tokens, vocab)
    want, off = ref.embed_grad(dout, ids, vocab, 2.5)
    got = aq.embed_backward(dout, ids, vocab, scale=2.5, fp32=fp32)
    out_type = F32 if fp32 else dtype
    assert got.dtype == out_type
    ref.check(got, want, off + ref.rounded(want.abs() + off, out_type))
    out = spaced(torch.zeros(vocab, dim, dtype=out_type, device=DEV))
    aq.embed_backward(spaced(dout), ids, vocab, scale=2.5, out=out)
    assert torch.equal(out, got) and torch.isnan(around(out)).all()


@pytest.mark.parametrize("ids", ["one", "two", "runs", "none"])
def test_embed_backward_long_runs(aq, ids):
    """Tokens whose places reach over many workgroups, begin and end anywhere in them."""
    n, vocab, dim = 3001, 600, 2100
    ids = {"one": ints([5] * n), "two": ints([5] * 1500 + [599] * 1501)[torch.randperm(n, device=DEV)],
           "runs": ints([i // 31 for i in range(n)]), "none": ints([-1, 600, 1 << 30] * 1001)[:n]}[ids]
    dout = rand(5, n, dim, dtype=BF16)
    want, off = ref.embed_grad(dout, ids, vocab, 1.0)
    got = aq.embed_backward(dout, ids, vocab, fp32=True)
    ref.check(got, want, off + ref.rounded(want.abs() + off, F32))
    for _ in range(3):
        assert torch.equal(aq.embed_backward(dout, ids, vocab, fp32=True), got)


def test_embed_gradient_is_the_adjoint(aq):
    """<embed(E), y> = <E, embed_backward(y)>, and differences of a function of one element."""
    table, ids = rand(6, 40, 24), ids_of(7, 90, 40)
    y = rand(8, 90, 24)
    g = aq.embed_backward(y, ids, 40, scale=0.5)
    a = (aq.embed(table, ids, scale=0.5).double() * y).sum()
    b = (table.double() * g).sum()
    assert abs(a - b) <= 1e-5 * (table.double().abs() * g.double().abs()).sum()


# --------------------------------------------------------------------------- norms

DIMS = [1, 7, 33, 64, 398, 520, 1025, 2048, 4096, 4100, 5120, 8192, 16384]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("rms", [True, False])
def test_layer_norm(aq, dtype, dim, rms):
    rows = 5
    x = (rand(9, rows, dim) * torch.tensor([1.0, 30.0, 0.01, 3.0, 1.0], device=DEV)[:, None] + 2.0).to(dtype)
    r, w, b = rand(10, rows, dim, dtype=dtype), rand(11, dim, dtype=dtype), rand(12, dim, dtype=dtype)
    for weight, bias, residual in ((w, None, None), (w, b, r), (None, None, r), (None, b, None)):
        h = x if residual is None else (x.float() + residual.float()).to(dtype)
        want, off, *_ = ref.norm(h, weight, bias, 1e-5, rms)
        got = aq.layer_norm(x, weight, bias, residual=residual, rms=rms)
        if residual is not None:
            got, s = got
            assert torch.equal(s, h)
        ref.check(got, want, off + ref.rounded(want.abs() + off, dtype))
    # rows apart, in place: the sum into x, the result into the residual
    xs, rs = spaced(x), spaced(r)
    y, s = aq.layer_norm(xs, w, b, residual=rs, rms=rms, out=rs, sum_out=xs)
    a = aq.layer_norm(x, w, b, residual=r, rms=rms)
    assert torch.equal(rs, a[0]) and torch.equal(xs, a[1])
    assert torch.isnan(around(xs)).all() and torch.isnan(around(rs)).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("rms", [True, False])
def test_layer_norm_backward(aq, dtype, dim, rms):
    rows = 6 if dim > 64 else 2500
    x = (rand(13, rows, dim) * (0.5 + uniform(14, rows, 1)) + 0.5).to(dtype)
    dy, ds, w = rand(15, rows, dim, dtype=dtype), rand(16, rows, dim, dtype=dtype), rand(17, dim, dtype=dtype)
    for weight, dsum, bias in ((w, None, True), (w, ds, False), (None, ds, True), (None, None, False)):
        (dx, dx_off), (dw, dw_off), (db, db_off) = ref.norm_grad(dy, x, weight, dsum, 1e-5, rms)
        got = aq.layer_norm_backward(dy, x, weight, dsum=dsum, rms=rms, bias=bias)
        ref.check(got[0], dx, dx_off + ref.rounded(dx.abs() + dx_off, dtype), "dx")
        assert (got[1] is None) == (weight is None) and (got[2] is None) == (not bias)
        if weight is not None:
            ref.check(got[1], dw, dw_off + ref.rounded(dw, F32), "dweight")
        if bias:
            ref.check(got[2], db, db_off + ref.rounded(db, F32), "dbias")
    a = aq.layer_norm_backward(dy, x, w, dsum=ds, rms=rms, bias=True)
    for which in range(3):  # rows apart; the gradient over each of its inputs
        t = [spaced(v) for v in (dy, x, ds)]
        g = aq.layer_norm_backward(t[0], t[1], w, dsum=t[2], rms=rms, bias=True, out=t[which])
        assert all(torch.equal(p, q) for p, q in zip(a, g)) and torch.equal(t[which], a[0])
        assert torch.isnan(around(t[which])).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [500, 1000, 2056, 4100, 5120, 8199, 12296, 16384])
def test_layer_norm_backward_many_rows(aq, dtype, dim):
    """More rows than workgroups: each takes several, some one more than others."""
    rows = 1101
    x = (rand(18, rows, dim) * (0.5 + uniform(19, rows, 1)) + 0.5).to(dtype)
    dy, w = rand(20, rows, dim, dtype=dtype), rand(21, dim, dtype=dtype)
    for dsum, rms in ((None, False), (x, True)):
        (dx, dx_off), (dw, dw_off), (db, db_off) = ref.norm_grad(dy, x, w, dsum, 1e-5, rms)
        got = aq.layer_norm_backward(dy, x, w, dsum=dsum, rms=rms, bias=True)
        ref.check(got[0], dx, dx_off + ref.rounded(dx.abs() + dx_off, dtype), "dx")
        ref.check(got[1], dw, dw_off + ref.rounded(dw, F32), "dweight")
        ref.check(got[2], db, db_off + ref.rounded(db, F32), "dbias")
        again = aq.layer_norm_backward(dy, x, w, dsum=dsum, rms=rms, bias=True)
        assert all(torch.equal(p, q) for p, q in zip(got, again))


def test_norm_no_rows(aq):
    x = rand(1, 0, 100)
    w = rand(2, 100)
    assert aq.layer_norm(x, w).shape == (0, 100)
    dx, dw, db = aq.layer_norm_backward(x, x, w, bias=True)
    assert dx.shape == (0, 100) and not dw.any() and not db.any()


@pytest.mark.parametrize("rms", [True, False])
def test_norm_gradient_by_differences(aq, rms):
    x, w, b, dy = (rand(20 + i, *s) for i, s in enumerate([(3, 50), (50,), (50,), (3, 50)]))
    dx, dw, db = aq.layer_norm_backward(dy, x, w, rms=rms, bias=True)

    def f(x, w, b):
        return (ref.norm(x, w, b, 1e-5, rms)[0] * dy.double()).sum()

    x, w, b = x.double(), w.double(), b.double()
    step = 1e-5
    for i in (0, 17, 49):
        e = torch.zeros(50, dtype=torch.float64, device=DEV)
        e[i] = step
        d = torch.zeros(3, 50, dtype=torch.float64, device=DEV)
        d[1, i] = step
        # (differences are off by step^2 and 1e-16 / step; the gradient by its roundings: 1e-5 holds both)
        for got, hi, lo in ((dx[1, i], f(x + d, w, b), f(x - d, w, b)), (dw[i], f(x, w + e, b), f(x, w - e, b)),
                            (db[i], f(x, w, b + e), f(x, w, b - e))):
            assert abs(float(got) - float((hi - lo) / (2 * step))) <= 1e-5 * (1 + abs(float(got)))


def test_norm_special_values(aq):
    """Rows of zeros, large means, infinities and NaN stay in their rows."""
    x = rand(30, 6, 300)
    x[0] = 0
    x[1] = 1000 + 0.25 * x[1]
    x[2, 5] = math.inf
    x[3, 7] = math.nan
    x[4] = 3.0
    for rms in (True, False):
        y = aq.layer_norm(x, rms=rms)
        want, off, *_ = ref.norm(x, None, None, 1e-5, rms)
        for i in (0, 1, 4, 5):
            ref.check(y[i], want[i], off[i] + ref.rounded(want[i].abs() + off[i], F32))
        assert not torch.isfinite(y[2]).all() and torch.isnan(y[3]).all()
        assert not torch.isnan(y[[0, 1, 4, 5]]).any()


# --------------------------------------------------------------------------- distillation

def distill_case(seed, rows, vocab, n, dtype, teacher_type, short=True):
    z = rand(seed, rows, vocab) * 2.5
    t, ids = torch.topk(z, n, dim=1)
    lse = torch.logsumexp(z.double() / 1.5, 1).float()
    if short and rows > 2:
        keep = (uniform(seed + 1, rows, 1) * n).long() + 1
        keep[2] = 0
        ids = torch.where(torch.arange(n, device=DEV) < keep, ids, -1 if seed % 2 else vocab)
    return (z + rand(seed + 2, rows, vocab)).to(dtype), t.to(teacher_type), ids.to(torch.int32).contiguous(), lse


@pytest.mark.parametrize("dtype,teacher", [(F16, F16), (BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("rows,vocab,n", [(1, 1, 1), (3, 5, 5), (4, 33, 7), (6, 1000, 999), (5, 8195, 64),
                                          (3, 32000, 100), (3, 70001, 2048), (2, 128256, 20), (2, 150003, 20)])
@pytest.mark.parametrize("rest", [False, True])
def test_distill(aq, dtype, teacher, rows, vocab, n, rest):
    z, t, ids, lse = distill_case(31, rows, vocab, n, dtype, teacher)
    lse = lse if rest else None
    w = 0.5 + uniform(33, rows)
    w[rows // 2] = 0 if rows > 3 else 2.0
    loss, loss_off, grad, grad_off = ref.distill(z, t, ids, lse, w, 1.5)
    got, g = aq.distill_loss(z, t, ids, teacher_lse=lse, weights=w, temperature=1.5)
    ref.check(got, loss, loss_off, "loss")
    ref.check(g, grad, grad_off + ref.rounded(grad.abs() + grad_off, dtype), "gradient")
    again, none = aq.distill_loss(z, t, ids, teacher_lse=lse, weights=w, temperature=1.5, grad=False)
    assert none is None and torch.equal(again, got)
    zs = spaced(z)  # rows apart, the gradient over the logits
    got2, g2 = aq.distill_loss(zs, spaced(t), ids, teacher_lse=lse, weights=w, temperature=1.5, out=zs)
    assert torch.equal(got2, got) and torch.equal(zs, g) and torch.isnan(around(zs)).all()
    # without weights every row counts once
    loss, loss_off, grad, grad_off = ref.distill(z, t, ids, lse, None, 1.5)
    got, g = aq.distill_loss(z, t, ids, teacher_lse=lse, temperature=1.5)
    ref.check(got, loss, loss_off, "loss")
    ref.check(g, grad, grad_off + ref.rounded(grad.abs() + grad_off, dtype), "gradient")


@pytest.mark.parametrize("dtype,teacher", [(F16, F32), (BF16, F16), (F32, F32)])
@pytest.mark.parametrize("vocab,n", [(9, 3), (130, 130), (1000, 64), (4099, 20), (16001, 300), (32000, 64), (65531, 50)])
def test_distill_many_rows(aq, dtype, teacher, vocab, n):
    """Enough rows that none is cut."""
    rows = 600
    some = [0, 1, 2, 3, 300, 599]
    z, t, ids, lse = distill_case(41, rows, vocab, n, dtype, teacher)
    if n > 4:
        ids[3, 4] = ids[3, 1]
    w = 0.5 + uniform(42, rows)
    w[1] = 0
    for rest in (None, lse + 2.0):  # (with the mass of entries that are listed twice below 1)
        at = None if rest is None else rest[some]
        loss, loss_off, grad, grad_off = ref.distill(z[some], t[some], ids[some], at, w[some], 1.5)
        got, g = aq.distill_loss(z, t, ids, teacher_lse=rest, weights=w, temperature=1.5)
        ref.check(got[some], loss, loss_off, "loss")
        ref.check(g[some], grad, grad_off + ref.rounded(grad.abs() + grad_off, dtype), "gradient")
        zs = spaced(z)
        got2, _ = aq.distill_loss(zs, t, ids, teacher_lse=rest, weights=w, temperature=1.5, out=zs)
        assert torch.equal(got2, got) and torch.equal(zs, g) and torch.isnan(around(zs)).all()
        # (a row's results do not depend on the others but by the order of its sums)
        few, gf = aq.distill_loss(z[some], t[some], ids[some], teacher_lse=at, weights=w[some], temperature=1.5)
        ref.check(few, loss, loss_off, "loss")
        ref.check(gf, grad, grad_off + ref.rounded(grad.abs() + grad_off, dtype), "gradient")


@pytest.mark.parametrize("dtype,teacher", [(F16, F32), (BF16, F16), (F32, F32)])
@pytest.mark.parametrize("vocab", [128256, 128255])
def test_distill_many_cut_rows(aq, dtype, teacher, vocab):
    """A gradient of more than the caches next to the processors hold, by slices."""
    rows, n = 140, 200
    some = [0, 1, 2, 3, 77, 139]
    z, t, ids, lse = distill_case(43, rows, vocab, n, dtype, teacher)
    ids[3, 4] = ids[3, 1]
    w = 0.5 + uniform(44, rows)
    w[1] = 0
    for rest in (None, lse + 2.0):
        at = None if rest is None else rest[some]
        loss, loss_off, grad, grad_off = ref.distill(z[some], t[some], ids[some], at, w[some], 1.5)
        got, g = aq.distill_loss(z, t, ids, teacher_lse=rest, weights=w, temperature=1.5)
        ref.check(got[some], loss, loss_off, "loss")
        ref.check(g[some], grad, grad_off + ref.rounded(grad.abs() + grad_off, dtype), "gradient")
        zs = spaced(z)
        got2, _ = aq.distill_loss(zs, t, ids, teacher_lse=rest, weights=w, temperature=1.5, out=zs)
        assert torch.equal(got2, got) and torch.equal(zs, g) and torch.isnan(around(zs)).all()


@pytest.mark.parametrize("rows", [3, 600])
@pytest.mark.parametrize("rest", [False, True])
def test_distill_same_id_several_times(aq, rest, rows):
    z, t, ids, lse = (v[:3] for v in distill_case(35, 3, 4001, 40, F32, F32, short=False))
    ids[0, 7] = ids[0, 3]
    ids[0, 39] = ids[0, 3]
    ids[1, :] = 17
    t = t - 3  # (so that the sums of the masses stay below 1)
    lse = lse + 4 if rest else None
    if rows > 3:  # (rows that are not cut)
        full = [None if v is None else v.repeat(rows // 3, *[1] * (v.dim() - 1)) for v in (z, t, ids, lse)]
        loss, loss_off, grad, grad_off = ref.distill(z, t, ids, lse, None, 1.5)
        got, g = aq.distill_loss(full[0], full[1], full[2], teacher_lse=full[3], temperature=1.5)
        ref.check(got[-3:], loss, loss_off, "loss")
        ref.check(g[-3:], grad, grad_off + ref.rounded(grad.abs() + grad_off, F32), "gradient")
        return
    loss, loss_off, grad, grad_off = ref.distill(z, t, ids, lse, None, 1.5)
    for _ in range(3):
        got, g = aq.distill_loss(z, t, ids, teacher_lse=lse, temperature=1.5)
        ref.check(got, loss, loss_off, "loss")
        ref.check(g, grad, grad_off + ref.rounded(grad.abs() + grad_off, F32), "gradient")


@pytest.mark.parametrize("copies", [1, 80])  # (rows that are cut, and not)
@pytest.mark.parametrize("rest", [False, True])
def test_distill_masked_and_special(aq, rest, copies):
    z, t, ids, lse = distill_case(37, 8, 5000, 30, F32, F32, short=False)
    lse = lse if rest else None
    low = torch.finfo(F32).min
    free = torch.ones(5000, dtype=torch.bool, device=DEV)
    free[ids[0].long()] = False
    z[0, free & (torch.arange(5000, device=DEV) % 3 == 0)] = -math.inf  # masked outside the list
    z[1, :] = torch.where(free, low, z[1])
    t[2, 5:] = -math.inf  # entries without mass
    z[3, :] = -math.inf
    z[4, 100] = math.nan
    z[5, :] = math.nan
    w = torch.ones(8, device=DEV)
    w[5] = 0
    z[6] *= 30  # a student that is sure
    ids[7] = -1
    z[7, 3] = 5.0
    many = [None if v is None else v.repeat(copies, *[1] * (v.dim() - 1)) for v in (z, t, ids, lse, w)]
    got, g = aq.distill_loss(*many[:3], teacher_lse=many[3], weights=many[4], temperature=1.5)
    got, g = got[-8:], g[-8:]
    for i in (0, 2, 6, 7):
        loss, loss_off, grad, grad_off = ref.distill(z[i:i + 1], t[i:i + 1], ids[i:i + 1],
                                                     None if lse is None else lse[i:i + 1], None, 1.5)
        ref.check(got[i:i + 1], loss, loss_off, f"loss {i}")
        ref.check(g[i:i + 1], grad, grad_off + ref.rounded(grad.abs() + grad_off, F32), f"gradient {i}")
    assert torch.isnan(got[4]) and torch.isnan(g[4]).any()
    assert got[5] == 0 and not g[5].any()
    if not rest:
        assert torch.isfinite(got[1]) and torch.isfinite(g[1]).all()
    # listed with mass, but impossible for the student
    z[0, ids[0, 0].long()] = -math.inf
    got, _ = aq.distill_loss(z[:1], t[:1], ids[:1], temperature=1.5)
    assert got[0] == math.inf


def test_distill_gradient_by_differences(aq):
    z, t, ids, lse = distill_case(39, 1, 60, 9, F32, F32)
    for rest in (None, lse):
        _, g = aq.distill_loss(z, t, ids, teacher_lse=rest, temperature=1.5)
        zd, step = z.double(), 1e-5
        for j in (int(ids[0, 0]), int(ids[0, 8]), 0, 59):
            d = torch.zeros_like(zd)
            d[0, j] = step
            hi, lo = (ref.distill(v, t, ids, rest, None, 1.5)[0][0] for v in (zd + d, zd - d))
            assert abs(float(g[0, j]) - float((hi - lo) / (2 * step))) <= 1e-5


# --------------------------------------------------------------------------- sampling

def rules(seed, rows, only=None):
    t = 0.3 + 1.2 * uniform(seed, rows)
    t[rows // 2] = 0 if rows > 2 else 1.0
    k = ints([[0, 1, 5, 40, 1000, 3, 200, 7][i % 8] for i in range(rows)])
    p = 0.4 + 0.65 * uniform(seed + 1, rows)
    m = (0.3 * uniform(seed + 2, rows) - 0.1)
    r = dict(temperature=t, top_k=k, top_p=p, min_p=m)
    return {n: r[n] for n in r if only is None or n in only}


def check_sample(aq, x, u, **r):
    got, lp = aq.sample(x, u, return_logprob=True, **r)
    assert got.dtype == torch.int32
    assert torch.equal(aq.sample(x, u, **r), got)
    for i in range(len(x)):
        at = {n: v[i].item() for n, v in r.items()}
        token, want = ref.sample(x[i], u[i].item(), at.get("temperature", 1.0), at.get("top_k", 0), at.get("top_p", 1.0),
                                 at.get("min_p", 0.0))
        assert int(got[i]) == token, (i, int(got[i]), token, at)
        if token >= 0:  # (weights' multiples of 2^-44 of the largest, and one rounding)
            assert abs(float(lp[i]) - want) <= 2.0 ** -23 * abs(want) + 2.0 ** -40 * math.exp(-want), (i, want)
        else:
            assert math.isnan(float(lp[i]))
    return got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 2), (5, 31), (9, 1000), (8, 8195), (8, 32000), (2, 128256), (1, 300007)])
@pytest.mark.parametrize("only", [(), ("temperature",), ("top_k",), ("top_p",), ("min_p",), None])
def test_sample(aq, dtype, rows, vocab, only):
    x = rand(41, rows, vocab) * 2.5
    x[:, vocab // 3] += 5
    x = x.to(dtype)
    check_sample(aq, x, uniform(42, rows), **rules(43, rows, only))


def test_sample_every_border(aq):
    """All numbers of a small row: each token exactly where its share begins."""
    x = torch.log(torch.tensor([1.0, 2, 4, 1, 8, 0, 16, 0], device=DEV)).repeat(32, 1)
    u = torch.arange(32, device=DEV).float() / 32
    want = [0] + [1] * 2 + [2] * 4 + [3] + [4] * 8 + [6] * 16
    got = aq.sample(x, u + 2.0 ** -12)
    assert got.tolist() == want
    # equal logits: exact shares
    x = torch.zeros(64, 64, device=DEV)
    u = torch.arange(64, device=DEV).float() / 64
    assert aq.sample(x, u).tolist() == list(range(64))
    assert aq.sample(x, u, top_k=ints([16] * 64)).tolist() == [i // 4 for i in range(64)]
    assert aq.sample(x, u, top_p=torch.full((64,), 0.25, device=DEV)).tolist() == [i // 4 for i in range(64)]
    assert aq.sample(x, u, min_p=torch.ones(64, device=DEV)).tolist() == list(range(64))
    assert aq.sample(x, u, temperature=torch.zeros(64, device=DEV)).tolist() == [0] * 64


@pytest.mark.parametrize("dtype", TYPES)
def test_sample_ties_and_masks(aq, dtype):
    rows, vocab = 24, 5003
    x = (rand(44, rows, vocab) * 2).round().to(dtype)  # few values, many ties
    x[:, ::7] = -math.inf
    x[1] = -math.inf
    x[2] = -math.inf
    x[2, 4000] = -5.0
    x[3, 11] = math.nan
    x[4] = torch.finfo(dtype).min
    x[5] = torch.finfo(dtype).min
    x[5, 77] = 1.0
    x[6, 99] = x[6, 1003] = math.inf
    x[7] = 0.0
    x[8] = -0.0
    x[8, 1::2] = 0.0
    for only in ((), ("top_k",), ("top_p",), ("min_p",), None):
        got = check_sample(aq, x, uniform(45, rows), **rules(46, rows, only))
        assert int(got[1]) == -1 and int(got[2]) == 4000 and int(got[3]) == -1 and int(got[5]) == 77
        assert int(got[6]) in (99, 1003)


@pytest.mark.parametrize("vocab", [8000, 30000, 128256, 300007])
def test_sample_flat_rows(aq, vocab):
    """Thousands of tokens kept, the last one among thousands that are near it."""
    x = rand(53, 8, vocab) * torch.tensor([0.01, 0.1, 0.5, 1.0, 1.5, 0.5, 0.5, 0.5], device=DEV)[:, None]
    u, full = uniform(54, 8), lambda v, t=F32: torch.full((8,), v, dtype=t, device=DEV)  # noqa: E731
    for r in (dict(top_p=full(0.9)), dict(top_p=full(0.3)), dict(min_p=full(0.05)), dict(top_k=full(700, torch.int32)),
              dict(top_k=full(vocab // 2, torch.int32)), dict(top_p=full(0.999), min_p=full(0.01)),
              dict(top_k=full(1500, torch.int32), top_p=full(0.8)), dict(top_k=full(vocab // 3, torch.int32), top_p=full(0.7)),
              dict(top_p=full(0.9), temperature=full(0.4)), dict(top_k=full(256, torch.int32), top_p=full(0.9))):
        check_sample(aq, x, u, **r)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [8000, 30000, 50001])
def test_sample_gaps_and_long_ties(aq, dtype, vocab):
    """Limits where no logit is, and among thousands of equal ones."""
    x = torch.full((6, vocab), -5.0, device=DEV)
    at = torch.randperm(vocab, device=DEV)
    x[:, at[:3000]] = 5.0
    x[1, at[3000:3003]] = 7.0
    x[2, at[3000:6000]] = 4.0
    x[3] = (rand(55, 1, vocab)[0] * 2).round()
    x[4] = (rand(56, 1, vocab)[0] * 300).round() / 64
    x[5, at[:2990]] = -math.inf
    x = x.to(dtype)
    u, full = uniform(57, 6), lambda v, t=F32: torch.full((6,), v, dtype=t, device=DEV)  # noqa: E731
    for r in (dict(min_p=full(0.5)), dict(min_p=full(0.1)), dict(min_p=full(1e-6)), dict(top_p=full(0.5)),
              dict(top_p=full(0.9999)), dict(top_k=full(100, torch.int32)), dict(top_k=full(2999, torch.int32)),
              dict(top_k=full(3001, torch.int32)), dict(top_k=full(200, torch.int32), top_p=full(0.5)),
              dict(top_k=full(2500, torch.int32), top_p=full(0.5)), dict(top_p=full(0.7), min_p=full(0.5)),
              dict(top_k=full(0, torch.int32), min_p=full(0.5)), dict(temperature=full(0.05), top_p=full(0.5))):
        check_sample(aq, x, u, **r)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [600, 8192, 32001, 128256])
def test_sample_mass_of_many(aq, dtype, vocab):
    """top-p of the mass of more tokens than a list holds, or than have any mass."""
    x = rand(58, 6, vocab) * torch.tensor([0.1, 0.7, 1.5, 3.0, 30.0, 2.0], device=DEV)[:, None]
    x[5, torch.arange(vocab, device=DEV) % 64 != 5] = -math.inf
    x[0, :vocab // 3] = 0.25
    x = x.to(dtype)
    u, full = uniform(59, 6), lambda v, t=F32: torch.full((6,), v, dtype=t, device=DEV)  # noqa: E731
    for k in (257, 599, vocab // 2, vocab - 1):
        for p, least in ((0.02, 0.0), (0.5, 0.3), (0.9, 0.0), (0.9999, 0.001), (1.0 - 2.0 ** -24, 0.0)):
            check_sample(aq, x, u, top_k=full(k, torch.int32), top_p=full(p), min_p=full(least))


def test_sample_extreme_rules(aq):
    x = rand(47, 12, 3000) * 3
    u = torch.tensor([0.0, 1.0 - 2.0 ** -24, 1.0, 2.0, -1.0, math.nan] * 2, device=DEV)
    inside = u.nan_to_num(0.0).clamp(0, 1 - 2.0 ** -24)
    got = aq.sample(x, u)
    assert torch.equal(got[[0, 1, 4, 5]], aq.sample(x, inside)[[0, 1, 4, 5]]) and (got >= 0).all() and (got < 3000).all()
    u = uniform(48, 12)
    first = x.argmax(1).to(torch.int32)
    full = lambda v, t=F32: torch.full((12,), v, dtype=t, device=DEV)  # noqa: E731
    plain = aq.sample(x, u)
    for r in (dict(top_k=full(1, torch.int32)), dict(top_p=full(0.0)), dict(top_p=full(-1.0)), dict(min_p=full(1.0)),
              dict(min_p=full(7.0)), dict(temperature=full(1e-30)), dict(temperature=full(-1.0)),
              dict(temperature=full(math.nan))):
        assert torch.equal(aq.sample(x, u, **r), first), r
    for r in (dict(top_k=full(0, torch.int32)), dict(top_k=full(-3, torch.int32)), dict(top_k=full(3000, torch.int32)),
              dict(top_k=full(2 ** 31 - 1, torch.int32)), dict(top_p=full(1.0)), dict(top_p=full(math.nan)),
              dict(top_p=full(9.0)), dict(min_p=full(0.0)), dict(min_p=full(math.nan)), dict(temperature=full(1.0))):
        assert torch.equal(aq.sample(x, u, **r), plain), r
    flat = check_sample(aq, x, u, temperature=full(1e30))
    assert len(set(flat.tolist())) > 6
    x[:, 5] = 1e30
    check_sample(aq, x, u, temperature=full(3.0))


def test_sample_rows_apart_and_of_one(aq):
    x = rand(49, 6, 4001)
    u = uniform(50, 6)
    r = rules(51, 6)
    want = aq.sample(x, u, **r)
    assert torch.equal(aq.sample(spaced(x), u, **r), want)
    for i in range(6):  # the same token whatever the batch
        one = aq.sample(x[i:i + 1], u[i:i + 1], **{n: v[i:i + 1] for n, v in r.items()})
        assert int(one) == int(want[i])
    same = x[:1].expand(6, 4001)  # one row for several draws
    assert torch.equal(aq.sample(same, u, **r), aq.sample(same.contiguous(), u, **r))
    assert aq.sample(x[:0], u[:0]).shape == (0,)


def test_sample_frequencies(aq):
    """65536 equally spaced numbers over one row: each token as often as its share."""
    n = 1 << 16
    x = rand(52, 1, 50)
    got = aq.sample(x.expand(n, 50), (torch.arange(n, device=DEV).float() + 0.5) / n)
    share = torch.softmax(x[0].double(), 0) * n
    assert ((torch.bincount(got.long(), minlength=50) - share).abs() <= 1.0 + 1e-6).all()
