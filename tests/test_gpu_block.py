"""The operators of ``block.py`` on the GPU against their definitions in 64 bits."""
import math

import pytest

torch = pytest.importorskip("torch")

import block_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda"
EPS = 1e-5


@pytest.fixture(scope="module")
def aq():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2401_06118_amd as aqlm
    return aqlm


def rand(seed, *shape, dtype=torch.float16, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype)


def within(got, want, tol, what=""):
    got = got.double().cpu()
    fin = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), fin), f"{what}: {int((torch.isfinite(got) != fin).sum())} not finite where the other is"
    assert torch.equal(got[~fin].nan_to_num(7.0, 8.0, 9.0), want[~fin].nan_to_num(7.0, 8.0, 9.0)), what
    over = (got - want).abs()[fin] - tol.expand_as(want)[fin]
    assert over.numel() == 0 or over.max() <= 0, f"{what}: {float(over.max()):.3g} over its bound"


# ---------------------------------------------------------------------------
# rotary positions and head norms

def rope_bound(dtype, want, size):
    # sums of up to 1024 squares, the factor and two products in fp32, rounded once
    return ref.UNIT[dtype] * want.abs() + 2.0 ** -19 * size + ref.TINY[dtype]


ROPE = [
    # tokens, heads, kv, dim, rot, interleaved, norms, dtype
    (1, 32, 32, 128, 128, False, "", torch.float16),
    (1, 1, 1, 2, 2, True, "qk", torch.float32),
    (7, 5, 3, 64, 64, True, "qk", torch.bfloat16),
    (33, 8, 1, 80, 80, False, "q", torch.float16),
    (33, 8, 1, 96, 48, False, "k", torch.bfloat16),
    (19, 4, 2, 128, 32, True, "qk", torch.float32),
    (1000, 64, 8, 128, 128, False, "qk", torch.float16),   # four heads a group
    (700, 28, 4, 256, 128, True, "", torch.bfloat16),
    (5, 3, 2, 512, 256, False, "qk", torch.float16),
    (9, 3, 2, 80, 40, False, "qk", torch.float16),         # general: halves that are no whole pieces
    (9, 3, 2, 50, 18, True, "qk", torch.bfloat16),         # general: odd head size
    (3, 2, 1, 1024, 1000, False, "qk", torch.float32),     # general: the largest head
    (6, 2, 2, 576, 64, True, "", torch.float16),           # general: more than 512
    (4, 2, 2, 128, 22, True, "q", torch.float16),          # general: the table's rows are not aligned
    (4, 2, 2, 40, 14, True, "qk", torch.float16),          # pairs that end inside a piece
]


def rope_inputs(tokens, heads, kv, dim, rot, norms, dtype, rows=300, seed=0):
    a = rand(seed, tokens, heads + kv, dim, dtype=dtype, scale=2.0)
    t = ref.table64(rows, rot).float()
    g = torch.Generator().manual_seed(seed + 1)
    pos = torch.randint(0, rows, (tokens,), generator=g).to(torch.int32)
    pos[-1] = rows - 1
    wq = (1 + rand(seed + 2, dim, dtype=torch.float32, scale=0.2)).to(dtype) if "q" in norms else None
    wk = (1 + rand(seed + 3, dim, dtype=torch.float32, scale=0.2)).to(dtype) if "k" in norms else None
    return a, t, pos, wq, wk


def dev(*ts):
    return [None if t is None else t.to(DEV) for t in ts]


def dbl(t):
    return None if t is None else t.double()


@pytest.mark.parametrize("tokens,heads,kv,dim,rot,inter,norms,dtype", ROPE)
def test_rope(aq, tokens, heads, kv, dim, rot, inter, norms, dtype):
    a, t, pos, wq, wk = rope_inputs(tokens, heads, kv, dim, rot, norms, dtype)
    da, dt, dp, dwq, dwk = dev(a, t, pos, wq, wk)
    q, k = aq.rope(da[:, :heads], da[:, heads:], dt, dp, q_weight=dwq, k_weight=dwk, eps=EPS, interleaved=inter)
    for got, x, w, name in ((q, a[:, :heads], wq, "q"), (k, a[:, heads:], wk, "k")):
        want, size = ref.rope64(x.double(), dbl(w), t.double(), pos.long(), inter, EPS)
        assert got.is_contiguous() and got.dtype == dtype
        within(got, want, rope_bound(dtype, want, size), name)
    # in place, in the fused activation
    aq.rope(da[:, :heads], da[:, heads:], dt, dp, q_weight=dwq, k_weight=dwk, eps=EPS, interleaved=inter,
            out=(da[:, :heads], da[:, heads:]))
    assert torch.equal(da[:, :heads], q) and torch.equal(da[:, heads:], k)


def test_rope_strides_and_alignment(aq):
    """Heads before tokens, gaps, and addresses that are not multiples of 16 bytes give the same bits."""
    a, t, pos, wq, wk = rope_inputs(21, 4, 2, 64, 64, "qk", torch.float16)
    da, dt, dp, dwq, dwk = dev(a, t, pos, wq, wk)
    kw = dict(q_weight=dwq, k_weight=dwk, eps=EPS)
    q, k = aq.rope(da[:, :4].contiguous(), da[:, 4:].contiguous(), dt, dp, **kw)
    turned = da.transpose(0, 1).contiguous().transpose(0, 1)
    oq = torch.empty(4, 21, 64, dtype=torch.float16, device=DEV).transpose(0, 1)
    ok = torch.empty(21, 2, 72, dtype=torch.float16, device=DEV)[..., :64]
    aq.rope(turned[:, :4], turned[:, 4:], dt, dp, out=(oq, ok), **kw)
    assert torch.equal(oq, q) and torch.equal(ok, k)
    odd = torch.empty(21 * 6 * 64 + 3, dtype=torch.float16, device=DEV)[3:].view(21, 6, 64)
    odd.copy_(da)
    q2, k2 = aq.rope(odd[:, :4], odd[:, 4:], dt, dp, **kw)
    for got, want in ((q2, q), (k2, k)):  # (the general kernel adds up in another order)
        assert (got.float() - want.float()).abs().max() <= 2.0 ** -9 * want.float().abs().max()


def test_rope_positions_outside(aq):
    """Positions that the table does not have give NaN in their tokens only."""
    for dim, rot in ((64, 32), (50, 18)):
        a, t, pos, _, _ = rope_inputs(6, 2, 1, dim, rot, "", torch.float16, rows=40)
        pos = torch.tensor([0, -1, 39, 40, 2 ** 31 - 1, 5], dtype=torch.int32)
        q, k = aq.rope(*dev(a[:, :2], a[:, 2:], t, pos))
        bad = torch.tensor([False, True, False, True, True, False])
        assert torch.isnan(q.cpu()[bad]).all() and torch.isnan(k.cpu()[bad]).all()
        assert not torch.isnan(q.cpu()[~bad]).any() and not torch.isnan(k.cpu()[~bad]).any()


def test_rope_special_values(aq):
    """NaN and infinities stay in their head; a head of zeros has a finite norm."""
    a, t, pos, wq, wk = rope_inputs(4, 3, 1, 64, 64, "qk", torch.float16)
    a[0, 0, 3] = math.nan
    a[1, 1, 5] = math.inf
    a[2, 2] = 0
    q, _ = aq.rope(*dev(a[:, :3], a[:, 3:], t, pos), q_weight=wq.to(DEV), k_weight=wk.to(DEV), eps=EPS)
    q = q.cpu()
    assert torch.isnan(q[0, 0]).all()
    assert not torch.isfinite(q[1, 1]).all()
    assert (q[2, 2] == 0).all()
    rest = torch.ones(4, 3, dtype=torch.bool)
    rest[0, 0] = rest[1, 1] = False
    assert torch.isfinite(q[rest]).all()


@pytest.mark.parametrize("tokens,heads,kv,dim,rot,inter,norms,dtype", ROPE)
def test_rope_backward(aq, tokens, heads, kv, dim, rot, inter, norms, dtype):
    a, t, pos, wq, wk = rope_inputs(tokens, heads, kv, dim, rot, norms, dtype)
    dy = rand(77, tokens, heads + kv, dim, dtype=dtype, scale=0.3)
    da, ddy, dt, dp, dwq, dwk = dev(a, dy, t, pos, wq, wk)
    args = (ddy[:, :heads], ddy[:, heads:], dt, dp)
    kw = dict(q=da[:, :heads], k=da[:, heads:], q_weight=dwq, k_weight=dwk, eps=EPS, interleaved=inter)
    got = aq.rope_backward(*args, **kw)
    again = aq.rope_backward(*args, **kw)
    for i, (x, g, w) in enumerate(((a[:, :heads], dy[:, :heads], wq), (a[:, heads:], dy[:, heads:], wk))):
        dx, mag, dw, wmag = ref.rope_grad64(g.double(), x.double(), dbl(w), t.double(), pos.long(), inter, EPS)
        # two sums of up to 1024 products and the factors in fp32, rounded once
        within(got[i], dx, ref.UNIT[dtype] * dx.abs() + 2.0 ** -18 * mag + ref.TINY[dtype], "dx")
        assert (got[2 + i] is None) == (w is None)
        if w is not None:  # a workgroup adds up to (items / 1024 + 32) terms, 1024 workgroups' sums follow
            n = tokens * heads / 1024 + 1100
            within(got[2 + i], dw, 2.0 ** -24 * n * wmag + 2.0 ** -19 * wmag, "dw")
            assert torch.equal(got[2 + i], again[2 + i])
        assert torch.equal(got[i], again[i])


def test_rope_backward_differences(aq):
    """Gradients against central differences of the definition in 64 bits."""
    tokens, heads, kv, dim, rot = 3, 2, 1, 16, 8
    a, t, pos, wq, wk = rope_inputs(tokens, heads, kv, dim, rot, "qk", torch.float32)
    dy = rand(5, tokens, heads + kv, dim, dtype=torch.float32)
    for inter in (False, True):
        got = aq.rope_backward(*dev(dy[:, :heads], dy[:, heads:], t, pos), q=a[:, :heads].to(DEV),
                               k=a[:, heads:].to(DEV), q_weight=wq.to(DEV), k_weight=wk.to(DEV), eps=EPS,
                               interleaved=inter)
        for i, (x, g, w) in enumerate(((a[:, :heads], dy[:, :heads], wq), (a[:, heads:], dy[:, heads:], wk))):
            def loss(x, w):
                return float((ref.rope64(x, w, t.double(), pos.long(), inter, EPS)[0] * g.double()).sum())
            x, w, h = x.double(), w.double(), 1e-5
            for n in range(x.numel()):
                d = torch.zeros(x.numel(), dtype=torch.float64)
                d[n] = h
                slope = (loss(x + d.view_as(x), w) - loss(x - d.view_as(x), w)) / (2 * h)
                assert abs(slope - float(got[i].flatten()[n])) <= 2e-5 * (1 + abs(slope))
            for n in range(dim):
                d = torch.zeros(dim, dtype=torch.float64)
                d[n] = h
                slope = (loss(x, w + d) - loss(x, w - d)) / (2 * h)
                assert abs(slope - float(got[2 + i][n])) <= 2e-5 * (1 + abs(slope))


@pytest.mark.parametrize("scaling", [None, {"kind": "linear", "factor": 4.0}, {"kind": "ntk", "factor": 2.0},
                                     {"kind": "yarn", "factor": 4.0, "original": 512},
                                     {"kind": "llama3", "factor": 8.0, "original": 1024}])
def test_rotary_table(aq, scaling):
    rows, rot, base = 2000, 64, 10000.0
    t = aq.rotary_table(rows, rot, base=base, scaling=scaling).double().cpu()
    i = torch.arange(rot // 2, dtype=torch.float64)
    f = base ** (-2 * i / rot)
    scale = 1.0
    if scaling is not None:
        kind, s = scaling["kind"], scaling["factor"]
        if kind == "linear":
            f = f / s
        elif kind == "ntk":
            f = (base * s ** (rot / (rot - 2))) ** (-2 * i / rot)
        else:
            turns = scaling["original"] * f / (2 * math.pi)
            if kind == "llama3":
                keep = ((turns - 1) / 3).clamp(0, 1)
            else:
                at = [rot * math.log(scaling["original"] / (n * 2 * math.pi)) / (2 * math.log(base)) for n in (32, 1)]
                lo, hi = max(0, math.floor(at[0])), min(rot - 1, math.ceil(at[1]))
                keep = 1 - ((i - lo) / (hi - lo)).clamp(0, 1)
                scale = 0.1 * math.log(s) + 1
            f = f * keep + f / s * (1 - keep)
    a = torch.arange(rows, dtype=torch.float64)[:, None] * f
    want = torch.stack([a.cos(), a.sin()], -1) * scale
    # one rounding to fp32; angles up to 2000 in 64 bits
    assert (t - want).abs().max() <= 2.0 ** -24 * scale + 1e-11
    half = aq.rotary_table(1, 2)
    assert torch.equal(half.cpu(), torch.tensor([[[1.0, 0.0]]]))


# ---------------------------------------------------------------------------
# the paged cache

class Batch:
    """Sequences with pages in a mixed order, and stale values everywhere else."""

    def __init__(self, lens, new, kv, dim, page, dtype, seed=0, layout="slot", stale=None, spare=2):
        self.lens, self.new, self.page, self.dtype = lens, new, page, dtype
        width = max(1, max(-(-n // page) for n in lens)) + 1
        count = sum(-(-n // page) for n in lens) + spare
        g = torch.Generator().manual_seed(seed)
        order = torch.randperm(count, generator=g)
        self.table = torch.full((len(lens), width), 10 ** 6, dtype=torch.int32)  # unused entries: no page
        at = 0
        for b, n in enumerate(lens):
            for i in range(-(-n // page)):
                self.table[b, i] = order[at]
                at += 1
        shape = (count, page, kv, dim)
        self.k, self.v = (torch.randn(shape, generator=g).to(dtype) for _ in range(2))
        if stale is not None:  # slots past the sequences' ends hold anything
            used = torch.zeros(count, page, dtype=torch.bool)
            for b, n in enumerate(lens):
                for j in range(n):
                    used[self.table[b, j // page].long(), j % page] = True
            self.k[~used] = stale
            self.v[~used] = stale
        self.layout = layout
        self.cu = torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32)
        self.kv_lens = torch.tensor(lens, dtype=torch.int32)
        self.total = sum(new)

    def place(self, t):
        """On the GPU, [pages, page, kv, dim] or the same values with heads before slots."""
        if self.layout == "head":
            return t.to(DEV).transpose(1, 2).contiguous().transpose(1, 2)
        return t.to(DEV)

    def gpu(self):
        return self.place(self.k), self.place(self.v), self.table.to(DEV), self.kv_lens.to(DEV), self.cu.to(DEV)


APPEND = [
    # lens, new, heads, kv, dim, rot, interleaved, norms, page, layout, dtype
    ([1], [1], 4, 4, 64, 64, False, "", 16, "slot", torch.float16),
    ([5, 40, 17, 64], [1, 1, 1, 1], 8, 2, 128, 128, False, "qk", 16, "slot", torch.float16),
    ([33, 0, 7, 100], [33, 1, 0, 9], 8, 2, 128, 64, True, "k", 8, "head", torch.bfloat16),
    ([12, 3], [5, 3], 3, 3, 80, 40, False, "qk", 4, "slot", torch.float16),     # general kernel
    ([12, 3], [5, 3], 3, 1, 50, 0, False, "q", 1, "slot", torch.float32),       # no rotation, pages of one
    ([700, 130], [600, 130], 32, 8, 128, 128, False, "qk", 64, "slot", torch.bfloat16),
]


@pytest.mark.parametrize("lens,new,heads,kv,dim,rot,inter,norms,page,layout,dtype", APPEND)
def test_paged_append(aq, lens, new, heads, kv, dim, rot, inter, norms, page, layout, dtype):
    bt = Batch(lens, new, kv, dim, page, dtype, layout=layout)
    a = rand(3, bt.total, heads + 2 * kv, dim, dtype=dtype)
    t = ref.table64(1000, rot).float() if rot else None
    _, _, _, wq, wk = rope_inputs(1, heads, kv, dim, max(rot, 2), norms, dtype)
    kc, vc, table, kl, cu = bt.gpu()
    da, dt, dwq, dwk = dev(a, t, wq, wk)
    q = aq.paged_append(da[:, :heads], da[:, heads:heads + kv], da[:, heads + kv:], kc, vc, table, kl, cu, table=dt,
                        q_weight=dwq, k_weight=dwk, eps=EPS, interleaved=inter)
    t64 = t.double() if rot else torch.zeros(1000, 0, 2, dtype=torch.float64)
    want_q, size_q = torch.zeros(bt.total, heads, dim, dtype=torch.float64), torch.zeros(bt.total, heads, dim, dtype=torch.float64)
    want_k, want_v, size_k = bt.k.double(), bt.v.double(), torch.zeros(bt.k.shape, dtype=torch.float64)
    for b, (n, m) in enumerate(zip(new, lens)):
        for i in range(n):
            tok, pos = int(bt.cu[b]) + i, m - n + i
            if pos < 0:
                continue
            p = torch.tensor([pos])
            want_q[tok], size_q[tok] = (x[0] for x in ref.rope64(a[tok:tok + 1, :heads].double(), dbl(wq), t64, p, inter, EPS))
            y, s = ref.rope64(a[tok:tok + 1, heads:heads + kv].double(), dbl(wk), t64, p, inter, EPS)
            at = int(bt.table[b, pos // page]), pos % page
            want_k[at], size_k[at], want_v[at] = y[0], s[0], a[tok, heads + kv:].double()
    within(q, want_q, rope_bound(dtype, want_q, size_q), "q")
    tol = rope_bound(dtype, want_k, size_k)
    tol[size_k == 0] = 0  # what was not written is as it was
    within(kc, want_k, tol, "k")
    assert torch.equal(vc.double().cpu(), want_v)
    # without queries
    kc2, vc2 = bt.gpu()[:2]
    assert aq.paged_append(None, da[:, heads:heads + kv], da[:, heads + kv:], kc2, vc2, table, kl, cu, table=dt,
                           k_weight=dwk, eps=EPS, interleaved=inter) is None
    assert torch.equal(kc2, kc) and torch.equal(vc2, vc)


def test_paged_append_pages_outside(aq):
    """Pages that the table or the cache does not have are not written to."""
    bt = Batch([40, 9], [2, 9], 2, 64, 16, torch.float16)
    bt.table[0, 2] = -3          # the new tokens of the first sequence are on it
    bt.table[1, 0] = 5000
    bt.kv_lens[1] = 10 ** 6      # and those of the second past the table's end
    a = rand(3, 11, 6, 64)
    kc, vc, table, kl, cu = bt.gpu()
    q = aq.paged_append(a[:, :2].to(DEV), a[:, 2:4].to(DEV), a[:, 4:].to(DEV), kc, vc, table, kl, cu)
    assert torch.equal(kc.cpu(), bt.k) and torch.equal(vc.cpu(), bt.v)
    assert torch.equal(q.cpu(), a[:, :2])


ATTEND = [
    # lens, new, heads, kv, dim, page, causal, window
    ([1], [1], 1, 1, 64, 16, True, 0),
    ([1], [1], 32, 32, 128, 16, True, 0),
    ([2], [1], 8, 1, 128, 1, True, 0),
    ([127, 128, 129, 33], [1] * 4, 8, 2, 128, 16, True, 0),
    ([1000], [1], 4, 4, 128, 64, True, 0),
    ([3000, 5, 0, 700], [1] * 4, 8, 1, 64, 32, True, 0),                  # an idle slot
    ([500, 90], [1, 1], 10, 2, 80, 16, True, 0),                          # heads shorter than the kernel's
    ([300, 31], [1, 1], 6, 2, 256, 8, True, 0),
    ([257], [1], 3, 3, 200, 8, True, 0),
    ([600, 10], [1, 1], 8, 2, 128, 16, True, 100),
    ([50, 9, 300], [5, 9, 3], 4, 4, 128, 16, True, 0),                    # drafts
    ([50, 9, 300], [4, 2, 3], 8, 2, 64, 16, True, 7),
    ([40, 70], [3, 2], 4, 2, 96, 16, False, 0),
    ([64], [64], 4, 1, 128, 16, True, 0),                                 # a whole prompt
    ([65], [33], 2, 2, 64, 16, True, 0),
    ([130, 1, 77], [130, 1, 40], 6, 2, 128, 8, True, 0),
    ([333], [200], 5, 5, 80, 32, True, 0),
    ([520], [100], 4, 2, 256, 64, True, 0),
    ([200], [170], 2, 1, 248, 64, True, 50),
    ([900, 30, 0, 257], [300, 30, 2, 17], 8, 2, 128, 16, True, 64),       # windows, an idle slot of two tokens
    ([400, 129], [129, 129], 4, 4, 128, 128, False, 0),
    ([300], [50], 4, 2, 64, 16, False, 40),
    ([20, 60], [30, 60], 4, 2, 128, 16, True, 0),                         # more tokens than keys: rows without keys
    ([20, 60], [7, 2], 4, 2, 128, 16, True, 1),
]


def attend_case(lens, new, heads, kv, dim, page, dtype, seed=1, **kw):
    bt = Batch(lens, new, kv, dim, page, dtype, seed=seed, **kw)
    a = rand(seed + 9, bt.total, heads + 1, dim, dtype=dtype, scale=1.5)
    return bt, a[:, :heads]


def check_attention(aq, bt, q, causal, window, scale=None, max_new=None, **kw):
    dtype = q.dtype
    s = q.shape[2] ** -0.5 if scale is None else scale
    want, size, score, lse = ref.attend64(q, bt.k, bt.v, bt.table, bt.lens, bt.cu, s, causal, window)
    outs = []
    for most in (max(bt.new), 0) if max_new is None else (max_new,):
        got, got_lse = aq.paged_attention(q.to(DEV), *bt.gpu(), causal=causal, window=window, scale=scale, max_new=most,
                                          return_lse=True, **kw)
        within(got, want, ref.attend_bound(dtype, want, size, score), f"out, max_new {most}")
        within(got_lse, lse, 2.0 ** -19 * (score[..., 0] + lse.abs().nan_to_num(0.0, 0.0, 0.0) + 2), "lse")
        outs.append((got, got_lse))
    return outs


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("lens,new,heads,kv,dim,page,causal,window", ATTEND)
def test_attention(aq, lens, new, heads, kv, dim, page, causal, window, dtype):
    bt, q = attend_case(lens, new, heads, kv, dim, page, dtype)
    check_attention(aq, bt, q, causal, window)


@pytest.mark.parametrize("max_new", [1, 400])
def test_attention_any_max_new(aq, max_new):
    """max_new is a hint: a wrong one gives the same results."""
    bt, q = attend_case([400, 90, 33], [300, 5, 1], 8, 2, 128, 16, torch.float16)
    check_attention(aq, bt, q, True, 0, max_new=max_new)


@pytest.mark.parametrize("lens,new,heads,kv", [([9000], [1], 4, 1), ([20000, 300], [1, 1], 8, 2), ([6000], [150], 2, 1),
                                               ([5000, 10, 4000], [40, 10, 80], 4, 1)])
def test_attention_split(aq, lens, new, heads, kv):
    """Units that many workgroups share: right, the same bits every time, the workspace ready for the next call."""
    bt, q = attend_case(lens, new, heads, kv, 128, 16, torch.bfloat16)
    ws = aq.attention_workspace(128)
    outs = []
    for _ in range(3):
        outs.append(check_attention(aq, bt, q, True, 0, max_new=max(new), workspace=ws)[0])
        assert int(ws[:16384].sum()) == 0
        ws[16384:].fill_(0xFF)  # whatever else the workspace holds
    assert all(torch.equal(o[0], outs[0][0]) and torch.equal(o[1], outs[0][1]) for o in outs)


@pytest.mark.parametrize("count,most", [(70, 90), (150, 40), (9, 200)])
def test_attention_many_sequences(aq, count, most):
    """Sequences of one unit and of several, in any order, more than a wave has lanes."""
    new = [1 + (37 * i) % most for i in range(count)]
    lens = [n + (53 * i) % 130 for i, n in enumerate(new)]
    bt, q = attend_case(lens, new, 4, 1, 64, 16, torch.float16)
    outs = [check_attention(aq, bt, q, True, 0, max_new=most)[0] for _ in range(2)]
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


@pytest.mark.parametrize("stale", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("new", [[1, 1, 1], [3, 2, 1], [60, 40, 77]])
def test_attention_stale_slots(aq, stale, new):
    """Slots past a sequence's end may hold anything."""
    bt, q = attend_case([70, 45, 129], new, 4, 2, 128, 16, torch.float16, stale=stale)
    check_attention(aq, bt, q, True, 0)


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
@pytest.mark.parametrize("new,window", [([4, 2], 0), ([4, 2], 30), ([50, 90], 0), ([50, 90], 25)])
def test_attention_values_of_unseen_keys(aq, value, dim, new, window):
    """A key that some rows see and others do not: an infinite or NaN value (or key)
    of it is theirs alone."""
    bt, q = attend_case([120, 95], new, 4, 2, dim, 16, torch.bfloat16)
    for b, j, h in ((0, 117, 0), (1, 94, 1), (0, 96, 1), (0, 118, 0)):
        bt.v[int(bt.table[b, j // 16]), j % 16, h, (5 * j) % dim] = value if j != 118 else -value
    got = check_attention(aq, bt, q, True, window)
    assert any((~torch.isfinite(o)).any() for o, _ in got)
    bt, q = attend_case([120, 95], new, 4, 2, dim, 16, torch.bfloat16)
    bt.k[int(bt.table[0, 118 // 16]), 118 % 16, 0, 3] = value
    seen = ref.visible(new[0], 120, True, window)[:, 118]
    for most in (max(new), 0):
        got = aq.paged_attention(q.to(DEV), *bt.gpu(), window=window, max_new=most).cpu()
        rows = torch.zeros(bt.total, dtype=torch.bool)
        rows[:new[0]] = seen
        assert torch.isfinite(got[~rows]).all() and torch.isfinite(got[:, 2:]).all()


def test_attention_extreme_scores(aq):
    """Scores far apart, of either sign, and one key that outweighs all others."""
    for new in ([1], [40]):
        bt, q = attend_case([300], new, 4, 2, 64, 16, torch.float16)
        bt.k *= 40
        check_attention(aq, bt, q, True, 0)
        bt.k[:] = -abs(bt.k)
        check_attention(aq, bt, abs(q), True, 0)
        check_attention(aq, bt, q, True, 0, scale=0.0)
        check_attention(aq, bt, q, True, 0, scale=-0.01)


def test_attention_layouts(aq):
    """Heads before slots in the pages, values with strides of their own, queries and
    outputs with tokens inside heads: the same bits."""
    for new in ([1, 1], [70, 3]):
        bt, q = attend_case([200, 90], new, 4, 2, 128, 16, torch.float16)
        base = aq.paged_attention(q.to(DEV), *bt.gpu())
        k, _, table, kl, cu = bt.gpu()
        bt.layout = "head"
        v = bt.gpu()[1]
        out = torch.empty(4, bt.total, 136, dtype=torch.float16, device=DEV)[..., :128].transpose(0, 1)
        qt = q.to(DEV).transpose(0, 1).contiguous().transpose(0, 1)
        aq.paged_attention(qt, k, v, table, kl, cu, out=out)
        assert torch.equal(out, base)
        wide = torch.zeros(2, table.shape[1] + 5, dtype=torch.int32, device=DEV)
        wide[:, :table.shape[1]] = table
        assert torch.equal(aq.paged_attention(qt, k, v, wide[:, :table.shape[1]], kl, cu), base)


def test_attention_bad_lengths_stay_inside(aq):
    """Page numbers and lengths that do not fit are cut to the arrays: no access
    outside, other sequences as ever."""
    for new in ([1, 1, 1], [40, 1, 20]):
        bt, q = attend_case([100, 60, 40], new, 4, 2, 64, 16, torch.float16)
        base = aq.paged_attention(q.to(DEV), *bt.gpu())
        bt.kv_lens = torch.tensor([100, 2 ** 31 - 1, -5], dtype=torch.int32)
        bt.table[1] = torch.tensor([-1, 2 ** 31 - 1] * 10)[:bt.table.shape[1]]
        got = aq.paged_attention(q.to(DEV), *bt.gpu())
        n = new[0]
        assert torch.equal(got[:n], base[:n])
        assert (got[-new[2]:] == 0).all()


def test_offsets_past_32_bits(aq):
    """Pages beyond 2^32 elements of the cache."""
    page, kv, dim = 16, 2, 128
    stride = page * kv * dim
    pages = (1 << 32) // stride + 40
    k = torch.empty(pages, page, kv, dim, dtype=torch.float16, device=DEV)
    v = torch.empty(pages, page, kv, dim, dtype=torch.float16, device=DEV)
    for new in ([1], [30]):
        bt, q = attend_case([200], new, 4, kv, dim, page, torch.float16)
        table = bt.table.clone()
        n = -(-200 // page)
        far = torch.arange(pages - n, pages).flip(0).to(torch.int32)
        for i in range(n):
            k[int(far[i])] = bt.k[int(table[0, i])].to(DEV)
            v[int(far[i])] = bt.v[int(table[0, i])].to(DEV)
        table[0, :n] = far
        got = aq.paged_attention(q.to(DEV), k, v, table.to(DEV), bt.kv_lens.to(DEV), bt.cu.to(DEV))
        assert torch.equal(got, aq.paged_attention(q.to(DEV), *bt.gpu()))
        x = rand(8, bt.total, 2 * kv, dim)
        aq.paged_append(None, x[:, :kv].to(DEV), x[:, kv:].to(DEV), k, v, table.to(DEV), bt.kv_lens.to(DEV),
                        bt.cu.to(DEV))
        last = int(table[0, 199 // page])
        assert torch.equal(k[last, 199 % page].cpu(), x[-1, :kv]) and torch.equal(v[last, 199 % page].cpu(), x[-1, kv:])


# ---------------------------------------------------------------------------
# logits

LOGITS = [
    # rows, vocab, history, biases, mask, dtype
    (1, 32000, 200, 5, True, torch.float16),
    (3, 1001, 64, 0, True, torch.bfloat16),
    (2, 33, 300, 40, True, torch.float32),       # more tokens and biases than words
    (5, 8193, 1, 1, False, torch.float32),
    (1, 1, 5, 3, True, torch.float32),
    (64, 20000, 100, 9, False, torch.float16),   # the larger slices
]


def logits_case(rows, vocab, history, biases, masked, dtype, seed=4):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(rows, vocab, generator=g) * 4).to(dtype)
    tokens = (vocab ** torch.rand(rows, history, generator=g)).to(torch.int32) - 1
    tokens[:, ::7] = -1                  # ids that are none
    tokens[:, ::11] = vocab
    lens = torch.randint(0, history + 1, (rows,), generator=g).to(torch.int32)
    lens[0] = history
    prompt = (lens.float() * torch.rand(rows, generator=g)).to(torch.int32)
    pen = [1 + torch.rand(rows, generator=g), torch.randn(rows, generator=g), torch.randn(rows, generator=g)]
    ids = values = mask = None
    if biases:
        ids = torch.randint(-1, min(vocab, 50), (rows, biases), generator=g).to(torch.int32)
        values = torch.randn(rows, biases, generator=g) * 3
    if masked:
        mask = torch.randint(-2 ** 31, 2 ** 31, (rows, -(-vocab // 32) + 1), generator=g).to(torch.int32)
        mask[-1] = 0
        mask[0, 0] |= 1
    return x, tokens, lens, prompt, pen, ids, values, mask


@pytest.mark.parametrize("rows,vocab,history,biases,masked,dtype", LOGITS)
def test_process_logits(aq, rows, vocab, history, biases, masked, dtype):
    x, tokens, lens, prompt, (r, f, p), ids, values, mask = logits_case(rows, vocab, history, biases, masked, dtype)
    want, size = ref.logits64(x, tokens, lens, prompt, r, f, p, ids, values, mask)
    args = dict(zip(("tokens", "token_lens", "prompt_lens", "repetition", "frequency", "presence", "bias_ids",
                     "bias_values", "mask"), dev(tokens, lens, prompt, r, f, p, ids, values, mask)))
    got = aq.process_logits(x.to(DEV), **args)
    # up to 4 + biases roundings in fp32 of the magnitudes, one to the type
    tol = ref.UNIT[dtype] * want.abs() * 1.001 + 2.0 ** -24 * (6 + biases) * size + ref.TINY[dtype]
    tol = torch.where(torch.isfinite(want), tol, torch.zeros_like(tol))
    within(got, want, tol)
    # in place, in rows that are part of a larger buffer with an odd pitch
    buf = torch.zeros(rows, vocab + 3, dtype=dtype, device=DEV)
    buf[:, :vocab] = x.to(DEV)
    view = buf[:, :vocab]
    aq.process_logits(view, out=view, **args)
    assert torch.equal(view, got) and (buf[:, vocab:] == 0).all()


def test_process_logits_parts(aq):
    """Each part alone, and none of them."""
    x, tokens, lens, prompt, (r, f, p), ids, values, mask = logits_case(3, 500, 40, 6, True, torch.float32)
    d = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    assert torch.equal(aq.process_logits(d(x)).cpu(), x)
    for kw in (dict(repetition=r), dict(frequency=f), dict(presence=p), dict(repetition=r, presence=p)):
        for pl in (None, prompt):
            got = aq.process_logits(d(x), tokens=d(tokens), token_lens=d(lens), prompt_lens=d(pl),
                                    **{k: d(v) for k, v in kw.items()})
            want, size = ref.logits64(x, tokens, lens, pl, kw.get("repetition"), kw.get("frequency"),
                                      kw.get("presence"), None, None, None)
            within(got, want, 2.0 ** -21 * size + 2.0 ** -126)
    got = aq.process_logits(d(x), bias_ids=d(ids), bias_values=d(values))
    want, size = ref.logits64(x, None, None, None, None, None, None, ids, values, None)
    within(got, want, 2.0 ** -21 * size + 2.0 ** -126)
    got = aq.process_logits(d(x), mask=d(mask)).cpu()
    want, _ = ref.logits64(x, None, None, None, None, None, None, None, None, mask)
    assert torch.equal(got.double(), want)
    empty = torch.zeros(3, 0, dtype=torch.int32, device=DEV)
    assert torch.equal(aq.process_logits(d(x), tokens=empty, token_lens=d(lens * 0), repetition=d(r)).cpu(), x)


def test_process_logits_without_history(aq):
    """Token lists of no entries through the C ABI: nothing is read from them."""
    import ctypes

    x = rand(1, 2, 100, dtype=torch.float32).to(DEV)
    ints, ones = torch.zeros(2, dtype=torch.int32, device=DEV), torch.full((2,), 3.0, device=DEV)
    out = torch.empty_like(x)
    rules = aq._lib.LogitRules(tokens=ints.data_ptr(), token_lens=ints.data_ptr(), history=0,
                               repetition=ones.data_ptr(), bias_ids=ints.data_ptr(), bias_values=ones.data_ptr())
    st = aq._lib.load().aqlm_process_logits(x.data_ptr(), 100, out.data_ptr(), 100, 2, 2, 100, ctypes.byref(rules),
                                            torch.cuda.current_stream().cuda_stream)
    assert st == 0 and torch.equal(out, x)


def test_process_logits_special_values(aq):
    """NaN, infinities and the type's lowest value: masked places are -inf whatever they
    hold, the others follow the arithmetic."""
    x = torch.tensor([[math.nan, math.inf, -math.inf, -65504.0, 65504.0, 1.0, -1.0, 2.0] * 2], dtype=torch.float16)
    mask = torch.tensor([[0x00FF]], dtype=torch.int32)
    tokens = torch.arange(16, dtype=torch.int32)[None]
    got = aq.process_logits(x.to(DEV), tokens=tokens.to(DEV), token_lens=torch.tensor([16], dtype=torch.int32, device=DEV),
                            repetition=torch.tensor([2.0], device=DEV), mask=mask.to(DEV)).cpu()[0]
    assert (got[8:] == -math.inf).all()
    assert torch.isnan(got[0]) and got[1] == math.inf and got[2] == -math.inf and got[3] == -math.inf
    assert got[4:8].tolist() == [32752.0, 0.5, -2.0, 1.0]


# ---------------------------------------------------------------------------
# streams, graphs, refusals

def test_other_streams(aq):
    """On a stream of its own, with tensors made on another, and no workspace given."""
    bt, q = attend_case([900, 50], [1, 1], 8, 2, 128, 16, torch.float16)
    gpu = bt.gpu()
    dq = q.to(DEV)
    base = aq.paged_attention(dq, *gpu)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    outs = []
    for _ in range(20):
        outs.append(aq.paged_attention(dq, *gpu, stream=s))
        aq.paged_attention(dq, *gpu)
    with torch.cuda.stream(s):
        outs.append(aq.paged_attention(dq, *gpu))
    s.synchronize()
    torch.cuda.synchronize()
    assert all(torch.equal(o, base) for o in outs)


def test_decode_step_in_a_graph(aq):
    """append, attention and logits captured once, replayed with other lengths and inputs
    between eager calls: each replay equals the eager result."""
    kv, heads, dim, page, seqs, width, vocab = 2, 8, 128, 16, 3, 40, 3000
    g = torch.Generator(device=DEV).manual_seed(1)
    rnd = lambda *s: torch.randn(*s, generator=g, device=DEV).half()  # noqa: E731
    k, v = rnd(seqs * width, page, kv, dim), rnd(seqs * width, page, kv, dim)
    table = torch.randperm(seqs * width, generator=g, device=DEV).to(torch.int32).view(seqs, width)
    t = aq.rotary_table(width * page, dim)
    a, x = rnd(seqs, heads + 2 * kv, dim), rnd(seqs, vocab)
    lens = torch.tensor([1, 1, 1], dtype=torch.int32, device=DEV)
    cu = torch.arange(seqs + 1, dtype=torch.int32, device=DEV)
    hist = torch.randint(0, vocab, (seqs, 50), generator=g, device=DEV).to(torch.int32)
    n = torch.tensor([50, 20, 0], dtype=torch.int32, device=DEV)
    pen = torch.full((seqs,), 1.3, device=DEV)

    def step(k, v):
        q = aq.paged_append(a[:, :heads], a[:, heads:heads + kv], a[:, heads + kv:], k, v, table, lens, cu, table=t)
        o = aq.paged_attention(q, k, v, table, lens, cu, max_new=1)
        return o, aq.process_logits(x, tokens=hist, token_lens=n, repetition=pen)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step(k.clone(), v.clone())
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, logits = step(k, v)
    for r in range(5):
        lens.copy_(torch.tensor([3 + 100 * r, 600 - 7 * r, 0 if r == 2 else 129 * r + 1]))
        a.copy_(rnd(*a.shape))
        x.copy_(rnd(*x.shape))
        want = step(k.clone(), v.clone())
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(logits, want[1]), r


def test_no_tokens(aq):
    """Calls without tokens do nothing."""
    z = lambda *s: torch.zeros(*s, dtype=torch.float16, device=DEV)  # noqa: E731
    i = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)  # noqa: E731
    t = aq.rotary_table(4, 64)
    q, k = aq.rope(z(0, 4, 64), z(0, 2, 64), t, i(0))
    assert q.shape == (0, 4, 64) and k.shape == (0, 2, 64)
    w = torch.ones(64, dtype=torch.float16, device=DEV)
    g = aq.rope_backward(z(0, 4, 64), z(0, 2, 64), t, i(0), q=z(0, 4, 64), k=z(0, 2, 64), q_weight=w, k_weight=w)
    assert (g[2] == 0).all() and (g[3] == 0).all()
    c = (z(3, 16, 2, 64), z(3, 16, 2, 64), i(1, 3), i(1), i(2))
    assert aq.paged_append(z(0, 4, 64), z(0, 2, 64), z(0, 2, 64), *c).shape == (0, 4, 64)
    assert aq.paged_attention(z(0, 4, 64), *c).shape == (0, 4, 64)
    assert aq.process_logits(z(0, 100)).shape == (0, 100)


def test_refusals(aq):
    """Arguments that do not fit raise before anything runs."""
    z = lambda *s, **k: torch.zeros(*s, dtype=k.get("dtype", torch.float16), device=DEV)  # noqa: E731
    i = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)  # noqa: E731
    t = aq.rotary_table(4, 64)
    E = (ValueError, aq.AqlmError)
    good = (z(3, 4, 64), z(3, 2, 64), t, i(3))
    for bad in ((z(3, 64),) + good[1:], (good[0], z(2, 2, 64)) + good[2:], (good[0], z(3, 2, 32)) + good[2:],
                good[:2] + (t.half(),) + good[3:], good[:2] + (aq.rotary_table(4, 128),) + good[3:],
                good[:3] + (i(2),), good[:3] + (i(3).long(),), (good[0].cpu(),) + good[1:],
                (good[0].double(),) + good[1:], (z(3, 4, 128)[..., ::2],) + good[1:]):
        with pytest.raises(E):
            aq.rope(*bad)
    with pytest.raises(E):
        aq.rope(*good, q_weight=z(32))
    with pytest.raises(E):
        aq.rope(*good, q_weight=torch.ones(64, device=DEV))
    with pytest.raises(E):
        aq.rope(*good, out=(z(3, 4, 32), z(3, 2, 64)))
    with pytest.raises(E):
        aq.rope_backward(*good, q_weight=z(64))
    for kw in (dict(positions=0, rot=64), dict(positions=4, rot=63), dict(positions=4, rot=64, scaling={"kind": "x"}),
               dict(positions=4, rot=64, scaling={"kind": "linear", "factor": 0.0})):
        with pytest.raises(E):
            aq.rotary_table(**kw)
    cache = dict(k_cache=z(3, 16, 2, 64), v_cache=z(3, 16, 2, 64), block_table=i(1, 3), kv_lens=i(1), cu_new=i(2))
    for name, bad in (("k_cache", z(3, 12, 2, 64)), ("v_cache", z(3, 16, 1, 64)), ("block_table", i(1, 3).long()),
                      ("kv_lens", i(2)), ("cu_new", i(1)), ("v_cache", z(3, 16, 2, 64, dtype=torch.bfloat16)),
                      ("block_table", i(0, 3))):
        c = dict(cache, **{name: bad})
        with pytest.raises(E):
            aq.paged_attention(z(2, 4, 64), **c)
        with pytest.raises(E):
            aq.paged_append(z(2, 4, 64), z(2, 2, 64), z(2, 2, 64), **c)
    for page in (z(3, 12, 2, 64),):  # not a power of two, in both
        with pytest.raises(E):
            aq.paged_attention(z(2, 4, 64), **dict(cache, k_cache=page, v_cache=page))
    for q in (z(2, 3, 64), z(2, 4, 32), z(2, 4, 64, dtype=torch.bfloat16)):
        with pytest.raises(E):
            aq.paged_attention(q, **cache)
    with pytest.raises(E):
        aq.paged_attention(z(2, 4, 64), **cache, workspace=z(100))
    with pytest.raises(E):
        aq.paged_attention(z(2, 4, 64), **cache, window=-1)
    with pytest.raises(E):
        aq.paged_attention(z(2, 4, 64), **cache, scale=math.nan)
    odd = dict(cache, k_cache=z(3, 16, 2, 60), v_cache=z(3, 16, 2, 60))
    with pytest.raises(E):
        aq.paged_attention(z(2, 4, 60), **odd)
    with pytest.raises(E):
        aq.paged_append(z(2, 4, 64), z(2, 1, 64), z(2, 2, 64), **cache)
    x = z(2, 100)
    for kw in (dict(tokens=i(2, 4)), dict(repetition=torch.ones(2, device=DEV)), dict(bias_ids=i(2, 3)),
               dict(mask=i(2, 3)), dict(tokens=i(2, 4), token_lens=i(3)), dict(tokens=i(3, 4), token_lens=i(2)),
               dict(out=z(2, 99)), dict(bias_ids=i(2, 2048), bias_values=torch.zeros(2, 2048, device=DEV)),
               dict(tokens=i(2, 4).long(), token_lens=i(2))):
        with pytest.raises(E):
            aq.process_logits(x, **kw)
