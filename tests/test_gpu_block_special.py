"""NaN and infinities through the operators of ``block.py``, against their definitions in 64 bits."""
import math

import pytest

torch = pytest.importorskip("torch")

import block_reference as ref  # noqa: E402
from test_gpu_block import DEV, attend_case, aq, check_attention, rand  # noqa: E402,F401

pytestmark = pytest.mark.gpu


def both_kernels(aq, bt, q, causal=True, window=0, scale=None):
    """A hint of one new token takes the kernel of a few rows, none the one of many (more than 16 rows)."""
    for most in (1, 0):
        check_attention(aq, bt, q, causal, window, scale=scale, max_new=most)


NAN_QUERIES = [([1], [1]), ([40], [1]), ([300, 90], [1, 1]), ([20000], [1]), ([300, 90], [30, 8]), ([6000], [40])]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("lens,new", NAN_QUERIES)
def test_nan_query(aq, lens, new, dtype):
    """Rows whose query holds a NaN are NaN, their lse too, however the keys are divided; the others are theirs."""
    bt, q = attend_case(lens, new, 4, 2, 128, 16, dtype)
    q[0, 1, 5] = math.nan
    q[-1, 2] = math.nan
    both_kernels(aq, bt, q)


NAN_KEYS = [
    # lens, new, first and last NaN key, window
    ([64], [1], 0, 64, 0),             # all keys
    ([300], [1], 32, 64, 0),           # all of a wave's
    ([20000, 50], [1, 1], 4000, 9000, 0),
    ([6000], [40], 1000, 3000, 0),
    ([6000], [40], 0, 6000, 0),
    ([300], [40], 250, 262, 50),       # seen by some rows
    ([300], [40], 290, 300, 0),
]


@pytest.mark.parametrize("lens,new,begin,end,window", NAN_KEYS)
def test_nan_keys(aq, lens, new, begin, end, window):
    """A run of NaN keys makes the rows that see one of them NaN, and no others."""
    bt, q = attend_case(lens, new, 4, 2, 64, 16, torch.bfloat16)
    for j in range(begin, end):
        bt.k[int(bt.table[0, j // 16]), j % 16] = math.nan
    both_kernels(aq, bt, q, window=window)


INF_VALUES = [([1], [1]), ([40], [1]), ([300, 90], [1, 1]), ([20000], [1]), ([300, 90], [30, 8]), ([6000], [40])]


def put_infinities(bt):
    """Of the first sequence's first kv head: +inf, -inf and both in columns of their own."""
    n = bt.lens[0]
    for j, d, v in ((5, 3, math.inf), (7, 3, math.inf), (9, 8, -math.inf), (11, 20, math.inf), (2 * n // 3, 20, -math.inf),
                    (n - 2, 40, -math.inf)):
        j = min(max(j, 0), n - 1)
        bt.v[int(bt.table[0, j // 16]), j % 16, 0, d] = v


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens,new", INF_VALUES)
def test_infinite_values(aq, lens, new, causal, dtype):
    """Infinite values of keys that all rows see: an infinite element, NaN where both signs meet."""
    bt, q = attend_case(lens, new, 4, 2, 64, 16, dtype)
    put_infinities(bt)
    both_kernels(aq, bt, q, causal=causal)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim", [64, 128, 200, 256])
@pytest.mark.parametrize("lens,new", [([300], [1]), ([300, 90], [30, 8]), ([2000], [40])])
def test_infinite_values_of_small_weight(aq, lens, new, dim, dtype):
    """However small a weight is, times an infinite value it is infinite."""
    bt, q = attend_case(lens, new, 4, 2, dim, 16, dtype)
    for i in range(40):
        j = i * (lens[0] - new[0] - 1) // 40
        bt.v[int(bt.table[0, j // 16]), j % 16, i % 2, i] = math.inf if i % 3 else -math.inf
    both_kernels(aq, bt, q, scale=0.75 * (64 / dim) ** 0.5)


UNROTATED = [(64, 32), (64, 4), (64, 6), (128, 64), (80, 40), (256, 252)]


def put_outside(x, rot, dim):
    """Infinities and NaN in the part that is not rotated, each beside a number of its pair."""
    for t, d, v in ((0, rot, math.inf), (1, dim - 1, -math.inf), (2, rot + 2, math.nan), (3, rot + 1, math.inf)):
        x[t, t % x.shape[1], d] = v


def same_bits(got, want):
    kind = torch.int32 if want.dtype == torch.float32 else torch.int16
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan)
    assert torch.equal(got.contiguous().view(kind)[~nan], want.contiguous().view(kind)[~nan])


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dim,rot", UNROTATED)
def test_interleaved_rotation_leaves_the_rest(aq, dim, rot, dtype):
    """Elements past the rotated part come back as they are, and reach no others: forward, gradient and cache."""
    a = rand(5, 4, 4, dim, dtype=dtype)
    put_outside(a, rot, dim)
    t = ref.table64(50, rot).float()
    pos = torch.tensor([0, 3, 49, 7], dtype=torch.int32)
    d, dt = a.to(DEV), t.to(DEV)
    q, k = aq.rope(d[:, :2], d[:, 2:], dt, pos.to(DEV), interleaved=True)
    g = aq.rope_backward(d[:, :2], d[:, 2:], dt, pos.to(DEV), interleaved=True)
    for got in (torch.cat([q, k], 1), torch.cat(g[:2], 1)):
        same_bits(got.cpu()[..., rot:], a[..., rot:])
        assert torch.isfinite(got[..., :rot]).all()
    kc, vc = (torch.zeros(2, 16, 2, dim, dtype=dtype, device=DEV) for _ in range(2))
    where = (kc, vc, *(torch.tensor(v, dtype=torch.int32, device=DEV) for v in ([[1]], [4], [0, 4])))
    for table in (dt, None):
        first = rot if table is not None else 0
        q = aq.paged_append(d[:, :2], d[:, 2:], d[:, 2:], *where, table=table, interleaved=True)
        same_bits(q.cpu()[..., first:], a[:, :2, first:])
        same_bits(kc[1, :4].cpu()[..., first:], a[:, 2:, first:])
        same_bits(vc[1, :4].cpu(), a[:, 2:])
        assert torch.isfinite(q[..., :first]).all() and torch.isfinite(kc[1, :4, :, :first]).all()
