"""The operators of ``block.py`` at the ends of what they take."""
import pytest

torch = pytest.importorskip("torch")

import block_reference as ref  # noqa: E402
from test_gpu_block import DEV, aq, rope_bound, within  # noqa: E402,F401

pytestmark = pytest.mark.gpu


def test_rope_of_many_heads(aq):
    """More heads than a launch may have waves along one axis (2^26), by the general kernel."""
    tokens, heads, kv, dim, dtype = (1 << 20) + 7, 60, 6, 2, torch.float16
    g = torch.Generator(device=DEV).manual_seed(3)
    a = torch.randn(tokens, heads + kv, dim, generator=g, device=DEV).half()
    t = ref.table64(100, dim).float()
    pos = (torch.arange(tokens, device=DEV) % 100).to(torch.int32)
    q, k = aq.rope(a[:, :heads], a[:, heads:], t.to(DEV), pos)
    x = torch.cat([q, k], 1)
    for at in (slice(0, 50), slice(1 << 19, (1 << 19) + 50), slice(tokens - 200, tokens)):
        want, size = ref.rope64(a[at].double().cpu(), None, t.double(), pos[at].long().cpu(), False, 1e-6)
        within(x[at], want, rope_bound(dtype, want, size))
    # a turn leaves each pair's length as it is (three roundings of two elements)
    length = lambda v: v.float().square().sum(-1)  # noqa: E731
    assert ((length(x) - length(a)).abs() <= 2.0 ** -8 * length(a) + 1e-6).all()
