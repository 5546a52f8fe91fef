"""Tensors of the caller that the operators of ``block.py`` write count as modified in place."""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_block import DEV, aq, rand  # noqa: E402,F401

pytestmark = pytest.mark.gpu


def test_written_tensors_count_as_modified(aq):
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    q, k, v = rand(1, 3, 4, 64).to(DEV), rand(2, 3, 2, 64).to(DEV), rand(3, 3, 2, 64).to(DEV)
    oq, ok, x = torch.empty_like(q), torch.empty_like(k), rand(4, 3, 100).to(DEV)
    kc, vc = (torch.zeros(2, 16, 2, 64, dtype=torch.float16, device=DEV) for _ in range(2))
    where = (kc, vc, ints([[0]]), ints([3]), ints([0, 3]))
    table, pos = aq.rotary_table(8, 64), ints([0, 1, 2])
    calls = [
        (lambda: aq.rope(q, k, table, pos, out=(oq, ok)), (oq, ok), (q, k, table, pos)),
        (lambda: aq.rope_backward(q, k, table, pos, out=(oq, ok)), (oq, ok), (q, k)),
        (lambda: aq.paged_append(q, k, v, *where, out=oq), (oq, kc, vc), (q, k, v)),
        (lambda: aq.paged_append(None, k, v, *where), (kc, vc), (k, v)),
        (lambda: aq.paged_attention(q, *where, out=oq), (oq,), (q, kc, vc)),
        (lambda: aq.process_logits(x, out=x), (x,), ()),
    ]
    for call, changed, kept in calls:
        before = [[t._version for t in ts] for ts in (changed, kept)]
        call()
        assert all(t._version > n for t, n in zip(changed, before[0]))
        assert all(t._version == n for t, n in zip(kept, before[1]))
    # a result that autograd has saved
    w = x.float().requires_grad_()
    y = w.exp()
    aq.process_logits(y.detach(), out=y.detach())
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_inference_tensors(aq):
    """Tensors that have no version are written as well."""
    with torch.inference_mode():
        x = rand(4, 3, 100).to(DEV)
        y = torch.zeros_like(x)
        aq.process_logits(x, out=y)
        assert torch.equal(x, y)
