"""Host-side checks of the C ABI of the operators around a block's products:
bad arguments are refused before anything is launched (fake pointers suffice)."""
import ctypes
import os

import pytest

from paper_2401_06118_amd import _lib

OK, NULL, SHAPE, UNSUP, ALIGN, WORKSPACE = 0, 1, 2, 3, 4, 6
P = 0x10000
F16, BF16, F32 = 0, 1, 2


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_lib.LIB_PATH):
        pytest.skip("library not built (run python -m paper_2401_06118_amd.build)")
    return _lib.load()


def heads(n=4, data=P, token=512, head=64):
    return _lib.Heads(data, token, head, n)


def rotation(table=P, rows=100, rot=64, inter=0, qw=None, kw=None):
    return _lib.Rotation(table, rows, rot, inter, qw, kw, 1e-6)


def cache(**kw):
    d = dict(k=P, v=P, k_page_stride=2048, k_slot_stride=128, k_head_stride=64, v_page_stride=2048, v_slot_stride=128,
             v_head_stride=64, pages=10, block_table=P, table_stride=8, kv_lens=P, cu_new=P, table_width=8, seqs=3,
             page_size=16, kv_heads=2, head_dim=64, dtype=F16)
    d.update(kw)
    return _lib.PagedCache(**d)


def ref(x):
    return None if x is None else ctypes.byref(x)


def rope(lib, q=heads(), k=heads(2), qo=heads(), ko=heads(2), dtype=F16, tokens=3, dim=64, pos=P, r=rotation()):
    return lib.aqlm_rope(ref(q), ref(k), ref(qo), ref(ko), dtype, tokens, dim, pos, ref(r), None)


def test_rope(lib):
    for kw in (dict(q=None), dict(k=None), dict(qo=None), dict(ko=None), dict(r=None), dict(pos=None),
               dict(q=heads(data=None)), dict(ko=heads(2, data=None)), dict(r=rotation(table=None))):
        assert rope(lib, **kw) == NULL, kw
    for kw in (dict(tokens=-1), dict(tokens=1 << 31), dict(dim=0), dict(dim=1025), dict(q=heads(0)), dict(qo=heads(3)),
               dict(q=heads(token=-1)), dict(qo=heads(token=8)), dict(ko=heads(2, head=32)), dict(r=rotation(rot=63)),
               dict(r=rotation(rot=66)), dict(r=rotation(rot=-2)), dict(r=rotation(rows=0)),
               dict(tokens=1 << 29, q=heads(token=512))):
        assert rope(lib, **kw) == SHAPE, kw
    assert rope(lib, dtype=3) == UNSUP and rope(lib, dtype=-1) == UNSUP
    for kw in (dict(q=heads(data=P + 1)), dict(dtype=F32, qo=heads(data=P + 2)), dict(pos=P + 2),
               dict(r=rotation(table=P + 4)), dict(r=rotation(qw=P + 1))):
        assert rope(lib, **kw) == ALIGN, kw
    assert rope(lib, tokens=0, pos=None, q=heads(data=None)) == OK


def test_rope_backward(lib):
    need = lib.aqlm_rope_backward_workspace_bytes(64)
    assert need > 0 and lib.aqlm_rope_backward_workspace_bytes(0) == 0 == lib.aqlm_rope_backward_workspace_bytes(1025)

    def call(dq=heads(), dk=heads(2), q=heads(), k=heads(2), gq=heads(), gk=heads(2), wq=P, wk=P, dtype=F16, tokens=3,
             dim=64, pos=P, r=rotation(qw=P, kw=P), ws=P, ws_bytes=need):
        return lib.aqlm_rope_backward(ref(dq), ref(dk), ref(q), ref(k), ref(gq), ref(gk), wq, wk, dtype, tokens, dim,
                                      pos, ref(r), ws, ws_bytes, None)

    for kw in (dict(dq=None), dict(gk=None), dict(q=None), dict(k=None), dict(wq=None), dict(wk=None), dict(ws=None),
               dict(pos=None), dict(r=None)):
        assert call(**kw) == NULL, kw
    for kw in (dict(tokens=0), dict(dim=0), dict(gq=heads(5)), dict(q=heads(5)), dict(gk=heads(2, head=8))):
        assert call(**kw) == SHAPE, kw
    assert call(dtype=7) == UNSUP
    assert call(ws_bytes=need - 1) == WORKSPACE
    assert call(ws=P + 8) == ALIGN and call(wq=P + 2) == ALIGN and call(k=heads(2, data=P + 1)) == ALIGN


def test_rotary_table(lib):
    f = lib.aqlm_rotary_table
    assert f(None, 4, 4, 1.0, P, None) == NULL and f(P, 4, 4, 1.0, None, None) == NULL
    assert f(P, 0, 4, 1.0, P, None) == SHAPE and f(P, 4, 0, 1.0, P, None) == SHAPE
    assert f(P, 1 << 31, 4, 1.0, P, None) == SHAPE
    assert f(P + 4, 4, 4, 1.0, P, None) == ALIGN and f(P, 4, 4, 1.0, P + 4, None) == ALIGN


BAD_CACHE = [
    (NULL, dict(k=None)), (NULL, dict(v=None)), (NULL, dict(block_table=None)), (NULL, dict(kv_lens=None)),
    (NULL, dict(cu_new=None)), (SHAPE, dict(pages=0)), (SHAPE, dict(pages=1 << 31)), (SHAPE, dict(table_width=0)),
    (SHAPE, dict(table_stride=-1)), (SHAPE, dict(seqs=0)), (SHAPE, dict(seqs=4097)), (SHAPE, dict(page_size=12)),
    (SHAPE, dict(page_size=0)), (SHAPE, dict(page_size=-16)), (SHAPE, dict(kv_heads=0)), (SHAPE, dict(head_dim=0)),
    (SHAPE, dict(k_page_stride=-8)), (SHAPE, dict(v_head_stride=-8)), (SHAPE, dict(table_width=1 << 20, page_size=2048)),
    (UNSUP, dict(dtype=5)), (ALIGN, dict(block_table=P + 2)), (ALIGN, dict(k=P + 1)),
]


@pytest.mark.parametrize("status,kw", BAD_CACHE)
def test_cache(lib, status, kw):
    c = cache(**kw)
    assert lib.aqlm_paged_append(None, ref(heads(2)), ref(heads(2)), None, ref(c), 3, ref(rotation()), None) == status
    need = lib.aqlm_paged_attention_workspace_bytes(64)
    assert lib.aqlm_paged_attention(ref(heads()), ref(heads()), None, ref(c), 3, 0, 1.0, 1, 0, P, need, None) == status


def test_paged_append(lib):
    def call(q=heads(), k=heads(2), v=heads(2), qo=heads(), c=cache(), tokens=3, r=rotation()):
        return lib.aqlm_paged_append(ref(q), ref(k), ref(v), ref(qo), ref(c), tokens, ref(r), None)
    for kw in (dict(k=None), dict(v=None), dict(c=None), dict(r=None), dict(q=None), dict(qo=None)):
        assert call(**kw) == NULL, kw
    for kw in (dict(k=heads(3)), dict(v=heads(1)), dict(tokens=-1), dict(qo=heads(3)), dict(r=rotation(rot=66)),
               dict(qo=heads(head=32)), dict(c=cache(head_dim=1032))):
        assert call(**kw) == SHAPE, kw
    assert call(q=heads(data=P + 1)) == ALIGN
    assert call(tokens=0) == OK


def test_paged_attention(lib):
    assert lib.aqlm_paged_attention_workspace_bytes(0) == 0
    assert lib.aqlm_paged_attention_workspace_bytes(60) == 0
    assert lib.aqlm_paged_attention_workspace_bytes(264) == 0
    need = lib.aqlm_paged_attention_workspace_bytes(64)

    def call(q=heads(), out=heads(), lse=None, c=cache(), tokens=3, most=0, scale=1.0, causal=1, window=0, ws=P, n=need):
        return lib.aqlm_paged_attention(ref(q), ref(out), lse, ref(c), tokens, most, scale, causal, window, ws, n, None)
    for kw in (dict(q=None), dict(out=None), dict(c=None), dict(ws=None), dict(q=heads(data=None))):
        assert call(**kw) == NULL, kw
    for kw in (dict(tokens=-1), dict(most=-1), dict(window=-1), dict(scale=float("nan")), dict(scale=float("inf")),
               dict(scale=3e38), dict(q=heads(3)), dict(out=heads(2)), dict(out=heads(head=32)),
               dict(tokens=1 << 29), dict(tokens=1 << 27, c=cache(table_width=1 << 20))):
        assert call(**kw) == SHAPE, kw
    assert call(c=cache(dtype=F32)) == UNSUP
    assert call(c=cache(head_dim=60)) == UNSUP
    assert call(c=cache(head_dim=264)) == UNSUP
    for kw in (dict(q=heads(data=P + 8)), dict(out=heads(token=516)), dict(c=cache(k=P + 8)),
               dict(c=cache(v_slot_stride=132)), dict(ws=P + 8), dict(lse=P + 2)):
        assert call(**kw) == ALIGN, kw
    assert call(n=need - 1) == WORKSPACE
    assert call(tokens=0) == OK


def test_process_logits(lib):
    def call(x=P, xs=100, out=P, os_=100, dtype=F16, rows=2, vocab=100, **kw):
        r = _lib.LogitRules(**kw)
        return lib.aqlm_process_logits(x, xs, out, os_, dtype, rows, vocab, ctypes.byref(r), None)
    assert lib.aqlm_process_logits(P, 100, P, 100, F16, 2, 100, None, None) == NULL
    for kw in (dict(x=None), dict(out=None), dict(tokens=P), dict(repetition=P), dict(presence=P), dict(bias_ids=P),
               dict(bias_values=P)):
        assert call(**kw) == NULL, kw
    for kw in (dict(rows=-1), dict(rows=65536), dict(vocab=0), dict(vocab=1 << 31), dict(xs=-1), dict(os_=99),
               dict(tokens=P, token_lens=P, history=-1), dict(tokens=P, token_lens=P, history=1 << 20),
               dict(tokens=P, token_lens=P, token_stride=-1), dict(bias_ids=P, bias_values=P, biases=2048),
               dict(bias_ids=P, bias_values=P, biases=-1), dict(mask=P, mask_stride=-1)):
        assert call(**kw) == SHAPE, kw
    assert call(dtype=3) == UNSUP
    for kw in (dict(x=P + 1), dict(dtype=F32, out=P + 2), dict(mask=P + 2), dict(tokens=P + 1, token_lens=P)):
        assert call(**kw) == ALIGN, kw
    assert call(rows=0, x=None) == OK
