"""Host-side checks of the operators of ``ends.py``: the C ABI refuses bad arguments before
anything is launched (fake pointers suffice), the Python module bad tensors."""
import ctypes
import math
import os

import pytest

from paper_2401_06118_amd import _lib

OK, NULL, SHAPE, UNSUP, ALIGN, WORKSPACE = 0, 1, 2, 3, 4, 6
P, Q = 0x10000, 0x20000
F16, BF16, F32 = 0, 1, 2
BIG = 1 << 62


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_lib.LIB_PATH):
        pytest.skip("library not built (run python -m paper_2401_06118_amd.build)")
    return _lib.load()


def refused(call, status, **changes):
    for name, values in changes.items():
        for v in values:
            assert call(**{name: v}) == status, (name, v)


def test_embed(lib):
    def call(table=P, ts=64, tokens=P, out=Q, os=64, dtype=F16, count=3, vocab=10, dim=64):
        return lib.aqlm_embed(table, ts, tokens, out, os, dtype, count, vocab, dim, 1.0, None)

    refused(call, NULL, table=[None], tokens=[None], out=[None])
    refused(call, SHAPE, ts=[-1], os=[-1, 63], count=[-1, (1 << 31) - 1], vocab=[0, -1, (1 << 30) + 1],
            dim=[0, -4, (1 << 24) + 1])
    refused(call, UNSUP, dtype=[-1, 3])
    refused(call, ALIGN, table=[P + 1], out=[Q + 1], tokens=[P + 2])
    assert call(dtype=F32, table=P + 2) == ALIGN
    assert call(count=0, table=None, tokens=None, out=None) == OK


def test_embed_backward(lib):
    room = lib.aqlm_embed_backward_workspace_bytes
    need = room(3, 10, 64, F16)
    assert need > 0 and room(0, 10, 64, F16) > 0 and room(100000, 10, 64, F16) > room(1000, 10, 64, F16)
    for bad in ((-1, 10, 64, F16), (3, 10, 0, F16), (3, 10, (1 << 24) + 1, F16), (3, 10, 64, 7), (1 << 31, 10, 64, F16),
                (3, 0, 64, F16), (3, (1 << 30) + 1, 64, F16)):
        assert room(*bad) == 0

    def call(dout=P, ds=64, tokens=P, grad=Q, gs=64, dtype=F16, gtype=F16, count=3, vocab=10, dim=64, ws=P, size=need):
        return lib.aqlm_embed_backward(dout, ds, tokens, grad, gs, dtype, gtype, count, vocab, dim, 1.0, ws, size, None)

    refused(call, NULL, dout=[None], tokens=[None], grad=[None], ws=[None])
    refused(call, SHAPE, ds=[-1], gs=[-1, 63], count=[-1, 1 << 31], vocab=[0], dim=[0])
    refused(call, UNSUP, dtype=[3], gtype=[BF16, 3])
    refused(call, ALIGN, dout=[P + 1], grad=[Q + 1], tokens=[P + 1], ws=[P + 8])
    refused(call, WORKSPACE, size=[0, need - 1])
    assert call(gtype=F32, grad=Q + 2) == ALIGN


def test_layer_norm(lib):
    def call(x=P, xs=64, r=None, rs=0, out=Q, os=64, s=None, ss=0, dtype=F16, rows=3, dim=64, n=(None, None, 1e-5, 0)):
        n = None if n is None else ctypes.byref(_lib.Norm(*n))
        return lib.aqlm_layer_norm(x, xs, r, rs, out, os, s, ss, dtype, rows, dim, n, None)

    refused(call, NULL, x=[None], out=[None], n=[None], s=[P])
    refused(call, SHAPE, xs=[-1], os=[-1, 63], rows=[-1], dim=[0, -1, 16385],
            n=[(None, None, -1.0, 0), (None, None, math.nan, 0)])
    refused(call, UNSUP, dtype=[-1, 3])
    refused(call, ALIGN, x=[P + 1], out=[Q + 1], r=[P + 1], n=[(P + 1, None, 0.0, 0), (None, P + 1, 0.0, 1)])
    assert call(r=P, rs=64, s=Q, ss=64) == SHAPE  # both results in one place
    assert call(r=P, rs=64, s=P, ss=32) == SHAPE and call(r=P, rs=-1, s=P, ss=64) == SHAPE
    assert call(rows=0, x=None, out=None) == OK


def test_layer_norm_backward(lib):
    need = lib.aqlm_layer_norm_backward_workspace_bytes(64)
    assert need > 0 and [lib.aqlm_layer_norm_backward_workspace_bytes(d) for d in (0, -1, 16385)] == [0, 0, 0]

    def call(dy=P, dys=64, x=P, xs=64, ds=None, dss=0, dx=Q, dxs=64, dw=P, db=None, dtype=F16, rows=3, dim=64,
             n=(None, None, 1e-5, 0), ws=P, size=need):
        n = None if n is None else ctypes.byref(_lib.Norm(*n))
        return lib.aqlm_layer_norm_backward(dy, dys, x, xs, ds, dss, dx, dxs, dw, db, dtype, rows, dim, n, ws, size, None)

    refused(call, NULL, dy=[None], x=[None], dx=[None], n=[None], ws=[None])
    refused(call, SHAPE, dys=[-1], xs=[-1], dxs=[-1, 63], rows=[-1], dim=[0, 16385], n=[(None, None, -1.0, 0)])
    refused(call, UNSUP, dtype=[3])
    refused(call, ALIGN, dy=[P + 1], x=[P + 1], dx=[Q + 1], ds=[P + 1], dw=[P + 2], db=[P + 2], ws=[P + 8],
            n=[(P + 1, None, 0.0, 0)])
    refused(call, WORKSPACE, size=[0, need - 1])
    assert call(ds=P, dss=-1) == SHAPE
    assert call(rows=0, dw=None, dy=None, x=None, dx=None, ws=None) == OK


def test_distill_loss(lib):
    def call(z=P, zs=1000, dtype=F16, t=P, tstride=8, tt=F32, ids=P, ids_s=8, lse=None, w=None, tau=1.0, loss=P, grad=Q,
             gs=1000, rows=3, vocab=1000, listed=8, ws=P, size=1 << 20):
        return lib.aqlm_distill_loss(z, zs, dtype, t, tstride, tt, ids, ids_s, lse, w, tau, loss, grad, gs, rows, vocab,
                                     listed, ws, size, None)

    room = lib.aqlm_distill_loss_workspace_bytes
    assert 0 < room(3, 1000, 8, F16) < room(3, 1000, 9, F16) and room(1 << 20, 1000, 8, F16) == 0
    assert [room(*v) for v in ((0, 1000, 8, F16), (3, 0, 8, F16), (3, 1000, 0, F16), (3, 1000, 8, 5))] == [0] * 4
    refused(call, NULL, ws=[None])
    refused(call, WORKSPACE, size=[0, room(3, 1000, 8, F16) - 1])
    refused(call, ALIGN, ws=[P + 8])

    refused(call, NULL, z=[None], t=[None], ids=[None], loss=[None])
    refused(call, SHAPE, zs=[-1], tstride=[-1], ids_s=[-1], gs=[-1, 999], rows=[-1, 1 << 22], vocab=[0, (1 << 19) + 1],
            listed=[0, -1, 2049], tau=[0.0, -1.0, math.nan, math.inf, 1e-45])
    refused(call, UNSUP, dtype=[3], tt=[-1])
    refused(call, ALIGN, z=[P + 1], t=[P + 2], grad=[Q + 1], ids=[P + 1], lse=[P + 2], w=[P + 1], loss=[P + 2])
    assert call(rows=0, z=None) == OK


def test_sample(lib):
    def room(rows, vocab, *r):
        return lib.aqlm_sample_workspace_bytes(rows, vocab, ctypes.byref(_lib.Sampling(*r)))

    need = room(3, 40000)
    assert need > 0 and room(6, 40000) == 2 * need and room(3, 40000, None, P) == need
    assert [room(*v) for v in ((3, 8192), (3, 32768, None, P), (0, 40000), (-1, 40000), (3, (1 << 19) + 1))] == [0] * 5
    assert room(1 << 20, 40000) < 1 << 26 and lib.aqlm_sample_workspace_bytes(3, 40000, None) == 0  # (rows in turn)

    def call(z=P, zs=40000, dtype=F16, rows=3, vocab=40000, u=P, r=(None, None, None, None), tokens=P, lp=None, ws=P,
             size=need):
        r = None if r is None else ctypes.byref(_lib.Sampling(*r))
        return lib.aqlm_sample(z, zs, dtype, rows, vocab, u, r, tokens, lp, ws, size, None)

    refused(call, NULL, z=[None], u=[None], r=[None], tokens=[None], ws=[None])
    refused(call, WORKSPACE, size=[0, need - 1])
    refused(call, SHAPE, zs=[-1], rows=[-1, (1 << 20) + 1], vocab=[0, -1, (1 << 19) + 1, BIG])
    refused(call, UNSUP, dtype=[3])
    refused(call, ALIGN, z=[P + 1], u=[P + 2], tokens=[P + 1], lp=[P + 2], ws=[P + 8],
            r=[(P + 1, None, None, None), (None, P + 1, None, None), (None, None, P + 1, None), (None, None, None, P + 1)])
    assert call(rows=0, z=None) == OK


def test_python_refuses_host_tensors():
    torch = pytest.importorskip("torch")
    from paper_2401_06118_amd import block

    if not os.path.exists(os.path.join(os.path.dirname(block.__file__), "_block.so")):
        pytest.skip("binding not built")
    import paper_2401_06118_amd as aq

    x, i, f = torch.zeros(3, 8), torch.zeros(3, dtype=torch.int32), torch.zeros(3)
    for call in (lambda: aq.embed(x, i), lambda: aq.embed_backward(x, i, 9), lambda: aq.layer_norm(x),
                 lambda: aq.layer_norm_backward(x, x), lambda: aq.distill_loss(x, x, i), lambda: aq.sample(x, f)):
        with pytest.raises(ValueError, match="must be a GPU tensor"):
            call()
