"""Host-side checks of kmeans_linear_*, kmeans_fp8_*, kmeans_table_* and
kmeans_clip_* that need no GPU: refusals that come before any device call."""
import ctypes as C
import math

import pytest
import torch

import paper_1902_09527_amd as km
from paper_1902_09527_amd import _native as N

FAKE = C.c_void_p(0x1000)   # never read: the checks before it fail
ODD = C.c_void_p(0x1010)
BAD, UNS = N.KM_ERR_INVALID_ARG, N.KM_ERR_UNSUPPORTED


def _why():
    return N.load().kmeans_mti_last_hip_error().decode()


def test_linear_sizes():
    size = lambda n=100, di=64, do=32, k=4, t=1, b=0: N.load().kmeans_linear_workspace_bytes(n, di, do, k, t, b)
    assert all(size(t=t, b=b) > 0 for t in range(3) for b in (0, 1)) and size(n=0) > 0 and size(n=2 ** 27) > 0
    assert [size(n=-1), size(n=2 ** 31), size(di=0), size(do=0), size(k=0), size(t=3), size(t=-1)] == [0] * 7
    assert [size(n=2 ** 27 + 1), size(di=2 ** 24 + 1), size(do=2 ** 24 + 1)] == [0] * 3
    assert size(n=2 ** 27, di=2 ** 20, do=2 ** 20) == 0 and "tiles" in _why()


def test_linear_forward_refusals():
    lib = N.load()
    need = lib.kmeans_linear_workspace_bytes(100, 64, 32, 4, 1, 0)

    def f(X=FAKE, ldx=64, n=100, di=64, do=32, k=4, t=1, W=FAKE, order=FAKE, sids=FAKE, off=FAKE, Y=FAKE, ws=FAKE, wsb=need):
        return lib.kmeans_linear_forward(X, ldx, n, di, do, k, t, W, order, sids, off, Y, ws, wsb, None)
    assert [f(X=None), f(ldx=63), f(n=-1), f(di=0), f(do=0), f(k=0), f(t=3), f(W=None), f(sids=None), f(off=None),
            f(Y=None), f(ws=None), f(wsb=need - 1), f(ws=ODD), f(ldx=2 ** 62)] == [BAD] * 15
    assert f(n=2 ** 27 + 1) == UNS
    assert f(X=None, n=0, sids=None, off=None, Y=None, order=None) == N.KM_OK


def test_linear_backward_refusals():
    lib = N.load()
    need = lib.kmeans_linear_workspace_bytes(100, 64, 32, 4, 2, 1)

    def f(dY=FAKE, lddy=32, X=FAKE, ldx=64, n=100, t=2, W=FAKE, off=FAKE, dX=FAKE, dW=FAKE, ws=FAKE, wsb=need):
        return lib.kmeans_linear_backward(dY, lddy, X, ldx, n, 64, 32, 4, t, W, FAKE, off, dX, dW, ws, wsb, None)
    assert [f(dY=None), f(lddy=31), f(X=None), f(ldx=63), f(n=-1), f(t=5), f(W=None), f(off=None), f(ws=None),
            f(wsb=need - 1), f(ws=ODD), f(lddy=2 ** 62)] == [BAD] * 12
    assert f(n=2 ** 27 + 1) == UNS


def test_fp8_refusals():
    lib = N.load()
    q = lambda X=FAKE, ld=200, n=10, d=200, t=0, v=FAKE, e=FAKE: lib.kmeans_fp8_quantize(X, ld, n, d, t, v, e, None)
    assert [q(X=None), q(ld=199), q(n=-1), q(d=0), q(t=3), q(v=None), q(e=None), q(n=2 ** 40 + 1), q(ld=2 ** 62)] == [BAD] * 9
    assert q(n=0, X=None, v=None, e=None) == N.KM_OK
    u = lambda v=FAKE, e=FAKE, n=10, d=200, t=0, X=FAKE: lib.kmeans_fp8_dequantize(v, e, n, d, t, X, None)
    assert [u(v=None), u(e=None), u(n=-1), u(d=0), u(t=3), u(X=None), u(n=2 ** 40 + 1)] == [BAD] * 7
    size = lambda n=100, di=200, do=32, k=4, t=1: lib.kmeans_fp8_workspace_bytes(n, di, do, k, t)
    assert all(size(t=t) > 0 for t in range(4)) and size(t=1) > size(t=N.KM_E4M3)
    assert [size(n=-1), size(di=0), size(do=0), size(k=0), size(t=4), size(t=-1), size(n=2 ** 27 + 1)] == [0] * 7
    need = size()

    def f(X=FAKE, ld=200, e=None, n=100, t=1, W=FAKE, we=FAKE, sids=FAKE, off=FAKE, Y=FAKE, yt=1, ws=FAKE, wsb=need):
        return lib.kmeans_fp8_forward(X, ld, e, n, 200, 32, 4, t, W, we, FAKE, sids, off, Y, yt, ws, wsb, None)
    assert [f(X=None), f(ld=199), f(n=-1), f(t=4), f(t=N.KM_E4M3), f(W=None), f(we=None), f(sids=None), f(off=None),
            f(Y=None), f(yt=3), f(ws=None), f(wsb=need - 1), f(ws=ODD)] == [BAD] * 14
    assert f(n=2 ** 27 + 1) == UNS


def test_table_refusals():
    lib = N.load()

    def f(ids=FAKE, n=10, k=5, d=8, t=0, table=FAKE, ld=8, scale=1.0, Y=FAKE):
        return lib.kmeans_table_forward(ids, n, k, d, t, table, ld, scale, Y, None)
    assert [f(ids=None), f(n=-1), f(k=0), f(d=0), f(t=3), f(table=None), f(ld=7), f(scale=math.nan), f(scale=math.inf),
            f(Y=None), f(ld=2 ** 62)] == [BAD] * 11
    assert f(n=0, ids=None, Y=None, table=None) == N.KM_OK
    size = lib.kmeans_table_workspace_bytes
    assert size(0, 5, 8, 0) > 0 and size(10, 5, 8, 2) > 0
    assert [size(-1, 5, 8, 0), size(2 ** 31, 5, 8, 0), size(10, 0, 8, 0), size(10, 5, 0, 0), size(10, 5, 8, 3)] == [0] * 5
    need = size(1000, 5, 8, 0)

    def b(dY=FAKE, ld=8, n=1000, k=5, d=8, t=0, order=FAKE, sids=FAKE, off=FAKE, scale=1.0, out=FAKE, ws=FAKE, wsb=need):
        return lib.kmeans_table_backward(dY, ld, n, k, d, t, order, sids, off, scale, out, ws, wsb, None)
    assert [b(dY=None), b(ld=7), b(n=-1), b(k=0), b(d=0), b(t=3), b(order=None), b(sids=None), b(off=None),
            b(scale=math.nan), b(out=None), b(ws=None), b(wsb=need - 1), b(ws=ODD), b(ld=2 ** 62)] == [BAD] * 15


def test_clip_refusals():
    lib = N.load()
    sizes = lambda *s: (C.c_int64 * len(s))(*s)
    size = lambda *s: lib.kmeans_clip_workspace_bytes(sizes(*s), len(s))
    assert size(5, 0, 7) > 0 and lib.kmeans_clip_workspace_bytes(None, 0) > 0
    assert size(5, -1) == 0 and size(2 ** 40, 1) == 0 and size(2 ** 62, 2 ** 62) == 0
    assert lib.kmeans_clip_workspace_bytes(None, 2) == 0 and lib.kmeans_clip_workspace_bytes(sizes(1), -1) == 0
    p, need = (C.c_void_p * 2)(0x1000, 0x2000), size(5, 7)

    def f(ts=p, out=None, s=sizes(5, 7), types=(C.c_int32 * 2)(0, 0), count=2, limit=1.0, norm=FAKE, ws=FAKE, wsb=need):
        return lib.kmeans_clip_norm(ts, out, s, types, count, limit, norm, ws, wsb, None)
    assert [f(ts=None), f(s=None), f(types=None), f(count=-1), f(norm=None), f(ws=None), f(wsb=need - 1), f(ws=ODD),
            f(out=p, limit=0.0), f(out=p, limit=-1.0), f(out=p, limit=math.nan), f(s=sizes(5, -7))] == [BAD] * 12


def test_binding_rejects_cpu_tensors():
    x, i = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32)
    w, plan = torch.zeros(2, 8, 8), km.ClusterPlan(i, i, i, torch.zeros(3, dtype=torch.int32), 4, 1, 2)
    q = km.BlockRows(x.to(torch.float8_e4m3fn), torch.ones(4, 1, dtype=torch.uint8))
    for call in (lambda: km.cluster_linear(x, w, plan), lambda: km.cluster_linear_backward(x, x, w, plan),
                 lambda: km.quantize_blocks(x), lambda: km.quantize_blocks(torch.zeros(2, 3, 0)), lambda: km.dequantize_blocks(q),
                 lambda: km.cluster_linear_fp8(x, km.BlockRows(w, w), plan), lambda: km.cluster_embedding(i, x),
                 lambda: km.cluster_embedding_backward(x, plan), lambda: km.global_norm([x]),
                 lambda: km.clip_global_norm([x], 1.0)):
        with pytest.raises(ValueError):
            call()
