"""Host-side checks of include/kmeans_ops.h that need no GPU: the exports, and
refusals that come before any device call."""
import ctypes as C
import math
import os
import re

import pytest

from paper_1902_09527_amd import _native as N

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = C.c_void_p(0x1000)   # never read: the checks before it fail
BAD = N.KM_ERR_INVALID_ARG


def test_header_declares_the_binding_exports():
    text = open(os.path.join(ROOT, "include", "kmeans_ops.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    assert sorted(set(re.findall(r"\b(kmeans_\w+)\s*\(", text))) == sorted(N.OPS_EXPORTS)
    for name in N.OPS_EXPORTS:
        assert hasattr(N.load(), name), name


def test_sort_refusals():
    lib = N.load()
    assert lib.kmeans_sort_workspace_bytes(10, 2, 4) > 0
    for n, m, k in ((-1, 1, 1), (1, 0, 1), (1, 1, 0), (2 ** 31, 1, 4), (2 ** 30, 2, 4), (1, 1, 2 ** 31 - 1)):
        assert lib.kmeans_sort_workspace_bytes(n, m, k) == 0
        assert lib.kmeans_sort_plan(FAKE, n, m, k, FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 20, None) == BAD
        assert lib.kmeans_sort_gather(FAKE, 8, n, m, k, 8, 0, FAKE, FAKE, FAKE, None) == BAD
    need = lib.kmeans_sort_workspace_bytes(5000, 1, 4)
    assert lib.kmeans_sort_plan(FAKE, 5000, 1, 4, FAKE, FAKE, FAKE, FAKE, FAKE, need - 1, None) == BAD
    assert lib.kmeans_sort_plan(FAKE, 5000, 1, 4, FAKE, FAKE, FAKE, FAKE, C.c_void_p(0x1008), need, None) == BAD
    assert b"workspace" in lib.kmeans_mti_last_hip_error()
    assert lib.kmeans_sort_plan(None, 5, 1, 4, FAKE, FAKE, FAKE, FAKE, FAKE, 256, None) == BAD
    assert lib.kmeans_sort_gather(FAKE, 7, 4, 1, 4, 8, 0, FAKE, FAKE, FAKE, None) == BAD       # ldx < d
    assert lib.kmeans_sort_gather(FAKE, 8, 4, 1, 4, 0, 0, FAKE, FAKE, FAKE, None) == BAD       # d
    assert lib.kmeans_sort_gather(FAKE, 8, 4, 1, 4, 8, 3, FAKE, FAKE, FAKE, None) == BAD       # type
    assert lib.kmeans_sort_gather(FAKE, 2 ** 62, 4, 1, 4, 8, 0, FAKE, FAKE, FAKE, None) == BAD
    assert lib.kmeans_sort_gather(None, 8, 4, 1, 4, 8, 0, FAKE, FAKE, FAKE, None) == BAD
    assert lib.kmeans_sort_combine(FAKE, 8, 4, 1, 4, 8, 0, None, FAKE, None, FAKE, None) == BAD
    assert lib.kmeans_sort_combine_backward(FAKE, 8, None, 8, 4, 1, 4, 8, 0, FAKE, FAKE, FAKE, FAKE, FAKE,
                                            None) == BAD                                        # dw without Z


def test_norm_refusals():
    lib = N.load()
    fwd = lambda X=FAKE, ld=8, n=4, d=8, t=0, eps=1e-5, y=FAKE: lib.kmeans_norm_forward(
        X, ld, n, d, t, None, None, 1, eps, y, FAKE, FAKE, None)
    assert [fwd(X=None), fwd(ld=7), fwd(n=-1), fwd(d=0), fwd(t=3), fwd(eps=-1.0), fwd(eps=math.nan),
            fwd(eps=math.inf), fwd(y=None), fwd(ld=2 ** 62)] == [BAD] * 10
    need = lib.kmeans_norm_workspace_bytes(1000, 64, 1)
    assert need >= 2 * 64 * 4 and lib.kmeans_norm_workspace_bytes(-1, 64, 1) == 0
    assert lib.kmeans_norm_workspace_bytes(10, 0, 1) == 0 and lib.kmeans_norm_workspace_bytes(10, 4, 9) == 0
    bwd = lambda ws=FAKE, wsb=need, dy=FAKE, ld=64: lib.kmeans_norm_backward(
        dy, ld, FAKE, 64, 1000, 64, 1, FAKE, FAKE, None, 1, FAKE, FAKE, FAKE, ws, wsb, None)
    assert [bwd(ws=None), bwd(wsb=need - 1), bwd(ws=C.c_void_p(0x1010)), bwd(dy=None), bwd(ld=63)] == [BAD] * 5


def test_adapter_refusals():
    lib = N.load()
    size = lambda n=100, di=64, do=32, k=4, r=8, t=1, b=0: lib.kmeans_adapter_workspace_bytes(n, di, do, k, r, t, b)
    assert size() > 0 and size(b=1) > 0 and size(n=0) > 0
    assert [size(n=-1), size(n=2 ** 31), size(di=0), size(do=0), size(k=0), size(r=0), size(t=3), size(r=129)] == [0] * 8

    def fwd(X=FAKE, ldx=64, n=100, r=8, W=FAKE, ids=FAKE, order=None, sids=None, off=None, ws=FAKE, wsb=size()):
        return lib.kmeans_adapter_forward(X, ldx, n, 64, 32, 4, r, 1, W, FAKE, FAKE, None, ids, order, sids, off, FAKE,
                                          FAKE, ws, wsb, None)
    assert [fwd(X=None), fwd(ldx=63), fwd(n=-1), fwd(W=None), fwd(ids=None), fwd(ids=None, order=FAKE),
            fwd(ids=None, sids=FAKE), fwd(ws=None), fwd(wsb=size() - 1), fwd(ws=C.c_void_p(0x1010))] == [BAD] * 10
    assert fwd(r=129) == N.KM_ERR_UNSUPPORTED
    assert fwd(n=2 ** 27 + 1) == N.KM_ERR_UNSUPPORTED
    assert lib.kmeans_sort_workspace_bytes(1, 1, 1) > 0
    assert lib.kmeans_norm_workspace_bytes(1, 2 ** 28 + 1, 0) == 0

    def bwd(dY=FAKE, H=FAKE, n=100, sids=FAKE, off=FAKE, dA=FAKE, wsb=size(b=1)):
        return lib.kmeans_adapter_backward(dY, 32, FAKE, 64, H, n, 64, 32, 4, 8, 1, FAKE, FAKE, FAKE, None, None, sids,
                                           off, FAKE, dA, FAKE, FAKE, wsb, None)
    assert [bwd(dY=None), bwd(H=None), bwd(n=-1), bwd(sids=None), bwd(off=None), bwd(dA=None),
            bwd(wsb=size(b=1) - 1)] == [BAD] * 7


def test_binding_rejects_cpu_tensors():
    import torch
    import paper_1902_09527_amd as km
    with pytest.raises(ValueError):
        km.cluster_sort(torch.zeros(4, dtype=torch.int32), 2)
    with pytest.raises(ValueError):
        km.layernorm(torch.zeros(4, 8))
