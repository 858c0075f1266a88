"""Every form of the shared product: tiles of 256, 128 and 64, the contraction
whole and in parts, results of aligned, ragged and odd widths, forward and
backward, over many clusters and several steps of r.  The form is asked for
(kmeans_adapter_tile), so that a size that goes to another one fails here.

Contractions are longer than the stages that are in flight (9 stages at 520 in
16 bits, 17 in float32).  Tolerances: those of test_gpu_ops_adapter, and without
a rounding of the inner products those of test_gpu_ops_adapter_precision.
"""
import ctypes as C

import pytest
import torch

import paper_1902_09527_amd as km
import test_gpu_ops_adapter as base
import test_gpu_ops_adapter_precision as precise
from paper_1902_09527_amd import _native as N

pytestmark = pytest.mark.gpu
DEV = base.DEV
LOW, F32 = [torch.bfloat16, torch.float16], [torch.float32]
CODE = {torch.float32: N.KM_F32, torch.bfloat16: N.KM_BF16, torch.float16: N.KM_F16}
K = 60

# rows, contraction, width of the results, the form
SIZES = [(LOW, 520, 776, 333, 64, 1), (LOW, 1030, 520, 264, 64, 1), (LOW, 203, 520, 1536, 64, 1),
         (LOW, 520, 1032, 333, 64, 4), (LOW, 2051, 1032, 72, 64, 4), (LOW, 203, 776, 333, 64, 7),
         (LOW, 203, 4104, 333, 64, 8), (LOW, 333, 4104, 72, 64, 8),
         (LOW, 3001, 520, 1001, 128, 1), (LOW, 6001, 520, 504, 128, 1), (LOW, 2051, 520, 1536, 128, 1),
         (LOW, 333, 4104, 3001, 128, 2), (LOW, 2051, 4104, 504, 128, 2), (LOW, 777, 4104, 1536, 128, 2),
         (LOW, 1500, 4104, 333, 128, 4), (LOW, 203, 4104, 2312, 128, 4), (LOW, 333, 4104, 1536, 128, 4),
         (LOW, 333, 4104, 1001, 128, 8), (LOW, 3001, 4104, 72, 128, 8), (LOW, 203, 4104, 1536, 128, 8),
         (LOW, 2051, 520, 4099, 256, 1), (LOW, 3001, 520, 2312, 256, 1), (LOW, 6001, 776, 1536, 256, 1),
         (LOW, 1030, 4104, 4099, 256, 2), (LOW, 4200, 4104, 1000, 256, 2), (LOW, 3001, 4104, 1536, 256, 2),
         (F32, 333, 520, 3001, 64, 1), (F32, 1030, 520, 1000, 64, 1), (F32, 777, 520, 1536, 64, 1),
         (F32, 1500, 520, 504, 64, 2), (F32, 777, 520, 333, 64, 4), (F32, 333, 2056, 333, 64, 8),
         (F32, 520, 520, 4099, 128, 1), (F32, 2051, 520, 1032, 128, 1), (F32, 1500, 520, 1536, 128, 1),
         (F32, 333, 776, 4099, 128, 2), (F32, 520, 776, 2312, 128, 2), (F32, 2051, 520, 333, 128, 4),
         (F32, 777, 2056, 333, 128, 8), (F32, 6001, 520, 2301, 256, 1), (F32, 6001, 520, 2312, 256, 1)]
CASES = [s + (t, back) for s in SIZES for t in s[0] for back in (False, True)]


def _form(n, din, dout, r, dtype, back):
    tile, splits = C.c_int32(), C.c_int32()
    assert N.load().kmeans_adapter_tile(n, din, dout, K, r, CODE[dtype], int(back), C.byref(tile), C.byref(splits)) == 0
    return tile.value, splits.value


def _case(n, inner, width, r, dtype, back):
    """The sizes of one pass: its contraction is over `inner` and its results are `width` wide."""
    din, dout = (width, inner) if back else (inner, width)
    return (din, dout), base._case(n + inner + r, n, din, dout, K, r, dtype)


@pytest.mark.parametrize("i", range(len(CASES)))
def test_forms(i):
    _, n, inner, width, tile, splits, dtype, back = CASES[i]
    for r in (48, 16, 128)[i % 2:i % 2 + 2]:
        print("case", n, inner, width, r, dtype, back, flush=True)
        (din, dout), c = _case(n, inner, width, r, dtype, back)
        assert _form(n, din, dout, r, dtype, back) == (tile, splits)
        y, h, g = base._run(c)
        precise._check(c, y, h, g)


@pytest.mark.parametrize("n,inner,width", [(2051, 520, 1536), (2051, 4104, 504), (3001, 520, 2312), (4200, 4104, 1000)])
@pytest.mark.parametrize("dtype", LOW)
def test_nonfinite_adapters_and_rows_stay_in_their_cluster(n, inner, width, dtype):
    c = base._case(n, n, inner, width, 5, 40, dtype)
    c["ids"][:4] = torch.tensor([0, 1, 2, -1], dtype=torch.int32)
    plan = km.cluster_sort(c["ids"], 5)
    args = lambda: [c[v] for v in ("W", "A", "B")] + [plan, c["s"]]
    y, h = km.adapter_linear(c["X"], *args())
    dx, da, db = km.adapter_linear_backward(c["dY"], c["X"], h, *args())
    c["A"][1, 3, 5], c["B"][1, 7, 2], c["B"][2, 0, 0] = float("inf"), float("nan"), float("-inf")
    i = int(torch.nonzero(c["ids"] == 0)[0])
    c["X"][i, 0], c["dY"][i, 0] = float("nan"), float("inf")
    y2, h2 = km.adapter_linear(c["X"], *args())
    dx2, da2, db2 = km.adapter_linear_backward(c["dY"], c["X"], h2, *args())
    ok = (c["ids"] != 1) & (c["ids"] != 2)
    ok[i] = False
    assert torch.equal(y2[ok], y[ok]) and torch.equal(h2[ok], h[ok]) and torch.equal(dx2[ok], dx[ok])
    assert torch.equal(da2[3:], da[3:]) and torch.equal(db2[3:], db[3:])
    assert not torch.isfinite(y2[c["ids"] == 1]).all() and not torch.isfinite(da2[0]).all()


def test_forms_that_are_asked_for_are_checked():
    lib, a, b = N.load(), C.c_int32(), C.c_int32()
    ask = lambda n=100, r=8, t=1, p=C.byref(a): lib.kmeans_adapter_tile(n, 64, 32, 4, r, t, 0, p, C.byref(b))
    assert [ask(n=-1), ask(r=0), ask(t=3), ask(p=None)] == [N.KM_ERR_INVALID_ARG] * 4
    assert ask(r=129) == N.KM_ERR_UNSUPPORTED
    assert ask(n=64) == 0 and (a.value, b.value) == (0, 1)
