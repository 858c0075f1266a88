"""The adapters' inner products between the two products, s h forward and g
backward: held in float32, so that y, dX and dA are rounded once.

Tolerances as in test_gpu_ops_adapter, but for the inner products: there is no
rounding of theirs to the rows' type.  The matrix cores take such a value v as
two of the rows' type, v rounded and its remainder rounded: off by at most
U^2 |v|, and for float16, whose exponents end at 2^-24, by 2^-38 of the largest
value that is held with the same power of two (float16 only; of a row's inner
products forward and for dX, of a cluster's for dA).
"""
import pytest
import torch

import paper_1902_09527_amd as km
from test_gpu_ops_adapter import DEV, F64, U, _case, _near, _sub, u

pytestmark = pytest.mark.gpu
LOW = [torch.bfloat16, torch.float16]


def _apart(dtype, v, most):
    """How far the two parts of v may be off; most: the largest magnitude that is held with it."""
    return U[dtype] ** 2 * v + (2.0 ** -38 * most if dtype == torch.float16 else 0.0)


def _check(c, y, h, grads):
    dtype, t = c["X"].dtype, U[c["X"].dtype]
    X, W, A, B, dY, s = (c[v].to(F64) for v in ("X", "W", "A", "B", "dY", "s"))
    (n, din), (dout, r), k = X.shape, B.shape[1:], A.shape[0]
    wy, yt = X @ W.T, 2 * (din + r) * u * (X.abs() @ W.abs().T)
    wx, xt = dY @ W, 2 * (dout + r) * u * (dY.abs() @ W.abs())
    wa, at, wb, bt = torch.zeros_like(A), torch.zeros_like(A), torch.zeros_like(B), torch.zeros_like(B)
    for q in range(k):
        i = torch.nonzero(c["ids"] == q)[:, 0]
        if not len(i):
            continue
        sh, mag = s[q] * X[i] @ A[q].T, s[q] * X[i].abs() @ A[q].abs().T
        off = 2 * (din + 1) * u * mag + _apart(dtype, mag, mag.amax(1, keepdim=True))
        wy[i] += sh @ B[q].T
        yt[i] += off @ B[q].abs().T + 2 * (din + r) * u * (sh.abs() @ B[q].abs().T)
        g, mag = s[q] * dY[i] @ B[q], s[q] * dY[i].abs() @ B[q].abs()
        sums = 2 * (dout + 1) * u * mag
        wx[i] += g @ A[q]
        xt[i] += (sums + _apart(dtype, mag, mag.amax(1, keepdim=True))) @ A[q].abs() \
            + 2 * (dout + r) * u * (g.abs() @ A[q].abs())
        wa[q] = g.T @ X[i]
        at[q] = (sums + _apart(dtype, mag, mag.max())).T @ X[i].abs() + 2 * len(i) * u * (g.abs().T @ X[i].abs())
        hr = h[i].to(F64)
        wb[q] = s[q] * dY[i].T @ hr
        bt[q] = 2 * len(i) * u * (s[q] * dY[i].abs().T @ hr.abs())
    for got, want, tol, what in zip((y,) + grads, (wy, wx, wa, wb), (yt, xt, at, bt), ("y", "dX", "dA", "dB")):
        assert torch.isfinite(got).all(), what
        _near(got, want, tol + t * want.abs() + _sub(dtype), what)


def _run(c):
    plan = km.cluster_sort(c["ids"], c["A"].shape[0])
    y, h = km.adapter_linear(c["X"], c["W"], c["A"], c["B"], plan, c["s"])
    grads = km.adapter_linear_backward(c["dY"], c["X"], h, c["W"], c["A"], c["B"], plan, c["s"])
    return y, h, grads


@pytest.mark.parametrize("dtype", LOW)
@pytest.mark.parametrize("n", [3, 40, 64, 65, 300, 1024, 1025, 3000])
@pytest.mark.parametrize("r", [1, 8, 16, 17, 24, 33, 64, 128])
def test_inner_products_are_not_rounded(r, n, dtype):
    """The adapters' term is the larger one here, and sums that cancel show a rounding of its parts."""
    c = _case(n + r, n, 96, 160, 5, r, dtype)
    c["W"] *= 0.125
    _check(c, *_run(c))


@pytest.mark.parametrize("dtype", LOW)
def test_long_clusters(dtype):
    c = _case(8, 9000, 128, 96, 3, 16, dtype)
    c["W"] *= 0.125
    _check(c, *_run(c))


# Magnitudes beside those of _case (whose values are about 1 but for A, B and W, of rows of length 1):
# s h up to some 3e5 with a finite y; g up to some 5e5 with finite gradients; s h, and g, among
# float16's subnormals (3e-7) while the results are not.
SCALES = {"large s h": dict(A=2.0 ** 13, s=8.0, B=2.0 ** -8, dY=2.0 ** -8),
          "large g": dict(dY=2.0 ** 9, B=2.0 ** 6, s=4.0, A=2.0 ** -10, X=2.0 ** -11),
          "small s h": dict(X=2.0 ** -12, A=2.0 ** -10, B=2.0 ** 10, W=0.0),
          "small g": dict(dY=2.0 ** -12, B=2.0 ** -12, A=2.0 ** 9, X=8.0, W=0.0)}


@pytest.mark.parametrize("n", [40, 300, 1100])
@pytest.mark.parametrize("name", list(SCALES))
def test_inner_products_beyond_the_range_of_float16(name, n):
    c = _case(n, n, 64, 96, 4, 16, torch.float16)
    for v, by in SCALES[name].items():
        c[v] *= by
    _check(c, *_run(c))


@pytest.mark.parametrize("dtype", LOW)
@pytest.mark.parametrize("n", [40, 300, 2000])
def test_one_infinite_index_leaves_the_others(n, dtype):
    """An infinite entry of B_c, column 2: g is not finite there and nowhere else."""
    c = _case(n, n, 64, 96, 3, 16, dtype, empty=0.0)
    y, h, (dx, da, db) = _run(c)
    c["B"][1, 7, 2] = float("inf")
    y2, h2, (dx2, da2, db2) = _run(c)
    rest = [j for j in range(16) if j != 2]
    assert not torch.isfinite(da2[1, 2]).any() and torch.isfinite(da2[1, rest]).all()
    assert (da2[1, rest].to(F64) - da[1, rest].to(F64)).abs().max() <= 2 * U[dtype] * da[1, rest].abs().max()
    mine = c["ids"] == 1
    assert torch.equal(y2[~mine], y[~mine]) and torch.equal(dx2[~mine], dx[~mine])
    cols = [j for j in range(96) if j != 7]
    assert torch.equal(y2[mine][:, cols], y[mine][:, cols]) and not torch.isfinite(y2[mine][:, 7]).any()
    assert not torch.isfinite(dx2[mine]).any()
    assert torch.equal(da2[[0, 2]], da[[0, 2]]) and torch.equal(db2, db)
