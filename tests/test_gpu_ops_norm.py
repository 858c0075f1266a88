"""Layer norm and its gradients against the formulas in float64.

Tolerances, first order in the roundoff u = 2^-24 of the float32 sums: a sum
over a row is off by at most K u times the sum of magnitudes, K = 64 + d / 128
additions in a row of any lane and its tree; a sum over rows likewise with
64 + n / 64.  Stored results are rounded once more (U of their type).
"""
import numpy as np
import pytest
import torch

import paper_1902_09527_amd as km

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
u = 2.0 ** -24


def _np(t):
    return t.detach().double().cpu().numpy()


def _case(rng, n, d, dtype, ptype, shift=0.0, pad=0):
    full = rng.standard_normal((n, d + pad)) * np.exp(0.5 * rng.standard_normal(d + pad)) + shift
    X = torch.from_numpy(full.astype(np.float32)).to(dtype).to(DEV)[:, :d]
    dY = torch.from_numpy(rng.standard_normal((n, d + pad)).astype(np.float32)).to(dtype).to(DEV)[:, :d]
    g = torch.from_numpy((1 + 0.3 * rng.standard_normal(d)).astype(np.float32)).to(ptype).to(DEV)
    b = torch.from_numpy((0.3 * rng.standard_normal(d)).astype(np.float32)).to(ptype).to(DEV)
    return (X if pad else X.contiguous()), (dY if pad else dY.contiguous()), g, b


def _check(X, dY, g, b, eps):
    n, d = X.shape
    t, K, Kn = U[X.dtype], 64 + d / 128, 64 + n / 64
    sub = 2.0 ** -25 if X.dtype == torch.float16 else 0.0
    y, mean, rstd = km.layernorm(X, g, b, eps)
    dx, dg, db = km.layernorm_backward(dY, X, mean, rstd, g)
    x, dy = _np(X), _np(dY)
    gv = np.ones(d) if g is None else _np(g)
    bv = np.zeros(d) if b is None else _np(b)
    mu = x.mean(1, keepdims=True)
    var = ((x - mu) ** 2).mean(1, keepdims=True)
    rs = 1 / np.sqrt(var + eps)
    xh = (x - mu) * rs
    mu_tol = K * u * np.abs(x).mean(1, keepdims=True)
    rel = 2 * K * u + 0.5 * (mu_tol * rs) ** 2          # of rs
    xh_tol = rs * mu_tol + np.abs(xh) * rel + 4 * u * np.abs(xh)
    assert (np.abs(_np(mean) - mu[:, 0]) <= mu_tol[:, 0]).all()
    assert (np.abs(_np(rstd) / rs[:, 0] - 1) <= rel[:, 0]).all()
    want = xh * gv + bv
    tol = t * np.abs(want) + np.abs(gv) * xh_tol + 4 * u * (np.abs(want) + np.abs(bv)) + sub
    assert y.dtype == X.dtype and (np.abs(_np(y) - want) <= tol).all()

    h = dy * gv
    s1, s2 = h.mean(1, keepdims=True), (h * xh).mean(1, keepdims=True)
    want = rs * (h - s1 - xh * s2)
    s1_tol = K * u * np.abs(h).mean(1, keepdims=True)
    s2_tol = K * u * np.abs(h * xh).mean(1, keepdims=True) + (np.abs(h) * xh_tol).mean(1, keepdims=True)
    tol = rs * (4 * u * (np.abs(h) + np.abs(s1) + np.abs(xh * s2)) + s1_tol + np.abs(xh) * s2_tol
                + np.abs(s2) * xh_tol) + np.abs(want) * (t + rel) + sub
    assert dx.dtype == X.dtype and (np.abs(_np(dx) - want) <= tol).all()
    tol = Kn * u * np.abs(dy * xh).sum(0) + (np.abs(dy) * xh_tol).sum(0)
    assert dg.dtype == torch.float32 and (np.abs(_np(dg) - (dy * xh).sum(0)) <= tol).all()
    assert (np.abs(_np(db) - dy.sum(0)) <= Kn * u * np.abs(dy).sum(0)).all()


WIDTHS = [1, 2, 7, 8, 31, 64, 65, 250, 256, 513, 1000, 1024, 1025, 2048, 4096, 4104, 8192, 8200, 16384, 20_001]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", WIDTHS)
def test_rows(d, dtype):
    rng = np.random.default_rng(d)
    for n in (1, 5, 130):
        X, dY, g, b = _case(rng, n, d, dtype, torch.float32, shift=0.5)
        _check(X, dY, g, b, 1e-5)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", [2049, 2050, 4097, 4098, 8188, 8194, 8196, 11_456, 16_392, 32_768])
def test_rows_of_many_lanes(d, dtype):
    rng = np.random.default_rng(d)
    for n in (1, 77):
        X, dY, g, b = _case(rng, n, d, dtype, dtype, shift=0.5)
        _check(X, dY, g, b, 1e-5)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d,pad", [(48, 16), (250, 3), (2048, 8), (9000, 24)])
def test_strided_rows_and_parameter_types(d, pad, dtype):
    rng = np.random.default_rng(d)
    X, dY, g, b = _case(rng, 37, d, dtype, dtype, pad=pad)
    _check(X, dY, g, b, 1e-6)
    _check(X, dY, g, None, 1e-6)
    _check(X, dY, None, None, 0.1)


@pytest.mark.parametrize("n,d", [(50_003, 16), (100_001, 250), (4097, 1024), (2000, 4096), (1500, 12_000)])
def test_many_rows(n, d):
    rng = np.random.default_rng(n)
    X, dY, g, b = _case(rng, n, d, torch.float32, torch.float32)
    _check(X, dY, g, b, 1e-5)


def test_rows_far_from_the_origin():
    """A mean 1000 times the spread: deviations are formed before they are squared."""
    rng = np.random.default_rng(2)
    for d in (100, 1024, 5000):
        X, dY, g, b = _case(rng, 33, d, torch.float32, torch.float32, shift=1000.0)
        _check(X, dY, g, b, 1e-5)


def test_constant_rows_and_single_columns():
    for d in (1, 64, 300):
        X = torch.full((4, d), 2.0, device=DEV)
        y, mean, rstd = km.layernorm(X, None, None, 1e-4)
        assert (mean == 2).all() and (y == 0).all()
        assert torch.allclose(rstd, torch.full_like(rstd, 100.0), rtol=1e-6)
        dx, dg, db = km.layernorm_backward(torch.ones_like(X), X, mean, rstd)
        assert (dg == 0).all() and (db == 4).all() and (dx == 0).all()


def test_nonfinite_rows_stay_in_their_rows():
    X = torch.randn(300, 128, device=DEV)
    want, _, _ = km.layernorm(X)
    X[7, 3], X[100, 5] = float("nan"), float("inf")
    y, _, _ = km.layernorm(X)
    ok = torch.ones(300, dtype=torch.bool, device=DEV)
    ok[7] = ok[100] = False
    assert torch.isnan(y[7]).all() and torch.isnan(y[100]).any()
    assert torch.equal(y[ok], want[ok])


def test_no_rows():
    X = torch.empty(0, 70, dtype=torch.bfloat16, device=DEV)
    y, mean, rstd = km.layernorm(X)
    dx, dg, db = km.layernorm_backward(X, X, mean, rstd)
    assert y.shape == dx.shape == (0, 70) and (dg == 0).all() and (db == 0).all() and dg.shape == (70,)


def test_gradient_against_differences():
    """Central differences of <G, Y> in float64 arithmetic of the float32
    kernel: a step of 1e-2 has a truncation error of order 1e-4 of the
    gradient's scale and a rounding error of about 1e-7 |G|.|Y| / 1e-2."""
    rng = np.random.default_rng(8)
    X, G, g, b = _case(rng, 6, 40, torch.float32, torch.float32)
    y, mean, rstd = km.layernorm(X, g, b)
    dx, dg, db = km.layernorm_backward(G, X, mean, rstd, g)
    f = lambda x, gg, bb: float((_np(km.layernorm(x, gg, bb)[0]) * _np(G)).sum())
    h = 1e-2
    scale = float(np.abs(_np(G)).sum())
    for t, grad in ((X, dx), (g, dg), (b, db)):
        d = torch.from_numpy(rng.standard_normal(tuple(t.shape)).astype(np.float32)).to(DEV)
        args = lambda s: [v + s * h * d if v is t else v for v in (X, g, b)]
        diff = (f(*args(1)) - f(*args(-1))) / (2 * h)
        assert abs(diff - float((_np(grad) * _np(d)).sum())) < 1e-3 * scale


def test_side_stream_graph_and_repeats():
    rng = np.random.default_rng(4)
    X, dY, g, b = _case(rng, 5000, 512, torch.bfloat16, torch.float32)
    y, mean, rstd = km.layernorm(X, g, b)
    want = (y,) + km.layernorm_backward(dY, X, mean, rstd, g)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y2, m2, r2 = km.layernorm(X, g, b, stream=side)
    got = (y2,) + km.layernorm_backward(dY, X, m2, r2, g, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y3, m3, r3 = km.layernorm(X, g, b)
        out = (y3,) + km.layernorm_backward(dY, X, m3, r3, g)
    for trial in range(3):
        X.mul_(1.25)
        graph.replay()
        torch.cuda.synchronize()
        ye, me, re = km.layernorm(X, g, b)
        want = (ye,) + km.layernorm_backward(dY, X, me, re, g)
        assert all(torch.equal(p, q) for p, q in zip(out, want)), trial


def test_refusals():
    X = torch.zeros(4, 16, device=DEV)
    g = torch.ones(16, device=DEV)
    for bad in (X.double(), X.cpu(), X[0], X.t()[:, ::2], X[:1].expand(4, 16)):
        with pytest.raises(ValueError):
            km.layernorm(bad)
    for bad in (g[:8], g.double(), g.half(), g.cpu(), g[None]):
        with pytest.raises(ValueError):
            km.layernorm(X, bad)
    with pytest.raises(ValueError):
        km.layernorm(X.half(), g, g.half())
    for eps in (-1.0, float("nan"), float("inf")):
        with pytest.raises(RuntimeError):
            km.layernorm(X, g, g, eps)
    y, mean, rstd = km.layernorm(X, g, g)
    for bad in (mean[:3], mean.double(), mean[:, None]):
        with pytest.raises(ValueError):
            km.layernorm_backward(X, X, bad, rstd, g)
    with pytest.raises(ValueError):
        km.layernorm_backward(X[:3], X, mean, rstd, g)
    with pytest.raises(ValueError):
        km.layernorm_backward(X.half(), X, mean, rstd, g)
