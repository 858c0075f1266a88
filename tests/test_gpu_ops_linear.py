"""Products with one weight per cluster (cluster_linear and its gradients)
against float64, cluster by cluster.

Tolerances.  A float32 sum of t products, in any order, is off by at most
2 t u times the sum of the magnitudes (u = 2^-24; the factor 2 covers sums
inside a matrix instruction that are not rounded to nearest).  A result is
rounded once to the rows' type (U).
"""
import pytest
import torch

import paper_1902_09527_amd as km

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
u = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16, torch.float16]
F64 = torch.float64


def _sub(dtype):   # half the spacing of float16's subnormals
    return 2.0 ** -25 if dtype == torch.float16 else 0.0


def _case(seed, n, din, dout, k, dtype, empty=0.1, pad=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    t = lambda *s, c=1.0: (torch.randn(*s, generator=g, device=DEV) * c).to(dtype)
    c = {"X": t(n, din + pad)[:, :din], "dY": t(n, dout + pad)[:, :dout], "W": t(k, dout, din, c=din ** -0.5)}
    ids = torch.randint(0, k, (n,), generator=g, device=DEV)
    bad = torch.where(torch.rand(n, generator=g, device=DEV) < 0.5, -3, k)
    c["ids"] = torch.where(torch.rand(n, generator=g, device=DEV) < empty, bad, ids).to(torch.int32)
    return c


def _near(got, want, tol, what):
    off = (got.to(F64) - want).abs() - tol
    assert (off <= 0).all(), "%s: off by %.3g over its tolerance" % (what, float(off.max()))


def _check(c, y, dx, dw):
    dtype, t = c["X"].dtype, U[c["X"].dtype]
    X, W, dY = (c[v].to(F64) for v in ("X", "W", "dY"))
    (n, din), (k, dout, _) = X.shape, W.shape
    z = lambda *s: torch.zeros(*s, dtype=F64, device=DEV)
    wy, ty, wx, tx, ww, tw = z(n, dout), z(n, dout), z(n, din), z(n, din), z(*W.shape), z(*W.shape)
    for q in range(k):
        i = torch.nonzero(c["ids"] == q)[:, 0]
        if not len(i):
            continue
        wy[i], ty[i] = X[i] @ W[q].T, 2 * din * u * (X[i].abs() @ W[q].abs().T)
        wx[i], tx[i] = dY[i] @ W[q], 2 * dout * u * (dY[i].abs() @ W[q].abs())
        ww[q], tw[q] = dY[i].T @ X[i], 2 * len(i) * u * (dY[i].abs().T @ X[i].abs())
    for got, want, tol, what in ((y, wy, ty, "Y"), (dx, wx, tx, "dX"), (dw, ww, tw, "dW")):
        assert got.dtype == dtype and got.shape == want.shape
        _near(got, want, tol + t * want.abs() + _sub(dtype), what)


def _run(c):
    """Rows in their own order, and sorted: the same results."""
    plan = km.cluster_sort(c["ids"], c["W"].shape[0])
    y = km.cluster_linear(c["X"], c["W"], plan)
    dx, dw = km.cluster_linear_backward(c["dY"], c["X"], c["W"], plan)
    _check(c, y, dx, dw)
    at = plan.order.long()
    ys = km.cluster_linear(c["X"][at], c["W"], plan, sorted_rows=True)
    dxs, dws = km.cluster_linear_backward(c["dY"][at], c["X"][at], c["W"], plan, sorted_rows=True)
    if c["X"].is_contiguous():   # strided rows may take another form
        assert torch.equal(ys, y[at]) and torch.equal(dxs, dx[at]) and torch.equal(dws, dw)
    return y, dx, dw


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 2, 15, 17, 48, 64, 65, 200, 1000])
@pytest.mark.parametrize("din,dout,k", [(16, 16, 3), (64, 64, 1), (128, 320, 40), (250, 130, 7), (33, 47, 300),
                                        (512, 1024, 20), (8, 1001, 9)])
def test_rows(n, din, dout, k, dtype):
    print("case", n, din, dout, k, dtype, flush=True)
    _run(_case(n * 7 + k, n, din, dout, k, dtype))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("din", [1, 2, 7, 8, 31, 32, 63, 64, 65, 72, 127, 128, 129, 136, 200, 256, 264])
def test_widths(din, dtype):
    for n, dout in ((5, din + 3), (150, 64), (130, 72)):
        _run(_case(din, n, din, dout, 4, dtype))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,din,dout,k", [(4200, 128, 4096, 5), (4097, 320, 1024, 8), (4500, 1000, 1100, 30),
                                          (2050, 136, 2304, 9), (3000, 257, 515, 3), (70000, 64, 64, 2),
                                          (66000, 40, 24, 1)])
def test_larger_tiles(n, din, dout, k, dtype):
    """Sizes at which the wider tiles are taken, forward and backward, and chunks are joined."""
    print("case", n, din, dout, k, dtype, flush=True)
    _run(_case(n, n, din, dout, k, dtype))


@pytest.mark.parametrize("dtype", TYPES)
def test_sizes_of_clusters(dtype):
    """Clusters that end inside a tile, at its end and a row behind it; of no row; and one of all rows."""
    sizes = [3000, 256, 257, 0, 1, 255, 64, 65, 0, 63, 512, 513]
    ids = torch.repeat_interleave(torch.arange(len(sizes), device=DEV), torch.tensor(sizes, device=DEV))
    n = len(ids)
    for din, dout in ((96, 72), (512, 2560)):
        c = _case(5, n, din, dout, len(sizes), dtype)
        c["ids"] = ids[torch.randperm(n, device=DEV)].to(torch.int32).contiguous()
        _run(c)
        c["ids"] = torch.full_like(c["ids"], 7)
        _run(c)


@pytest.mark.parametrize("dtype", TYPES)
def test_strided_rows(dtype):
    for pad in (8, 3):
        for n in (20, 333, 3000):
            _run(_case(pad, n, 64, 128, 5, dtype, pad=pad))


@pytest.mark.parametrize("dtype", TYPES)
def test_unaligned_weights(dtype):
    for n in (30, 400):
        c = _case(2, n, 64, 96, 5, dtype)
        flat = torch.empty(c["W"].numel() + 1, dtype=dtype, device=DEV)
        flat[1:] = c["W"].reshape(-1)
        c["W"] = flat[1:].view(c["W"].shape)
        _run(c)


@pytest.mark.parametrize("n", [3, 300])
def test_rows_in_no_cluster(n):
    y, dx, dw = _run(_case(1, n, 64, 64, 4, torch.bfloat16, empty=1.0))
    assert (y == 0).all() and (dx == 0).all() and (dw == 0).all()


def test_sorted_rows_of_several_slots():
    c = _case(3, 500, 96, 80, 9, torch.bfloat16)
    ids = torch.stack([c["ids"], (c["ids"] + 1).clamp_max(8)], 1).contiguous()
    plan = km.cluster_sort(ids, 9)
    d = dict(c, X=km.cluster_gather(c["X"], plan), dY=km.cluster_gather(c["dY"], plan), ids=plan.sorted_ids)
    y = km.cluster_linear(d["X"], d["W"], plan, sorted_rows=True)
    _check(d, y, *km.cluster_linear_backward(d["dY"], d["X"], d["W"], plan, sorted_rows=True))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [30, 400, 3000])
def test_nonfinite_values_stay_in_their_cluster(n, dtype):
    c = _case(9, n, 64, 96 if n < 3000 else 2048, 5, dtype)
    c["ids"][:4] = torch.tensor([0, 1, 2, -1], dtype=torch.int32)
    y, dx, dw = _run(c)
    c["W"][1, 3, 5], c["W"][1, 7, 2], c["W"][2, 0, 0] = float("inf"), float("nan"), float("-inf")
    i = int(torch.nonzero(c["ids"] == 0)[0])
    c["X"][i, 0], c["dY"][i, 0] = float("nan"), float("inf")
    c["X"][c["ids"] == -3], c["dY"][c["ids"] == -3] = float("nan"), float("inf")
    plan = km.cluster_sort(c["ids"], 5)
    y2 = km.cluster_linear(c["X"], c["W"], plan)
    dx2, dw2 = km.cluster_linear_backward(c["dY"], c["X"], c["W"], plan)
    ok = (c["ids"] != 1) & (c["ids"] != 2)
    ok[i] = False
    assert torch.equal(y2[ok], y[ok]) and torch.equal(dx2[ok], dx[ok]) and torch.equal(dw2[1:], dw[1:])
    assert not torch.isfinite(y2[c["ids"] == 1]).all() and not torch.isfinite(dw2[0]).all()


def test_no_rows():
    c = _case(2, 0, 64, 32, 4, torch.bfloat16)
    plan = km.cluster_sort(c["ids"], 4)
    assert km.cluster_linear(c["X"], c["W"], plan).shape == (0, 32)
    dx, dw = km.cluster_linear_backward(c["dY"], c["X"], c["W"], plan)
    assert dx.shape == (0, 64) and (dw == 0).all()


def test_one_gradient_of_two():
    c = _case(4, 200, 96, 64, 6, torch.float16)
    plan = km.cluster_sort(c["ids"], 6)
    dx, dw = km.cluster_linear_backward(c["dY"], c["X"], c["W"], plan)
    a = km.cluster_linear_backward(c["dY"], c["X"], c["W"], plan, need_dW=False)
    b = km.cluster_linear_backward(c["dY"], c["X"], c["W"], plan, need_dX=False)
    assert torch.equal(a[0], dx) and a[1] is None and b[0] is None and torch.equal(b[1], dw)


def test_gradient_against_differences():
    """<G, Y> is linear in X and in W, so central differences are exact but for
    float32 rounding, about K u of the sums' magnitudes."""
    c = _case(11, 120, 48, 40, 5, torch.float32)
    y, *grads = _run(c)
    plan = km.cluster_sort(c["ids"], 5)
    f = lambda **k: float((km.cluster_linear(*(dict(c, **k)[v] for v in ("X", "W")), plan).to(F64)
                           * c["dY"].to(F64)).sum())
    scale = float((y.abs().to(F64) * c["dY"].abs().to(F64)).sum())
    for name, grad in zip(("X", "W"), grads):
        d = torch.randn_like(c[name])
        diff = (f(**{name: c[name] + d}) - f(**{name: c[name] - d})) / 2
        assert abs(diff - float((grad.to(F64) * d.to(F64)).sum())) < 1e-5 * scale, name


@pytest.mark.parametrize("n,din", [(24, 256), (700, 256), (5000, 1024)])
def test_side_stream_graph_and_repeats(n, din):
    c = _case(n, n, din, 1536, 12, torch.bfloat16)

    def step(stream=None):
        plan = km.cluster_sort(c["ids"], 12, stream=stream)
        y = km.cluster_linear(c["X"], c["W"], plan, stream=stream)
        return (y,) + km.cluster_linear_backward(c["dY"], c["X"], c["W"], plan, stream=stream)
    want = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for trial in range(3):
        c["X"].mul_(-0.75)
        c["ids"].copy_((c["ids"] + 1).clamp_max(11))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, step())), trial


def test_refusals():
    c = _case(1, 10, 32, 16, 4, torch.bfloat16, empty=0.0)
    X, W, ids = c["X"], c["W"], c["ids"]
    plan = km.cluster_sort(ids, 4)
    ok = dict(X=X, W=W, plan=plan)
    for bad in (dict(X=X[:9]), dict(X=X.float()), dict(X=X.t()), dict(X=X[:, :31]), dict(W=W.transpose(1, 2)),
                dict(W=W.float()), dict(W=W.cpu()), dict(W=W[:3]), dict(W=W[0]), dict(W=W[:, :0]),
                dict(plan=km.cluster_sort(ids, 5)), dict(plan=km.cluster_sort(ids[:9].contiguous(), 4)),
                dict(plan=km.cluster_sort(ids.view(5, 2), 4))):
        with pytest.raises(ValueError):
            km.cluster_linear(**dict(ok, **bad))
    with pytest.raises(TypeError):
        km.cluster_linear(X, W, ids)
    with pytest.raises(ValueError, match="requires a gradient"):
        km.cluster_linear(X, W.clone().requires_grad_(), plan)
    good = dict(dY=c["dY"], X=X, W=W, plan=plan)
    for bad in (dict(dY=c["dY"][:, :15]), dict(dY=c["dY"].float()), dict(dY=c["dY"][:9]),
                dict(plan=km.cluster_sort(ids, 5))):
        with pytest.raises(ValueError):
            km.cluster_linear_backward(**dict(good, **bad))
