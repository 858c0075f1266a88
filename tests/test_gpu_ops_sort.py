"""Rows sorted by cluster and back (cluster_sort, cluster_gather,
cluster_combine and its gradients) against numpy's stable sort and float64
sums.

Tolerances: a stored result is rounded once (unit roundoff U of its type); a
float32 sum of t terms that are added in any order is off by at most about t
U32 times the sum of their magnitudes.
"""
import numpy as np
import pytest
import torch

import paper_1902_09527_amd as km

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
U32 = 2.0 ** -24


def _ids(rng, n, m, k, empty):
    ids = rng.integers(0, k, (n, m)).astype(np.int64)
    bad = rng.choice([-1, -7, k, k + 5, -2 ** 31, 2 ** 31 - 1], (n, m))
    return np.where(rng.random((n, m)) < empty, bad, ids).astype(np.int32)


def _expect(ids, k):
    flat = ids.reshape(-1).astype(np.int64)
    key = np.where((flat < 0) | (flat >= k), k, flat)
    order = np.argsort(key, kind="stable")
    pos = np.empty_like(order)
    pos[order] = np.arange(len(order))
    srt = key[order]
    return order, pos.reshape(ids.shape), np.where(srt < k, srt, -1), np.searchsorted(srt, np.arange(k + 1))


def _check_plan(ids, k, plan=None):
    plan = plan or km.cluster_sort(torch.from_numpy(ids).to(DEV), k)
    order, pos, sid, off = _expect(ids, k)
    np.testing.assert_array_equal(plan.order.cpu().numpy(), order)
    np.testing.assert_array_equal(plan.pos.cpu().numpy(), pos)
    np.testing.assert_array_equal(plan.sorted_ids.cpu().numpy(), sid)
    np.testing.assert_array_equal(plan.offsets.cpu().numpy(), off)
    return plan


@pytest.mark.parametrize("k", [1, 2, 8, 64, 1000, 1023, 1024, 5000, 100_000, 3_000_000])
@pytest.mark.parametrize("n,m", [(1, 1), (2, 1), (63, 1), (64, 1), (65, 3), (512, 2), (1024, 1), (1025, 1),
                                 (2048, 1), (2049, 1), (4099, 2), (70_001, 1)])
def test_plan(n, m, k):
    rng = np.random.default_rng(n * 31 + m * 7 + k)
    for empty in (0.0, 0.3):
        _check_plan(_ids(rng, n, m, k, empty), k)


@pytest.mark.parametrize("k", [2047, 4094, 4095, 4096, 4097])
@pytest.mark.parametrize("n", [1025, 30_011, 300_007, 1_200_000])
def test_plan_at_the_edge_of_one_pass(n, k):
    rng = np.random.default_rng(n + k)
    _check_plan(_ids(rng, n, 1, k, 0.05), k)


@pytest.mark.parametrize("k", [1, 63, 64, 8191, 8192, 8193])
@pytest.mark.parametrize("n", [64, 128, 129, 960, 1024, 6081, 6144, 6145])
def test_plan_at_the_edges_of_ranking(n, k):
    rng = np.random.default_rng(n * 3 + k)
    _check_plan(_ids(rng, n, 1, k, 0.1), k)
    _check_plan(np.sort(_ids(rng, n, 1, k, 0.0), axis=0)[::-1].copy(), k)
    _check_plan(np.full((n,), k - 1, np.int32), k)


@pytest.mark.parametrize("n", [1, 100, 5000])
def test_plan_with_every_slot_empty_or_one_cluster(n):
    _check_plan(np.full((n, 2), -1, np.int32), 9)
    _check_plan(np.full((n,), 4, np.int32), 9)
    _check_plan(np.full((n,), 8, np.int32), 9)


def test_plan_of_many_rows():
    rng = np.random.default_rng(5)
    _check_plan(_ids(rng, 3_000_001, 1, 100, 0.01), 100)     # tiles of more than four rounds
    _check_plan(np.sort(_ids(rng, 1_500_000, 1, 1000, 0.0), axis=0), 1000)


def test_no_rows():
    plan = km.cluster_sort(torch.empty(0, 2, dtype=torch.int32, device=DEV), 7)
    assert plan.offsets.cpu().tolist() == [0] * 8 and plan.order.numel() == 0
    x = torch.empty(0, 16, device=DEV)
    w = torch.empty(0, 2, device=DEV)
    assert km.cluster_gather(x, plan).shape == (0, 16)
    assert km.cluster_combine(x, plan, w).shape == (0, 16)
    dz, dw = km.cluster_combine_backward(x, x, plan, w)
    assert dz.shape == (0, 16) and dw.shape == (0, 2)


def _rows(rng, n, d, dtype, pad=0):
    """n rows of width d; pad: columns between them (a view of a wider table)."""
    full = torch.from_numpy(rng.standard_normal((n, d + pad)).astype(np.float32)).to(dtype).to(DEV)
    return full[:, :d] if pad else full


def _np(t):
    return t.detach().double().cpu().numpy()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", [1, 3, 8, 32, 100, 250, 256, 1001, 2048])
@pytest.mark.parametrize("n,m,k,empty,pad", [(1, 1, 3, 0.0, 0), (77, 2, 5, 0.2, 8), (600, 3, 1000, 0.5, 3),
                                             (1300, 1, 40, 1.0, 0)])
def test_rows_and_gradients(n, m, k, empty, pad, d, dtype):
    rng = np.random.default_rng(n + d)
    ids = _ids(rng, n, m, k, empty)
    plan = _check_plan(ids, k)
    order, pos, sid, off = _expect(ids, k)
    used, live = pos < off[k], sid >= 0

    X = _rows(rng, n, d, dtype, pad)
    Xs = km.cluster_gather(X, plan)
    want = np.where(live[:, None], _np(X)[order // m], 0.0)
    assert Xs.dtype == dtype and Xs.is_contiguous()
    np.testing.assert_array_equal(_np(Xs), want)

    # Rows and weights of empty slots hold NaN and infinity, which must not be read.
    Z = _rows(rng, n * m, d, dtype, pad)
    w = torch.from_numpy(rng.random((n, m)).astype(np.float32)).to(DEV)
    Z[torch.from_numpy(~live).to(DEV)] = float("nan")
    w[torch.from_numpy(~used).to(DEV)] = float("inf")
    z64 = np.where(live[:, None], _np(Z), 0.0)[pos]          # n, m, d
    w64 = np.where(used, _np(w), 0.0)
    for weights, wv in ((w, w64), (None, used.astype(float))):
        Y = km.cluster_combine(Z, plan, weights)
        terms = wv[:, :, None] * z64
        tol = U[dtype] * np.abs(terms.sum(1)) + (m + 1) * U32 * np.abs(terms).sum(1)
        tol += 2.0 ** -25 if dtype == torch.float16 else 0.0   # subnormal spacing
        assert (np.abs(_np(Y) - terms.sum(1)) <= tol).all()

    dY = _rows(rng, n, d, dtype, pad)
    dZ, dw = km.cluster_combine_backward(dY, Z, plan, w)
    want = np.where(live[:, None], w64.reshape(-1)[order][:, None] * _np(dY)[order // m], 0.0)
    tol = (U[dtype] + U32) * np.abs(want) + (2.0 ** -25 if dtype == torch.float16 else 0.0)
    assert (np.abs(_np(dZ) - want) <= tol).all()
    prod = z64 * _np(dY)[:, None, :] * used[:, :, None]
    tol = (d + 2) * U32 * np.abs(prod).sum(2)
    assert dw.dtype == torch.float32
    assert (np.abs(_np(dw) - prod.sum(2)) <= tol).all()
    assert (_np(dw)[~used] == 0).all()


def test_gradients_against_differences():
    """<G, Y> and its differences along a direction, float32 rows: the passes
    are linear in Z, w and X, so a central difference is exact but for
    rounding (about 1e-6 of the sum of magnitudes over a step of one)."""
    rng = np.random.default_rng(3)
    n, m, k, d = 50, 2, 6, 24
    plan = km.cluster_sort(torch.from_numpy(_ids(rng, n, m, k, 0.2)).to(DEV), k)
    Z, G, dirZ = (_rows(rng, r, d, torch.float32) for r in (n * m, n, n * m))
    w, dirw = (torch.from_numpy(rng.standard_normal((n, m)).astype(np.float32)).to(DEV) for _ in range(2))
    dZ, dw = km.cluster_combine_backward(G, Z, plan, w)
    f = lambda z, v: float((_np(km.cluster_combine(z, plan, v)) * _np(G)).sum())
    scale = n * m * d
    assert abs((f(Z + dirZ, w) - f(Z - dirZ, w)) / 2 - float((_np(dZ) * _np(dirZ)).sum())) < 1e-6 * scale
    assert abs((f(Z, w + dirw) - f(Z, w - dirw)) / 2 - float((_np(dw) * _np(dirw)).sum())) < 1e-6 * scale
    X, dirX, Gs = (_rows(rng, r, d, torch.float32) for r in (n, n, n * m))
    g = lambda x: float((_np(km.cluster_gather(x, plan)) * _np(Gs)).sum())
    dX = km.cluster_combine(Gs, plan)
    assert abs((g(X + dirX) - g(X - dirX)) / 2 - float((_np(dX) * _np(dirX)).sum())) < 1e-6 * scale


def test_rows_past_2_to_31_elements():
    """Row offsets beyond 32 bits: 17 million rows of 128 (4.3 GB in 16 bits)."""
    n, d, k = 17_000_003, 128, 3
    ids = (torch.arange(n, device=DEV, dtype=torch.int32) % 3)
    plan = km.cluster_sort(ids, k)
    X = torch.zeros(n, d, dtype=torch.bfloat16, device=DEV)
    X[:, 0] = (torch.arange(n, device=DEV) % 251).to(torch.bfloat16)
    X[:, 127] = (torch.arange(n, device=DEV) % 241).to(torch.bfloat16)
    Xs = km.cluster_gather(X, plan)
    order = plan.order.long()
    assert torch.equal(Xs[:, 0], X[:, 0][order]) and torch.equal(Xs[:, 127], X[:, 127][order])
    Y = km.cluster_combine(Xs, plan)
    assert torch.equal(Y[:, 0], X[:, 0]) and torch.equal(Y[:, 127], X[:, 127])


def test_side_stream_and_graph():
    rng = np.random.default_rng(11)
    n, m, k, d = 3000, 2, 50, 96
    ids = torch.from_numpy(_ids(rng, n, m, k, 0.1)).to(DEV)
    X = _rows(rng, n, d, torch.bfloat16)
    w = torch.rand(n, m, device=DEV)
    plan = km.cluster_sort(ids, k)
    want = km.cluster_combine(km.cluster_gather(X, plan), plan, w)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    p2 = km.cluster_sort(ids, k, stream=side)
    got = km.cluster_combine(km.cluster_gather(X, p2, stream=side), p2, w, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want) and torch.equal(p2.order, plan.order)

    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        p3 = km.cluster_sort(ids, k)
        out = km.cluster_combine(km.cluster_gather(X, p3), p3, w)
    for trial in range(4):   # replays with new ids, and eager work between them
        ids.copy_(torch.from_numpy(_ids(rng, n, m, k, 0.1)).to(DEV))
        X.mul_(0.5)
        g.replay()
        torch.cuda.synchronize()
        pe = km.cluster_sort(ids, k)
        want = km.cluster_combine(km.cluster_gather(X, pe), pe, w)
        assert torch.equal(out, want) and torch.equal(p3.pos, pe.pos), trial


def test_refusals():
    ids = torch.zeros(10, 2, dtype=torch.int32, device=DEV)
    plan = km.cluster_sort(ids, 4)
    X = torch.zeros(10, 8, device=DEV)
    Z = torch.zeros(20, 8, device=DEV)
    w = torch.zeros(10, 2, device=DEV)
    for bad in (ids.long(), ids.t(), ids.cpu(), torch.zeros(2, 2, 2, dtype=torch.int32, device=DEV)):
        with pytest.raises(ValueError):
            km.cluster_sort(bad, 4)
    for k in (0, -1, 2 ** 31 - 1):
        with pytest.raises(RuntimeError):
            km.cluster_sort(ids, k)
    for bad in (X[:9], X.double(), X.t(), X.cpu(), X[0], X.expand(10, 8)[:, :0], X[:1].expand(10, 8)):
        with pytest.raises(ValueError):
            km.cluster_gather(bad, plan)
    with pytest.raises(TypeError):
        km.cluster_gather(X, ids)
    with pytest.raises(ValueError):
        km.cluster_combine(X, plan, w)            # n rows in place of n m
    for bad in (w[:9], w.double(), w.t(), w.cpu()):
        with pytest.raises(ValueError):
            km.cluster_combine(Z, plan, bad)
    with pytest.raises(ValueError):
        km.cluster_combine_backward(X, Z.half(), plan, w)
    with pytest.raises(ValueError):
        km.cluster_combine_backward(X, Z[:, :4], plan, w)
