"""Places beyond 4 GB: weights, strides, tables, 8-bit values and tensors whose
offsets in bytes or elements do not fit 32 bits."""
import pytest
import torch

import paper_1902_09527_amd as km

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -8   # half a step of bfloat16


def _near(got, want, most, terms):
    """One rounding of the result, and a float32 sum of `terms` products."""
    tol = U * want.abs() + terms * 2.0 ** -24 * most
    assert bool(((got.double() - want).abs() <= tol).all())


def test_weights_and_strides():
    n, d, k, ld = 300, 4096, 150, 2 ** 23 + 8   # 5 GB of weights; rows 16 MB apart, 5 GB
    W = torch.empty(k, d, d, device=DEV, dtype=torch.bfloat16).normal_(std=d ** -0.5)
    flat = torch.empty(n * ld, device=DEV, dtype=torch.bfloat16)
    X, dY = flat.as_strided((n, d), (ld, 1)), flat.as_strided((n, d), (ld, 1), 2 * d)
    X.normal_()
    dY.normal_()
    ids = torch.arange(n, device=DEV, dtype=torch.int32) % k
    for rows in (n, 40):   # 40: the form for few rows, of the last clusters
        x, dy, i = X[n - rows:], dY[n - rows:], ids[n - rows:].contiguous()
        plan = km.cluster_sort(i, k)
        y = km.cluster_linear(x, W, plan)
        dx, dw = km.cluster_linear_backward(dy, x, W, plan)
        for c in (0, 1, k // 2, k - 2, k - 1):
            at = (i == c).nonzero()[:, 0]
            a, b, w = x[at].double(), dy[at].double(), W[c].double()
            _near(y[at], a @ w.t(), a.abs() @ w.abs().t(), d)
            _near(dx[at], b @ w, b.abs() @ w.abs(), d)
            _near(dw[c], b.t() @ a, b.abs().t() @ a.abs(), rows)
        del y, dx, dw
    q, Wq = km.quantize_blocks(X), km.quantize_blocks(W)
    plan = km.cluster_sort(ids, k)
    y = km.cluster_linear_fp8(q, Wq, plan, dtype=torch.float32)
    for c in (0, k - 1):
        at = (ids == c).nonzero()[:, 0]
        a = km.dequantize_blocks(q).double()[at]
        w = km.dequantize_blocks(km.BlockRows(Wq.values[c], Wq.exponents[c])).double()
        assert bool(((y[at].double() - a @ w.t()).abs() <= (d + 2) * 2.0 ** -24 * (a.abs() @ w.abs().t())).all())


def test_table():
    k, d, n = 700_001, 4096, 4000   # 5.7 GB
    table = torch.empty(k, d, device=DEV, dtype=torch.bfloat16).normal_()
    ids = torch.randint(0, k, (n,), device=DEV, dtype=torch.int32)
    ids[:3], ids[3:5] = k - 1, 0
    got = km.cluster_embedding(ids, table, 2.0)
    assert torch.equal(got, table[ids.long()] * 2)
    dT = km.cluster_embedding_backward(got, km.cluster_sort(ids, k))
    for c in (0, k - 1):
        at = (ids == c).nonzero()[:, 0]
        want = got[at].double()
        _near(dT[c], want.sum(0), want.abs().sum(0), n)
    used = ids.unique().long()
    assert float(dT.float().abs().sum(1).nonzero().numel()) == len(used)


def test_8_bit_rows():
    n, d = 1_100_000, 4096   # 9 GB, 4.5 GB in 8 bits
    X = torch.empty(n, d, device=DEV, dtype=torch.bfloat16).normal_()
    q = km.quantize_blocks(X)
    for at in (0, n // 2, n - 7):
        part = km.quantize_blocks(X[at:at + 7])
        assert torch.equal(q.values[at:at + 7].view(torch.uint8), part.values.view(torch.uint8))
        assert torch.equal(q.exponents[at:at + 7], part.exponents)
    back = km.dequantize_blocks(q, torch.bfloat16)
    assert torch.equal(back[-7:], km.dequantize_blocks(part, torch.bfloat16))


def test_clipping():
    n = 2 ** 31 + 1001   # elements
    t = torch.ones(n, device=DEV, dtype=torch.bfloat16)
    t[-1] = 0
    limit = (n - 1) ** 0.5 / 4
    norm = km.clip_global_norm([t], limit)
    assert abs(float(norm) - (n - 1) ** 0.5) <= 2.0 ** -22 * float(norm)
    assert float(t[-1]) == 0 and bool((t[:-1] == 0.25).all())
