"""Products with one weight per cluster where tiles are more than the blocks of 256
threads that one dimension of a launch holds (2^24): a cluster a row, of one column.

Every result is one product, or a row of no cluster or a weight of no row: exact but for
its one rounding."""
import pytest
import torch

import paper_1902_09527_amd as km

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _clusters(n, k):
    """Each of the first n clusters of one row, but for some rows in none."""
    g = torch.Generator(device=DEV)
    g.manual_seed(n)
    ids = torch.randperm(n, generator=g, device=DEV).to(torch.int32)
    ids[::1001] = -1
    return g, ids, km.cluster_sort(ids, k)


def test_one_column():
    n = k = 2 ** 24 + 2 ** 20 + 77
    g, ids, plan = _clusters(n, k)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV).half()
    X, dY, W = rand(n, 1), rand(n, 1), rand(k, 1, 1)
    none, at = (ids < 0)[:, None], ids.clamp_min(0).long()
    product = lambda a, b: torch.where(none, 0.0, a.float() * b.float()).half()
    assert torch.equal(km.cluster_linear(X, W, plan), product(X, W[at, 0]))
    dX, dW = km.cluster_linear_backward(dY, X, W, plan)
    assert torch.equal(dX, product(dY, W[at, 0]))
    want = torch.zeros(k, dtype=torch.float16, device=DEV)
    want[at[~none[:, 0]]] = product(dY, X)[~none]
    assert torch.equal(dW[:, 0, 0], want)


def test_one_column_in_8_bits():
    n = k = 2 ** 24 + 2 ** 20 + 77
    g, ids, plan = _clusters(n, k)
    q = lambda *s: km.quantize_blocks(torch.randn(*s, generator=g, device=DEV))
    X, W = q(n, 1), q(k, 1, 1)
    x, w = km.dequantize_blocks(X), km.dequantize_blocks(W)[ids.clamp_min(0).long(), 0]
    for dtype in (torch.float32, torch.bfloat16):
        y = km.cluster_linear_fp8(X, W, plan, dtype=dtype)
        assert torch.equal(y, torch.where((ids < 0)[:, None], 0.0, x * w).to(dtype))


def test_wide_results():
    n, k, dout = 2 ** 22, 2 ** 22 + 5, 301   # five tiles of columns a row
    g, ids, plan = _clusters(n, k)
    X = torch.randn(n, 1, generator=g, device=DEV).half()
    W = torch.randn(k, dout, 1, generator=g, device=DEV).half()
    y = km.cluster_linear(X, W, plan)
    for part in torch.arange(n, device=DEV).split(2 ** 18):
        i = ids[part]
        want = torch.where((i < 0)[:, None], 0.0, X[part].float() * W[i.clamp_min(0).long(), :, 0].float()).half()
        assert torch.equal(y[part], want)
