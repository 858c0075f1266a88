"""Gradients of the rows where the tile does not divide the width: its last tile of
columns moves left until it is whole.  Weights that fill whole 2 MB pages, so that
nothing of theirs lies behind them, and tiles of 256, 128 and 64."""
import pytest
import torch

import paper_1902_09527_amd as km
from test_gpu_ops_linear import TYPES, _case, _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,din,dout,k", [(16_384, 1408, 4096, 8), (65_536, 1408, 2048, 64), (16_384, 320, 1024, 16),
                                          (16_384, 576, 1024, 32), (16_384, 2040, 2048, 64), (300, 320, 1024, 16),
                                          (2000, 72, 1024, 4), (500, 4064, 128, 3)])
def test_last_tile_of_columns(n, din, dout, k, dtype):
    print("case", n, din, dout, k, dtype, flush=True)
    c = _case(n + din, n, din, dout, k, dtype)
    plan = km.cluster_sort(c["ids"], k)
    y = km.cluster_linear(c["X"], c["W"], plan)
    dx, dw = km.cluster_linear_backward(c["dY"], c["X"], c["W"], plan)
    _check(c, y, dx, dw)
    at = plan.order.long()
    assert torch.equal(km.cluster_linear_backward(c["dY"][at], c["X"][at], c["W"], plan, sorted_rows=True,
                                                  need_dW=False)[0], dx[at])
