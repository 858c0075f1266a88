"""Sizes beyond 32 bits are refused by the operators' bindings, not taken for their low
bits.  Tensors without memory stand for the GPU's: the refusals come before any is
read."""
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import paper_1902_09527_amd as km
from paper_1902_09527_amd import _native as N

BIG = 2 ** 32 + 8   # low bits: 8


def _calls():
    t = lambda *s, dtype=torch.bfloat16: torch.empty(*s, dtype=dtype, device="cuda:0")
    ids = lambda n: t(n, dtype=torch.int32)
    plan = lambda n, k: km.ClusterPlan(ids(n), ids(n), ids(n), ids(k + 1), n, 1, k)
    blocks = lambda *s: km.BlockRows(t(*s, dtype=torch.float8_e4m3fn),
                                     t(*s[:-1], (s[-1] + 127) // 128, dtype=torch.uint8))
    return {
        "rows of a table": lambda: km.cluster_embedding(ids(4), t(BIG, 8)),
        "columns of a table": lambda: km.cluster_embedding(ids(4), t(8, BIG)),
        "columns of a gradient": lambda: km.cluster_embedding_backward(t(4, BIG), plan(4, 8)),
        "columns moved": lambda: km.cluster_gather(t(4, BIG), plan(4, 8)),
        "columns combined": lambda: km.cluster_combine(t(4, BIG), plan(4, 8)),
        "columns normalised": lambda: km.layernorm(t(4, BIG)),
        "columns quantised": lambda: km.quantize_blocks(t(4, BIG)),
        "columns of blocks": lambda: km.dequantize_blocks(blocks(4, BIG)),
        "results of a projection": lambda: km.adapter_linear(t(4, 8), t(BIG, 8), t(8, 8, 8), t(8, BIG, 8), ids(4)),
        "adapters": lambda: km.adapter_linear(t(4, 8), t(8, 8), t(BIG, 8, 8), t(BIG, 8, 8), ids(4)),
        "rank": lambda: km.adapter_linear(t(4, 8), t(8, 8), t(8, BIG, 8), t(8, 8, BIG), ids(4)),
        "results of weights": lambda: km.cluster_linear(t(4, 8), t(8, BIG, 8), plan(4, 8)),
        "columns of weights": lambda: km.cluster_linear(t(4, BIG), t(8, 8, BIG), plan(4, 8)),
        "results of their gradients": lambda: km.cluster_linear_backward(t(4, BIG), t(4, 8), t(8, BIG, 8), plan(4, 8)),
        "results in 8 bits": lambda: km.cluster_linear_fp8(t(4, 8), blocks(8, BIG, 8), plan(4, 8)),
        "columns in 8 bits": lambda: km.cluster_linear_fp8(blocks(4, BIG), blocks(8, 8, BIG), plan(4, 8)),
    }


@pytest.mark.parametrize("which", ["rows of a table", "columns of a table", "columns of a gradient", "columns moved",
                                   "columns combined", "columns normalised", "columns quantised", "columns of blocks",
                                   "results of a projection", "adapters", "rank", "results of weights",
                                   "columns of weights", "results of their gradients", "results in 8 bits",
                                   "columns in 8 bits"])
def test_beyond_32_bits(which):
    with FakeTensorMode(), torch.no_grad():
        with pytest.raises(N.KMError) as e:
            _calls()[which]()
    assert e.value.status == N.KM_ERR_INVALID_ARG and "at most 2^" in str(e.value)
