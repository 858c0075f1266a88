"""Tensors with a forward-mode tangent: refused, with or without grad mode, as the
library's calls would lose it; tensors without memory stand for the GPU's."""
import pytest
import torch
import torch.autograd.forward_ad as fw
from torch._subclasses.fake_tensor import FakeTensorMode

import paper_1902_09527_amd as km
from paper_1902_09527_amd import ops


def _calls(x):
    t = lambda *s, dtype=torch.float32: torch.empty(*s, dtype=dtype, device="cuda:0")
    ids = lambda n: t(n, dtype=torch.int32)
    n, d, k = x.shape[0], x.shape[1], 3
    plan = km.ClusterPlan(ids(n), ids(n), ids(n), ids(k + 1), n, 1, k)
    W = km.BlockRows(t(k, 8, d, dtype=torch.float8_e4m3fn), t(k, 8, 1, dtype=torch.uint8))
    return [lambda: km.cluster_gather(x, plan), lambda: km.cluster_combine(x, plan),
            lambda: km.cluster_combine_backward(x, t(n, d), plan, t(n)), lambda: km.layernorm(x),
            lambda: km.layernorm_backward(t(n, d), x, t(n), t(n)),
            lambda: km.adapter_linear(x, t(d, d), t(k, 4, d), t(k, d, 4), ids(n)),
            lambda: km.adapter_linear_backward(t(n, d), x, t(n, 4), t(d, d), t(k, 4, d), t(k, d, 4), plan),
            lambda: km.cluster_linear(x, t(k, 8, d), plan),
            lambda: km.cluster_linear_backward(t(n, 8), x, t(k, 8, d), plan),
            lambda: km.quantize_blocks(x), lambda: km.cluster_linear_fp8(x, W, plan),
            lambda: km.cluster_embedding(ids(n), x), lambda: km.cluster_embedding_backward(x, plan),
            lambda: km.global_norm([t(4), x]), lambda: km.clip_global_norm([t(4), x], 1.0),
            lambda: km.clip_global_norm([t(n, d)], 1.0, out=[x])]


@pytest.mark.parametrize("which", range(16))
def test_tangents_are_refused(which):
    with FakeTensorMode(), fw.dual_level():
        x = torch.empty(6, 16, device="cuda:0")
        with pytest.raises(ValueError, match="tangent"):
            _calls(fw.make_dual(x, torch.empty(6, 16, device="cuda:0")))[which]()
        with torch.no_grad(), pytest.raises(ValueError, match="tangent"):
            _calls(fw.make_dual(x, torch.empty(6, 16, device="cuda:0")))[which]()


def test_what_is_not_refused():
    """Tensors without a tangent while a level is open, and those whose tangent an
    autograd.Function takes care of itself."""
    x = torch.ones(3)
    seen = []

    class F(torch.autograd.Function):
        @staticmethod
        def forward(ctx, v):
            ops._not_followed((v, None))
            seen.append(True)
            return 2 * v

        @staticmethod
        def jvp(ctx, t):
            return 2 * t

    with fw.dual_level():
        d = fw.make_dual(x, torch.full((3,), 5.0))
        ops._not_followed((x, None, torch.zeros(2, dtype=torch.int32)))
        with pytest.raises(ValueError, match="tangent"):
            ops._not_followed((x, d))
        assert bool((fw.unpack_dual(F.apply(d)).tangent == 10).all()) and seen
    ops._not_followed((x,))
