"""Tensors that require gradients: refused while autograd would follow the call
(it records nothing of it), taken without grad mode and in the forward and
backward of an autograd.Function."""
import pytest
import torch

import paper_1902_09527_amd as km

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _calls():
    n, m, d, k, r = 12, 2, 16, 3, 4
    ids = (torch.arange(n * m, device=DEV) % k).to(torch.int32).view(n, m)
    plan, one = km.cluster_sort(ids, k), km.cluster_sort(ids[:, 0].contiguous(), k)
    t = lambda *s: torch.randn(*s, device=DEV)
    X, Z, w, g, dY = t(n, d), t(n * m, d), t(n, m), t(d), t(n, d)
    W, A, B, s = t(d, d), t(k, r, d), t(k, d, r), t(k)
    y, mean, rstd = km.layernorm(X, g)
    y, h = km.adapter_linear(X, W, A, B, one, s)
    return [(km.cluster_gather, [X, plan]), (km.cluster_combine, [Z, plan, w]),
            (km.cluster_combine_backward, [dY, Z, plan, w]), (km.layernorm, [X, g, t(d)]),
            (km.layernorm_backward, [dY, X, mean, rstd, g]),
            (km.adapter_linear, [X, W, A, B, ids[:, 0].contiguous(), s]),
            (km.adapter_linear_backward, [dY, X, h, W, A, B, one, s])]


@pytest.mark.parametrize("which", range(7))
def test_inputs_that_require_gradients(which):
    f, args = _calls()[which]
    want = f(*args)
    want = want if isinstance(want, tuple) else (want,)
    for i, t in enumerate(args):
        if not isinstance(t, torch.Tensor) or not t.is_floating_point():
            continue
        given = list(args)
        given[i] = t.clone().requires_grad_()
        with pytest.raises(ValueError, match="requires a gradient"):
            f(*given)
        with torch.no_grad():
            got = f(*given)
        got = got if isinstance(got, tuple) else (got,)
        assert all(torch.equal(p, q) and not p.requires_grad for p, q in zip(got, want))


def test_in_an_autograd_function():
    class Norm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, g, b):
            y, mean, rstd = km.layernorm(x, g, b)
            ctx.save_for_backward(x, mean, rstd, g)
            return y

        @staticmethod
        def backward(ctx, dy):
            return km.layernorm_backward(dy, *ctx.saved_tensors)

    x, dy = torch.randn(9, 32, device=DEV), torch.randn(9, 32, device=DEV)
    g, b = torch.randn(32, device=DEV), torch.randn(32, device=DEV)
    _, mean, rstd = km.layernorm(x, g, b)
    want = km.layernorm_backward(dy, x, mean, rstd, g)
    leaves = [t.clone().requires_grad_() for t in (x, g, b)]
    Norm.apply(*leaves).backward(dy)
    assert all(torch.equal(t.grad, w) for t, w in zip(leaves, want))
