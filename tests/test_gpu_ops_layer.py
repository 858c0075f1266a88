"""The operators together, as examples/cluster_layer.py runs them: the whole
layer's result and gradients against float64 autograd of its formula, and a
short training run that lowers its loss."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("cluster_layer", os.path.join(ROOT, "examples", "cluster_layer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_layer_against_float64_autograd():
    """Five results of this chain are rounded to bfloat16 (u = 2^-8) one after
    the other, each with a relative error of at most u; sums of many such
    errors with random signs stay well below their sum.  The bar is 5 u of the
    result's norm."""
    m = _example()
    n, dim, out, k, r = 700, 64, 48, 6, 8
    layer = m.Layer(dim, out, k, r, DEV, seed=3)
    layer.master["B"] = torch.randn(k, out, r, device=DEV) * 0.3
    layer.refresh()
    X = torch.randn(n, dim, device=DEV).bfloat16()
    ids = torch.stack([torch.randint(0, k, (n,), device=DEV), torch.randint(-1, k, (n,), device=DEV)], 1).int()
    w = torch.rand(n, 2, device=DEV)
    Y, saved = layer.forward(X, ids, w)
    dY = torch.randn(n, out, device=DEV).bfloat16()
    grads, dX, dw = layer.backward(dY, saved)

    f = lambda t: t.detach().double().requires_grad_()
    x, a, b, ga, be, ww = f(X), f(layer.A), f(layer.B), f(layer.master["gamma"]), f(layer.master["beta"]), f(w)
    xn = torch.nn.functional.layer_norm(x, (dim,), ga, be, 1e-5)
    y = torch.zeros(n, out, dtype=torch.float64, device=DEV)
    for j in range(2):
        c = ids[:, j].long()
        used = (c >= 0)[:, None]
        c = c.clamp_min(0)
        h = (a[c] * xn[:, None, :]).sum(2)
        z = xn @ layer.W.double().T + layer.scale.double()[c][:, None] * (b[c] * h[:, None, :]).sum(2)
        y = y + torch.where(used, ww[:, j:j + 1] * z, 0.0)
    y.backward(dY.double())
    for name, got, want in (("Y", Y, y), ("dX", dX, x.grad), ("dw", dw, ww.grad), ("A", grads["A"], a.grad),
                            ("B", grads["B"], b.grad), ("gamma", grads["gamma"], ga.grad),
                            ("beta", grads["beta"], be.grad)):
        rel = float((got.double() - want.detach()).norm() / want.detach().norm())
        assert rel < 5 * 2.0 ** -8, (name, rel)


def test_training_lowers_the_loss_and_serves():
    r = _example().main(rows=4096, dim=128, out=96, clusters=12, rank=8, steps=15)
    assert r["losses"][-1] < 0.7 * r["losses"][0]
    assert all(b < a for a, b in zip(r["losses"], r["losses"][1:]))
    assert r["served"].shape == (4, 96) and torch.isfinite(r["served"].float()).all()
