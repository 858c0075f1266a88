"""A layer conditioned on clusters: clustering, training and serving.

    python examples/cluster_layer.py [--rows 16384] [--dim 256] [--clusters 32]

Rows (token embeddings) are layer-normed and clustered with k-means; each row
goes to its two nearest clusters, through a shared projection that is frozen
and a low-rank adapter per cluster that is trained, and comes back as the
weighted sum of the two results.  A few steps of gradient descent on the
adapters and the norm's parameters lower the loss; then single rows are served
with the adapter of their nearest cluster.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1902_09527_amd as km  # noqa: E402


class Layer:
    """Parameters in bfloat16 as the kernels take them, float32 copies of the trained ones."""

    def __init__(self, dim, out, clusters, rank, device, seed=0):
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=g, device=device)
        self.W = (r(out, dim) * dim ** -0.5).bfloat16()
        self.scale = torch.full((clusters,), 2.0, device=device)
        self.master = {"A": r(clusters, rank, dim) * dim ** -0.5, "B": torch.zeros(clusters, out, rank, device=device),
                       "gamma": torch.ones(dim, device=device), "beta": torch.zeros(dim, device=device)}
        self.refresh()

    def refresh(self):
        self.A, self.B = self.master["A"].bfloat16(), self.master["B"].bfloat16()

    def forward(self, X, ids, weights):
        """(result, what the backward pass needs).  ids: int32 [n, m]; weights: float32 [n, m]."""
        m = self.master
        N, mean, rstd = km.layernorm(X, m["gamma"], m["beta"])
        plan = km.cluster_sort(ids, len(self.scale))
        Ns = km.cluster_gather(N, plan)
        Z, H = km.adapter_linear(Ns, self.W, self.A, self.B, plan, self.scale, sorted_rows=True)
        return km.cluster_combine(Z, plan, weights), (X, mean, rstd, plan, Ns, Z, H, weights)

    def backward(self, dY, saved):
        """Gradients of the parameters, the rows and the router's weights."""
        X, mean, rstd, plan, Ns, Z, H, weights = saved
        dZ, dw = km.cluster_combine_backward(dY, Z, plan, weights)
        dNs, dA, dB = km.adapter_linear_backward(dZ, Ns, H, self.W, self.A, self.B, plan, self.scale,
                                                 sorted_rows=True)
        dN = km.cluster_combine(dNs, plan)
        dX, dgamma, dbeta = km.layernorm_backward(dN, X, mean, rstd, self.master["gamma"])
        return {"A": dA, "B": dB, "gamma": dgamma, "beta": dbeta}, dX, dw

    def update(self, grads, rates):
        for name, g in grads.items():
            self.master[name].sub_(g.float(), alpha=rates[name])
        self.refresh()

    def serve(self, X, ids):
        """Few rows, one cluster each."""
        N, _, _ = km.layernorm(X, self.master["gamma"], self.master["beta"])
        return km.adapter_linear(N, self.W, self.A, self.B, ids, self.scale)[0]


def route(N, centroids, slots=2):
    """The nearest clusters of each row and their weights."""
    d = torch.cdist(N.float(), centroids)
    near, ids = torch.topk(d, slots, dim=1, largest=False)
    return ids.to(torch.int32).contiguous(), torch.softmax(-near, 1).contiguous()


def main(rows=16384, dim=256, out=384, clusters=32, rank=16, steps=20, seed=0, device="cuda:0"):
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    centres = torch.randn(clusters, dim, generator=g, device=device) * 2
    kind = torch.randint(0, clusters, (rows,), generator=g, device=device)
    X = (centres[kind] + torch.randn(rows, dim, generator=g, device=device)).bfloat16()
    layer = Layer(dim, out, clusters, rank, device, seed)

    # Cluster the normed rows: k-means++ seeds, then k-means.
    N = km.layernorm(X)[0].float()
    u = torch.rand(clusters, generator=torch.Generator().manual_seed(seed), dtype=torch.float64).numpy()
    assign, centroids, stats = km.run(N, km.kmeanspp(N, clusters, u)["C"], max_iters=20)
    ids, weights = route(N, centroids)
    weights[:, 0] = 1 - weights[:, 1:].sum(1)

    # Every kind of row has a target map of its own.
    shift = torch.randn(clusters, out, generator=g, device=device)
    target = (N @ layer.W.float().T + shift[kind]).bfloat16()
    # Steps below the curvature's inverse: of B about 8 rank / clusters, of A
    # dim / rank times that and more as B grows; the norm's parameters act on
    # every row through W (largest squared singular value about
    # (1 + sqrt(out / dim))^2).
    slow = 0.05 / (1 + (out / dim) ** 0.5) ** 2
    rates = {"A": 0.002 * clusters / dim, "B": 0.025 * clusters / rank, "gamma": slow, "beta": slow}
    losses = []
    for _ in range(steps):
        Y, saved = layer.forward(X, ids, weights)
        diff = Y.float() - target.float()
        losses.append(float((diff * diff).mean()))
        grads, _, _ = layer.backward((diff * (2.0 / rows)).bfloat16(), saved)
        layer.update(grads, rates)
    served = layer.serve(X[:4], assign[:4].contiguous())
    return {"losses": losses, "iterations": stats["iterations"], "served": served, "clusters": clusters}


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("rows", 16384), ("dim", 256), ("out", 384), ("clusters", 32), ("rank", 16), ("steps", 20)):
        ap.add_argument("--" + name, type=int, default=value)
    r = main(**vars(ap.parse_args()))
    print("k-means: %d iterations; loss %.4f -> %.4f in %d steps; served %s" % (
        r["iterations"], r["losses"][0], r["losses"][-1], len(r["losses"]), tuple(r["served"].shape)))
