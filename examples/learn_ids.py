"""Learn a clustering: a small model that assigns new points.

Exact kernel K-means gives ids to the points it was run on.  A new point would
need its kernel values against all of them; a model trained on the ids answers
with one matrix product.  The steps:

1. cluster the points (Gaussian kernel, K-means++ seeding);
2. train layer norm + linear head on the ids: softmax cross entropy;
3. go on with the clustering's soft assignments: distillation from each point's
   nearest clusters, teacher logits -D / tau;
4. assign new points with the model, and count how many go where kernel K-means
   itself would put them.

    python examples/learn_ids.py [--points 8000] [--clusters 10] [--steps 60]
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2601_17136_amd import datagen, kkm  # noqa: E402


def cluster(ctx, X, gamma, k, seed):
    """Ids (device int32), their sizes and self-terms, and the points' distances to the clusters."""
    import torch
    n, d = X.shape
    kkm.kkm_build_kernel(ctx, X, n, d, kkm.KKM_GAUSS, kkm.make_params(gamma, k_hint=k))
    ids = torch.empty(n, dtype=torch.int32, device="cuda")
    kkm.kkm_init_kmeanspp(ctx, k, np.random.default_rng(seed).random(k), ids)
    kkm.kkm_iterate(ctx, ids, k, 50, 0.0)
    D, z = torch.empty(n, k, device="cuda"), torch.empty(k, device="cuda")
    kkm.kkm_step(ctx, ids, k, z=z, D=D)
    return ids, torch.bincount(ids.long(), minlength=k), z, D


class Model:
    """y = layer norm(x), logits = y w^T + log of the clusters' shares; plain gradient descent with momentum."""

    def __init__(self, ctx, d, counts, lr=0.5, momentum=0.9):
        import torch
        f32 = {"device": "cuda", "dtype": torch.float32}
        self.ctx, self.lr, self.momentum = ctx, lr, momentum
        self.params = [torch.ones(d, **f32), torch.zeros(d, **f32), torch.zeros(counts.numel(), d, **f32)]
        self.grads = [torch.empty_like(p) for p in self.params]
        self.speed = [torch.zeros_like(p) for p in self.params]
        self.offset = torch.log(counts.float() / counts.sum())  # -inf: an empty cluster is never the answer

    def _buffers(self, x):
        import torch
        n = x.shape[0]
        return torch.empty_like(x), *(torch.empty(n, device="cuda") for _ in range(4))

    def step(self, x, loss_and_gradient):
        """One descent step on all of x; loss_and_gradient(y, w, dloss, loss, lse, dy, dw).  Returns the mean loss."""
        import torch
        gamma, beta, w = self.params
        dgamma, dbeta, dw = self.grads
        y, mean, rstd, loss, lse = self._buffers(x)
        dloss, dy = torch.full_like(loss, 1.0 / x.shape[0]), torch.empty_like(x)
        kkm.kkm_layer_norm(self.ctx, x, gamma, beta, 1e-5, y, mean, rstd)
        loss_and_gradient(y, w, dloss, loss, lse, dy, dw)
        kkm.kkm_layer_norm_grad(self.ctx, x, gamma, dy, mean, rstd, None, dgamma, dbeta)
        for p, g, v in zip(self.params, self.grads, self.speed):
            v.mul_(self.momentum).add_(g)
            p.sub_(v, alpha=self.lr)
        return float(loss.mean())

    def assign(self, x):
        """Ids of new points."""
        import torch
        gamma, beta, w = self.params
        y = torch.empty_like(x)
        kkm.kkm_layer_norm(self.ctx, x, gamma, beta, 1e-5, y)
        return torch.argmax(y @ w.t() + self.offset, dim=1)


def kernel_assign(X, ids, counts, z, gamma, new):
    """Where kernel K-means puts new points: argmin_j z_j - 2/|L_j| sum_{i in L_j} K(new, i)."""
    import torch
    sums = torch.zeros(new.shape[0], counts.numel(), device="cuda", dtype=torch.float64)
    K = torch.exp(-gamma * torch.cdist(new.double(), X.double()) ** 2)
    sums.index_add_(1, ids.long(), K)
    D = torch.where(counts > 0, z.double() - 2 * sums / counts.clamp(min=1), float("inf"))
    return torch.argmin(D, dim=1)


def run(points=8000, new=1000, clusters=10, dims=64, steps=60, nearest=4, tau=0.05, seed=0, log=print):
    import torch
    X, _ = datagen.make_points(2, n=points + new, d=dims)
    X = torch.from_numpy(X).cuda()
    old, fresh = X[:points].contiguous(), X[points:].contiguous()
    gamma = 1.0 / dims
    ctx = kkm.kkm_create(kkm.current_stream_handle())
    try:
        ids, counts, z, D = cluster(ctx, old, gamma, clusters, seed)
        want = kernel_assign(old, ids, counts, z, gamma, fresh)
        top = torch.topk(-D / tau, nearest, dim=1)
        top_ids, top_logits = top.indices.to(torch.int32), top.values.contiguous()
        model = Model(ctx, dims, counts)

        def by_ids(y, w, dloss, loss, lse, dy, dw):
            kkm.kkm_head_grad(ctx, y, w, ids, dloss, loss, lse, dy, dw, offset=model.offset)

        def by_distances(y, w, dloss, loss, lse, dy, dw):
            kkm.kkm_distill_grad(ctx, y, w, top_ids, top_logits, dloss, loss, lse, dy, dw, offset=model.offset)

        out = {}
        for name, task in (("ids", by_ids), ("distances", by_distances)):
            losses = [model.step(old, task) for _ in range(steps)]
            agree = float((model.assign(fresh) == want).float().mean())
            log(f"{name}: mean loss {losses[0]:.4f} -> {losses[-1]:.4f}, new points assigned alike {agree:.1%}")
            out[name] = (losses, agree)
        return out
    finally:
        kkm.kkm_destroy(ctx)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--points", type=int, default=8000)
    ap.add_argument("--new", type=int, default=1000)
    ap.add_argument("--clusters", type=int, default=10)
    ap.add_argument("--dims", type=int, default=64)
    ap.add_argument("--steps", type=int, default=60)
    run(**vars(ap.parse_args()))
