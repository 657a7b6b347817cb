"""Points of several sources, one shared model, a small part of each source's own.

Exact kernel K-means gives ids to points.  The same points come from several
sources whose features are off in ways of their own (a few directions turned and
scaled), so one shared projection does not fit all.  The steps:

1. cluster the points (Gaussian kernel, K-means++ seeding);
2. shared: a projection, which stays as it is, and a class head on it, trained on
   the clean points' ids;
3. each source trains a low-rank adapter beside the projection: the adapted
   projection, the head's cross entropy, both gradients, and an update along the
   orthogonalised momentum;
4. new points of every source get ids from the adapted model's logits, empty
   clusters masked out.

    python examples/adapt_sources.py [--points 6000] [--sources 4] [--steps 40]
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from examples.learn_ids import cluster  # noqa: E402
from paper_2601_17136_amd import datagen, kkm  # noqa: E402


class Model:
    """y = w x + the source's adapter, logits = head y."""

    def __init__(self, ctx, d, width, classes, sources, rank, seed=0):
        import torch
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*shape):
            return torch.randn(*shape, device="cuda", generator=gen)

        self.ctx, self.classes = ctx, classes
        self.w = normal(width, d) / d ** 0.5
        self.head = torch.zeros(classes, width, device="cuda")
        # down starts at random and up at zero: no source differs from the shared model at first
        self.down, self.up = normal(sources, rank, d) / d ** 0.5, torch.zeros(sources, width, rank, device="cuda")
        self.speeds = [torch.zeros_like(t) for t in (self.head, self.down, self.up)]

    def features(self, x, sources):
        import torch
        y = torch.empty(x.shape[0], self.w.shape[0], device="cuda")
        kkm.kkm_adapted_linear(self.ctx, x, self.w, self.down, self.up, sources, y)
        return y

    def step(self, x, sources, ids, rate, shared):
        """One update, of the head (shared) or of the adapters.  Returns the mean loss."""
        import torch
        n = x.shape[0]
        y = self.features(x, sources)
        loss, lse, dloss = (torch.full((n,), 1.0 / n, device="cuda") for _ in range(3))
        dy, dhead = torch.empty_like(y), torch.empty_like(self.head)
        kkm.kkm_head_grad(self.ctx, y, self.head, ids, dloss, loss, lse, dy, dhead)
        if shared:
            kkm.kkm_orthogonal_step(self.ctx, self.head, dhead, self.speeds[0], rate)
        else:
            ddown, dup = torch.empty_like(self.down), torch.empty_like(self.up)
            kkm.kkm_adapted_linear_grad(self.ctx, x, self.w, self.down, self.up, sources, dy, None, ddown, dup)
            kkm.kkm_orthogonal_step(self.ctx, self.down, ddown, self.speeds[1], rate)
            kkm.kkm_orthogonal_step(self.ctx, self.up, dup, self.speeds[2], rate)
        return float(loss.mean())

    def assign(self, x, sources, masks=None, mask_ids=None):
        """Ids of new points and their log probabilities."""
        import torch
        logits = self.features(x, sources) @ self.head.t()
        ids, logp = torch.empty(x.shape[0], dtype=torch.int32, device="cuda"), torch.empty(x.shape[0], device="cuda")
        kkm.kkm_choose(self.ctx, logits, None, ids, logp, masks=masks, mask_ids=mask_ids)
        return ids, logp


def distort(x, sources, count, seed):
    """Each source's own change of a few directions of its points."""
    import torch
    d = x.shape[1]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    out = x.clone()
    for s in range(count):
        a, b = (torch.randn(d, 3, device="cuda", generator=gen) / d ** 0.5 for _ in range(2))
        mine = sources == s
        out[mine] += 5.0 * (x[mine] @ a) @ b.t()
    return out


def run(points=6000, new=600, clusters=8, dims=48, width=64, sources=4, rank=6, steps=40, seed=0, log=print):
    import torch
    X, _ = datagen.make_points(2, n=points + new, d=dims)
    X = torch.from_numpy(X).cuda()
    X = ((X - X.mean(0)) / (X.std(0) + 1e-3)).contiguous()
    ctx = kkm.kkm_create(kkm.current_stream_handle())
    try:
        all_ids, counts, _, _ = cluster(ctx, X, 1.0 / dims, clusters, seed)
        ids, want = all_ids[:points].contiguous(), all_ids[points:]
        gen = torch.Generator(device="cuda").manual_seed(seed + 1)
        source = torch.randint(0, sources, (points + new,), device="cuda", generator=gen).int()
        seen = distort(X, source, sources, seed + 2)
        old, old_source = seen[:points].contiguous(), source[:points].contiguous()
        fresh, fresh_source = seen[points:].contiguous(), source[points:].contiguous()
        model = Model(ctx, dims, width, clusters, sources, rank, seed)
        none = torch.full((points,), -1, dtype=torch.int32, device="cuda")
        # a bit per cluster that is not empty
        masks = torch.zeros(1, (clusters + 31) // 32, dtype=torch.int64, device="cuda")
        for v in torch.nonzero(counts > 0)[:, 0].tolist():
            masks[0, v // 32] |= 1 << v % 32
        masks = torch.where(masks >= 2 ** 31, masks - 2 ** 32, masks).int()
        mask_ids = torch.zeros(new, dtype=torch.int32, device="cuda")

        def agree():
            got, _ = model.assign(fresh, fresh_source, masks, mask_ids)
            return float((got == want).float().mean())

        out = {"shared": [model.step(X[:points].contiguous(), none, ids, 0.05, True) for _ in range(steps)]}
        before = agree()
        out["adapters"] = [model.step(old, old_source, ids, 0.02, False) for _ in range(steps)]
        out["agree"] = (before, agree())
        for name in ("shared", "adapters"):
            log(f"{name}: mean loss {out[name][0]:.4f} -> {out[name][-1]:.4f}")
        log(f"new points assigned as clustered: {before:.1%} by the shared model, {out['agree'][1]:.1%} with adapters")
        return out
    finally:
        kkm.kkm_destroy(ctx)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--points", type=int, default=6000)
    ap.add_argument("--sources", type=int, default=4)
    ap.add_argument("--rank", type=int, default=6)
    ap.add_argument("--steps", type=int, default=40)
    run(**vars(ap.parse_args()))
