"""A model of routed linear experts whose router is a clustering: ASGD learns the centroids, their scores route the samples, and
the experts and the router are then trained by gradient steps through the 8-bit products.

    python -m paper_1505_04956_amd.clusterwise [--samples N] [--steps S] [--shared] [--limit L] [--small]

The samples are a mixture around k centres (the generator of the clustering workloads); the target of a sample is a linear map of it
that differs from centre to centre, so a model that sends every sample to the map of its cluster can learn what one map cannot.  With
--shared every sample also passes through one map that all clusters have in common, so that the experts learn what differs.  With --limit
a step's gradients are clipped to that norm, with --small the trained maps are also evaluated in 4 bits.
"""
from __future__ import annotations

import argparse

import numpy as np
import torch

from . import binding as B
from . import experts as X
from . import gradients as G
from . import micro as M
from . import workloads


class ClusterwiseLinear:
    """y = sum over the best `choices` clusters e of weight_e(x) * W_e x, and with `shared` S x of one map for all.  Master weights and centroids
    are float32; the products see them in 8-bit blocks, laid out again after each step."""

    def __init__(self, centroids, outputs, choices=2, seed=0, sharpness=1.0, shared=False):
        k, d = centroids.shape
        gen = torch.Generator(device=centroids.device)
        gen.manual_seed(seed)
        self.centroids, self.sharpness = centroids, sharpness
        self.w = torch.randn((k, outputs, d), generator=gen, device=centroids.device) / d ** 0.5
        self.shared = torch.zeros((outputs, d), device=centroids.device) if shared else None
        self.rule = X.Rule(choices, score=X.SOFTMAX)

    def logits(self, x, centroids=None):
        c = self.centroids if centroids is None else centroids
        return self.sharpness * (x @ c.t() - 0.5 * (c * c).sum(1))

    def forward(self, x, train=False):
        logits = self.logits(x)
        ids, weights = X.route(logits, self.rule)
        x = x.bfloat16()
        y = X.experts(x, ids, weights, X.quantize_weights(self.w), train=train)
        y, kept = y if train else (y, None)
        of_all = None
        if self.shared is not None:
            s = X.linear(x, X.quantize_weights(self.shared), train=train)
            s, of_all = s if train else (s, None)
            y = y.float() + s.float()
        return (y, (logits, ids, kept, of_all)) if train else y

    def small(self):
        """The maps in 4 bits, kept for evaluation with the router that belongs to them: a function of samples x that gives what forward(x) does now, also
        when the model is trained on, at a quarter of 16-bit weights' bytes."""
        centroids = self.centroids.clone()
        w = M.quantize(self.w)
        shared = None if self.shared is None else M.quantize(self.shared)

        def forward(x):
            ids, weights = X.route(self.logits(x, centroids), self.rule)
            x = x.bfloat16()
            y = M.experts(x, ids, weights, w)
            return y if shared is None else y.float() + M.linear(x, shared).float()
        return forward

    def step(self, x, target, rate, limit=None):
        """One step against half the mean squared error, its gradients clipped to the norm `limit`; returns that error before the step."""
        y, (logits, ids, kept, of_all) = self.forward(x, train=True)
        off = y.float() - target
        loss = 0.5 * (off * off).sum(1).mean()
        d_y = (off / len(x)).bfloat16()
        _, d_w, d_weights = X.experts_backward(d_y, kept, X.quantize_weights(self.w, turned=True))
        d_logits = X.route_backward(logits, self.rule, ids, d_weights)
        d_c = self.sharpness * (d_logits.t() @ x - d_logits.sum(0)[:, None] * self.centroids)
        if of_all is not None:
            _, d_shared = X.linear_backward(d_y, of_all, X.quantize_weights(self.shared, turned=True))
        if limit is not None:
            G.clip([d_w, d_c] if of_all is None else [d_w, d_c, d_shared], limit)
        if of_all is not None:
            self.shared -= rate * self.rule.k / len(self.w) * d_shared         # (all rows pass through it, so many times more than through an expert)
        self.w -= rate * d_w
        self.centroids = self.centroids - rate * d_c
        return loss


def learn_centroids(x, k, workers=64, minibatch=500, epochs=3):
    """k centroids of the samples x [N, d] float32 on the GPU by ASGD (one common start, so that the workers' means are means of
    the same clusters)."""
    g = B.ASGD(k, x.shape[1], workers, minibatch, 0.05, E=4)
    g.load_shards(x)
    pick = torch.randperm(len(x), generator=torch.Generator().manual_seed(1))[:k]
    g.set_state(-1, x[pick.to(x.device)].cpu().numpy())
    g.run_epochs(epochs)
    w = torch.from_numpy(np.ascontiguousarray(g.get_mean_state())).to(x.device)
    g.close()
    return w


def run(samples=200_000, steps=60, k=16, d=32, outputs=24, batch=8192, rate=0.05, seed=1234, shared=False, report=None, limit=None, small=None):
    """(losses of the steps, loss of the best single linear map) on one synthetic data set.  limit: of the norm of a step's gradients; small: is given the
    loss of the trained model over all samples in 8 and in 4 bits."""
    wl = workloads.Workload("clusterwise", samples, d, k, 64, 500, 0.05, 4, 3, 1.0, "uniform10", "equal", data_seed=seed)
    x = torch.from_numpy(workloads.generate_host(wl)).cuda()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    centroids = learn_centroids(x, k)
    x = x - x.mean(0)                                                     # products in 8 bits lose least around the origin
    centroids = centroids - centroids.mean(0)
    maps = torch.randn((k, outputs, d), generator=gen, device="cuda") / d ** 0.5
    near = (x @ centroids.t() - 0.5 * (centroids * centroids).sum(1)).argmax(1)
    target = torch.empty((samples, outputs), device="cuda")
    for e in range(k):
        target[near == e] = x[near == e] @ maps[e].t()
    one = torch.linalg.lstsq(x.cpu(), target.cpu()).solution.cuda()
    single = 0.5 * (x @ one - target).square().sum(1).mean().item()
    model = ClusterwiseLinear(centroids, outputs, shared=shared)
    losses = []
    for s in range(steps):
        at = torch.randint(0, samples, (batch,), generator=gen, device="cuda")
        losses.append(model.step(x[at], target[at], rate, limit).item())
        if report:
            report("step %d: loss %.4f" % (s, losses[-1]))
    if small:
        small(*(0.5 * (f(x).float() - target).square().sum(1).mean().item() for f in (model.forward, model.small())))
    return losses, single


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--samples", type=int, default=200_000)
    p.add_argument("--steps", type=int, default=60)
    p.add_argument("--shared", action="store_true")
    p.add_argument("--limit", type=float)
    p.add_argument("--small", action="store_true")
    a = p.parse_args()
    got, alone = run(a.samples, a.steps, shared=a.shared, report=print, limit=a.limit,
                     small=(lambda eight, four: print("loss over all samples in 8 bits %.4f, in 4 bits %.4f" % (eight, four))) if a.small else None)
    print("loss %.4f after %d steps; the best single linear map: %.4f" % (got[-1], len(got), alone))
