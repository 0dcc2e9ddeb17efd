"""A frozen backbone with 4-bit weights from loading to adapter training.

    python examples/mx4_backbone.py

1. The projections of a few pre-norm layers are quantised to mx4 (runtime.Mx4Linear); a layer is
       o = n W^T,   y = res x + gate N(o) w_post,   n' = N(y) w_pre      (runtime.BlockNorm, one call for the second and third)
2. What 4 bits lost is partly recovered: norms, gates and residual scales are tuned against the states of the full-precision
   layers, with the exact gradients through norms (BlockNorm.backward) and frozen projections (Mx4Linear.input_grad).
3. The first epoch: every sample goes through the layers once, four bits on both sides, and the layers' states fill the cache.
4. Later epochs train the side adapters from the cache alone (runtime.Session).

Weights, samples and labels are seeded random numbers.
"""
from __future__ import annotations

import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2408_10746_amd import runtime as rt  # noqa: E402
from paper_2408_10746_amd.inputs import Workload  # noqa: E402


class Backbone:
    """`layers` frozen projections with their norms; parameters of the norms are the only ones that are ever tuned."""

    def __init__(self, weights, device):
        self.d, self.dev = weights[0].shape[0], device
        self.linear = [rt.Mx4Linear.from_weights(w) for w in weights]
        one = lambda n, at: torch.full((n,), at, device=device)  # noqa: E731
        self.params = [dict(w_post=one(self.d, 1.0), gate=one(1, 0.5), res=one(1, 1.0), w_pre=one(self.d, 1.0)) for _ in weights]
        self.first = rt.BlockNorm(self.d, w_pre=one(self.d, 1.0))
        self.norm = [rt.BlockNorm(self.d, **p) for p in self.params]

    def forward(self, x, x4: bool = False):
        """States of every layer and what the way back needs: [(x, o, y)]."""
        n, seen = torch.empty_like(x), []
        self.first.forward(x, n=n)
        for linear, norm in zip(self.linear, self.norm):
            o, y, after = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
            linear.forward(n, o, x4=x4)
            norm.forward(x, o, y, after)
            seen.append((x, o, y))
            x, n = y, after
        return seen

    def backward(self, seen, dy):
        """Gradients of the norms' parameters, given that of the last layer's states (whose own norm nobody reads)."""
        grads = [{k: torch.empty_like(p) for k, p in ps.items()} for ps in self.params]
        dn = torch.zeros_like(dy)
        for (x, o, _), linear, norm, g in zip(reversed(seen), reversed(self.linear), reversed(self.norm), reversed(grads)):
            dx, do, before = torch.empty_like(dy), torch.empty_like(dy), torch.empty_like(dy)
            norm.backward(x, o, dy, dn, dx, do, g)
            linear.input_grad(do, before)
            dy, dn = dx, before
        return grads


def full_precision(x, weights):
    """The same layers on unquantised weights, for the states that tuning aims at."""
    rms = lambda z: z / torch.sqrt((z * z).mean(-1, keepdim=True) + 1e-5)  # noqa: E731
    x = x.float()
    n = rms(x)
    for w in weights:
        x = x + 0.5 * rms(n @ w.t())
        n = rms(x)
    return x


def main(layers=4, d=256, tokens=64, samples=32, steps=30, epochs=4, device="cuda:0", say=print):
    dev = torch.device(device)
    torch.cuda.set_device(dev)
    g = torch.Generator(device=dev).manual_seed(0)
    weights = [torch.randn(d, d, generator=g, device=dev) / d ** 0.5 for _ in range(layers)]
    net = Backbone(weights, dev)

    # ---- tuning norms and gates, 16 samples' tokens a step
    tuned = []
    for step in range(steps):
        x = torch.randn(16 * tokens, d, generator=g, device=dev).bfloat16()
        seen = net.forward(x)
        off = seen[-1][2].float() - full_precision(x, weights)
        tuned.append(float((off * off).mean()))
        for ps, gs in zip(net.params, net.backward(seen, (2 * off / off.numel()).bfloat16())):
            for k, p in ps.items():
                p -= 0.05 * p.numel() * gs[k]  # a vector's values share the mean's curvature between them
    say(f"distance to the full-precision states: {tuned[0]:.5f} before tuning, {tuned[-1]:.5f} after {steps} steps")

    # ---- first epoch: states of all layers into the cache
    w = Workload("mx4_example", L=layers, d=d, n_max=tokens, B=8, r=32, C=2, N=samples, cache_dtype="bf16")
    sess = rt.Session(w, device=device)
    labels = torch.randint(0, 2, (samples,), generator=g, device=dev, dtype=torch.int32)
    for at in range(0, samples, w.B):
        # a class shifts its samples' embeddings, so that there is something to learn
        x = (torch.randn(w.B, tokens, d, generator=g, device=dev) + 0.25 * (2 * labels[at:at + w.B, None, None] - 1)).bfloat16()
        seen = net.forward(x.view(-1, d), x4=True)
        acts = torch.stack([y.view(w.B, tokens, d) for _, _, y in seen], 1).contiguous()
        sess.cache_fill(np.arange(at, at + w.B), acts)

    # ---- later epochs: adapters from the cache
    rng, losses = np.random.default_rng(0), []
    p0 = np.zeros(sess.P, dtype=np.float32)
    for layer in range(layers):
        wd, _, _, _, lam = rt.pb.pac_param_offsets(sess.ctx, layer)
        p0[wd:wd + d * w.r] = rng.standard_normal(d * w.r) / d ** 0.5
        p0[lam] = 0.5
    cls = rt.pb.pac_param_offsets(sess.ctx, -1)[0]
    p0[cls:cls + d * w.C] = rng.standard_normal(d * w.C) / d ** 0.5
    sess.set_params(p0)
    for _ in range(epochs):
        order = rng.permutation(samples)
        for at in range(0, samples, w.B):
            ids = order[at:at + w.B]
            sess.step(ids, labels[torch.from_numpy(ids).to(dev)].contiguous())
            losses.append(float(sess.loss.item()))
    say(f"adapter training from the cache: loss {losses[0]:.4f} at the first step, {losses[-1]:.4f} at the last of {len(losses)}")
    return tuned, losses


if __name__ == "__main__":
    main()
