"""Trains one pre-norm block with a gated feed-forward on a synthetic surface mesh.

    y   = x + PhysicsAttention(LN1(x))
    out = y + GatedFeedForward(LN2(y))

in float32: both norms (with the residual sum of the second), the layer and the feed-forward
run and differentiate in the library, the gradients are clipped by their global norm there
too (the paper's recipe clips at 1), and torch's AdamW makes the step.  The loss is the
relative L2 error against a smooth field of the coordinates.

    python examples/train_gated_block.py --points 20000 --steps 50
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2602_04940_amd import (GatedFeedForward, GatedWeights, GradClip, LayerWeights,  # noqa: E402
                                  PhysicsAttention, ResidualNorm)

LAYER = ("W2", "b2", "W1", "b1", "Wq", "Wk", "Wv", "W3", "b3")
GATED = ("Wg", "bg", "Wu", "bu", "Wd", "bd")


class GatedBlock:
    """The block's parameters (device float32 tensors in self.p) and its two passes."""

    def __init__(self, C, H, M, F, max_points, seed=0, activation="silu", group_span=4096, device="cuda"):
        gen = torch.Generator().manual_seed(seed)
        dh = C // H

        def xavier(*shape):
            return (torch.rand(shape, generator=gen) * 2 - 1) * math.sqrt(6.0 / (shape[-2] + shape[-1]))
        p = dict(W2=xavier(C, H * M), b2=torch.zeros(H * M), W1=xavier(C, C), b1=torch.zeros(C), Wq=xavier(H, dh, dh),
                 Wk=xavier(H, dh, dh), Wv=xavier(H, dh, dh), W3=xavier(C, C), b3=torch.zeros(C), g1=torch.ones(C),
                 n1=torch.zeros(C), g2=torch.ones(C), n2=torch.zeros(C), Wg=xavier(C, F), bg=torch.zeros(F),
                 Wu=xavier(C, F), bu=torch.zeros(F), Wd=xavier(F, C), bd=torch.zeros(C))
        self.p = {k: v.to(device) for k, v in p.items()}
        self.tile = group_span * max(1, 1_000_000 // group_span)
        self.attention = PhysicsAttention(C, H, M, dtype="fp32", group_span=group_span, max_points=max_points)
        self.norm1, self.norm2 = ResidualNorm(C, "fp32"), ResidualNorm(C, "fp32")
        self.ff = GatedFeedForward(C, F, activation=activation, dtype="fp32")

    def close(self):
        for part in (self.attention, self.norm1, self.norm2, self.ff):
            part.close()

    def forward(self, x):
        """out, keeping what the backward pass reads."""
        p = self.p
        self.layer_weights = LayerWeights({k: p[k] for k in LAYER})
        self.ff.load(GatedWeights({k: p[k] for k in GATED}, "fp32"))
        _, h1 = self.norm1.forward(x, p["g1"], p["n1"])
        a = self.attention.forward(self.layer_weights, h1, tile=self.tile)
        y, h2 = self.norm2.forward(a, p["g2"], p["n2"], residual=x)
        self.kept = (x, h1, y, h2)
        return y + self.ff.forward(h2)

    def backward(self, g):
        """dx and the gradient of every parameter for the output gradient g."""
        p, (x, h1, y, h2) = self.p, self.kept
        dh2, ff = self.ff.backward(h2, g)
        dy, dg2, dn2 = self.norm2.backward(y, dh2, p["g2"], residual_grad=g)
        dh1, layer = self.attention.backward(self.layer_weights, h1, dy, tile=self.tile)
        dx, dg1, dn1 = self.norm1.backward(x, dh1, p["g1"], residual_grad=dy)
        grads = {k[1:]: v for k, v in {**ff, **layer}.items()}
        grads.update(g1=dg1, n1=dn1, g2=dg2, n2=dn2)
        return dx, grads


def relative_l2(out, target):
    """The loss and its gradient."""
    d, size = out - target, target.norm()
    err = d.norm()
    return err / size, d / (err * size)


def surface(points, C, seed=0):
    """Features [points, C] of an ellipsoid surface and a smooth field on it [points, C]."""
    from dataclasses import replace
    from ts3_synth import WORKLOADS
    from ts3_synth.workloads import small_features
    x = small_features(replace(WORKLOADS["ellipsoid_4k_fp32"], C=C), points)
    rng = np.random.default_rng(seed)
    field = np.tanh(x @ (rng.standard_normal((C, 8)) / math.sqrt(C))) @ rng.standard_normal((8, C))
    return x.astype(np.float32), field.astype(np.float32)


def train(points=20_000, steps=50, C=64, H=4, M=32, F=171, lr=1e-2, seed=0):
    """Trains a block; returns the losses and the gradient norms before clipping."""
    x, field = (torch.from_numpy(a).cuda() for a in surface(points, C, seed))
    block, clip = GatedBlock(C, H, M, F, points, seed), GradClip()
    names = sorted(block.p)
    optimizer = torch.optim.AdamW([block.p[k] for k in names], lr=lr, weight_decay=0.05)
    losses, norms = [], []
    for _ in range(steps):
        loss, g = relative_l2(block.forward(x), field)
        _, grads = block.backward(g)
        norms.append(clip([grads[k] for k in names], 1.0))
        for k in names:
            block.p[k].grad = grads[k]
        optimizer.step()
        losses.append(loss)
    block.close()
    clip.close()
    return [float(v) for v in losses], [float(v) for v in norms]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--points", type=int, default=20_000)
    ap.add_argument("--steps", type=int, default=50)
    args = ap.parse_args()
    losses, norms = train(args.points, args.steps)
    for i in range(0, len(losses), max(1, len(losses) // 10)):
        print(f"step {i:4d}  relative L2 {losses[i]:.4f}  gradient norm {norms[i]:.3f}")
    print(f"step {len(losses) - 1:4d}  relative L2 {losses[-1]:.4f}")
