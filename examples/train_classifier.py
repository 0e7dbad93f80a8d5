#!/usr/bin/env python3
"""Trains a small image classifier with the library's layers and operators alone.

A step runs them as a network's training does:
  conv 3x3 -> rectifier -> max pool -> conv 3x3 -> rectifier -> average pool
  -> layer norm -> inner product -> log probabilities of the labels, the five
  likeliest classes and their entropy,
then the same in reverse (the log probabilities' gradient, the inner product's,
the layer norm's with its weight and bias, the pools' and convolutions'), and
before the update the gradients are clipped to a global norm.  Rectifiers and
the update itself are torch's.  The images are synthetic: a texture of 4 x 4
pixels for each class, repeated, and noise.

  python examples/train_classifier.py [--steps 60] [--batch 64]
"""
import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_1903_06934_amd as m  # noqa: E402

CLASSES, SIZE = 20, 16
WIDTHS = (32, 64)


def images(batch, generator):
    """(x [batch, 3, SIZE, SIZE], labels [batch]): textures of the classes in noise."""
    textures = torch.randn(CLASSES, 3, 4, 4, generator=torch.Generator().manual_seed(5))
    labels = torch.randint(CLASSES, (batch,), generator=generator)
    x = textures.repeat(1, 1, SIZE // 4, SIZE // 4)[labels]
    x = x + 0.5 * torch.randn(batch, 3, SIZE, SIZE, generator=generator)
    return x.cuda(), labels.cuda()


def parameters(seed=0):
    """The network's weights, as the layers take them."""
    g = torch.Generator().manual_seed(seed)

    def filters(k, c, f):
        return torch.randn(k, c, f, f, generator=g).mul_((2.0 / (c * f * f)) ** 0.5).cuda()

    a, b = WIDTHS
    zeros = lambda n: torch.zeros(n, device="cuda")
    return {"w1": filters(a, 3, 3), "b1": zeros(a), "w2": filters(b, a, 3), "b2": zeros(b),
            "scale": torch.ones(b, device="cuda"), "shift": zeros(b),
            "w3": filters(CLASSES, b, 1), "b3": zeros(CLASSES)}


def step(p, x, labels, max_norm):
    """(LogProbs of the labels, gradients clipped to max_norm, their norm before)."""
    n = x.shape[0]
    a1 = torch.relu_(m.conv_fwd(x, p["w1"], p["b1"], pad=1))
    p1, mask = m.pool_fwd(a1, (2, 2), 2)
    a2 = torch.relu_(m.conv_fwd(p1, p["w2"], p["b2"], pad=1))
    side = a2.shape[2]
    p2, _ = m.pool_fwd(a2, (side, side), 1, mode="avg")
    rows = p2.view(n, -1)
    normed, mean, rstd = m.layernorm_fwd(rows, p["scale"], p["shift"])
    logits = m.conv_fwd(normed.view(n, -1, 1, 1), p["w3"], p["b3"])
    out = m.logprob_fwd(logits.view(n, -1), labels, top=5)

    g = {}
    # The loss is the mean of -logp.
    dlogp = torch.full((n,), -1.0 / n, device="cuda")
    dlogits = m.logprob_bwd(logits.view(n, -1), out.stats, labels, dlogp)
    d = dlogits.view(n, -1, 1, 1)
    g["w3"], g["b3"] = m.conv_bwd_weight(normed.view(n, -1, 1, 1), d, (1, 1))
    dnormed = m.conv_bwd_data(d, p["w3"], (1, 1))
    drows, g["scale"], g["shift"] = m.layernorm_bwd(dnormed.view(n, -1), rows, mean, rstd,
                                                    p["scale"])
    d2 = m.pool_bwd(drows.view_as(p2), (side, side), (side, side), 1, mode="avg")
    d2 *= a2 > 0
    g["w2"], g["b2"] = m.conv_bwd_weight(p1, d2, (3, 3), pad=1)
    d1 = m.pool_bwd(m.conv_bwd_data(d2, p["w2"], tuple(p1.shape[2:]), pad=1),
                    tuple(a1.shape[2:]), (2, 2), 2, mask=mask)
    d1 *= a1 > 0
    g["w1"], g["b1"] = m.conv_bwd_weight(x, d1, (3, 3), pad=1)
    norm = m.grad_clip([g[k] for k in p], max_norm)
    return out, g, norm


def train(steps, batch, rate=0.1, momentum=0.9, max_norm=1.0, report=None):
    """The mean loss of each step; report(i, loss, LogProbs, labels, norm) after each."""
    gen = torch.Generator().manual_seed(1)
    p = parameters()
    speed = {k: torch.zeros_like(v) for k, v in p.items()}
    losses = []
    for i in range(steps):
        x, labels = images(batch, gen)
        out, g, norm = step(p, x, labels, max_norm)
        for k in p:
            p[k].sub_(speed[k].mul_(momentum).add_(g[k]), alpha=rate)
        losses.append(float(-out.logp.mean()))
        if report:
            report(i, losses[-1], out, labels, norm)
    return losses


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--batch", type=int, default=64)
    args = ap.parse_args()

    def report(i, loss, out, labels, norm):
        if i % 10 == 0 or i == args.steps - 1:
            hit = out.top_index == labels[:, None]
            print(f"step {i:4d}  loss {loss:.4f}  top-1 {hit[:, 0].float().mean():.2f}  "
                  f"top-5 {hit.any(1).float().mean():.2f}  entropy {out.entropy.mean():.3f}  "
                  f"gradient norm {float(norm):.3f}", flush=True)

    train(args.steps, args.batch, report=report)


if __name__ == "__main__":
    main()
