#!/usr/bin/env python
"""Data-parallel training of a small language model with compressed gradients, on one GPU with simulated nodes.

Per node and step: a gated feed-forward block between an embedding and a vocabulary matrix, whose activations are kept in 8 bits between the
forward and the backward pass (swiglu_forward, pack_activation), the loss of the last layer without its logits
(linear_cross_entropy_grad), and weight gradients written straight into the compressor's stacks (weight_gradient, d_weight).  Then PowerSGD+
compresses the stacks of all nodes, and momentum SGD applies the reconstruction (msgd_update) to float32 weights, of which the
model uses a bfloat16 copy.

The task is synthetic: the next token is a fixed function of the current one, so the loss falls from log(vocabulary) towards zero.

  python examples/compressed_training.py [--steps 60] [--nodes 2] [--vocab 2000] [--width 256] [--inner 512] [--tokens 1024] [--rank 8]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2509_11254_b200 as psgd


def rms_norm(x):
    """x / rms(x) per row, and the factor for the backward pass."""
    f = torch.rsqrt(x.float().square().mean(1, keepdim=True) + 1e-6)
    return (x.float() * f).to(torch.bfloat16), f


def rms_norm_backward(d, x, f):
    y = x.float() * f
    return f * (d.float() - y * (d.float() * y).mean(1, keepdim=True))


class Model:
    """embedding -> x + down(silu(gate(n(x))) * up(n(x))) -> n -> vocabulary; the embedding is not trained."""

    def __init__(self, vocab, width, inner, nodes, rank, seed=0, device="cuda"):
        g = torch.Generator(device=device)
        g.manual_seed(seed)

        def normal(*shape, scale):
            return torch.randn(shape, generator=g, device=device) * scale

        self.vocab, self.width, self.inner, self.nodes = vocab, width, inner, nodes
        self.embedding = normal(vocab, width, scale=1.0).to(torch.bfloat16)
        # float32 weights and momentum, stacked as the compressor stacks matrices of one shape: [gate, up], [down], [vocabulary]
        self.X = {"gate_up": normal(2, inner, width, scale=width ** -0.5), "down": normal(1, width, inner, scale=0.5 * inner ** -0.5), "head": normal(1, vocab, width, scale=0.02)}
        self.mom = {k: torch.zeros_like(v) for k, v in self.X.items()}
        opt = dict(r=rank, N=nodes, refresh_period=20, seed=seed, device=device)
        self.compress = {"gate_up": psgd.PowerSGDPlus(inner, width, count=2, grad_dtype="bfloat16", **opt),
                         "down": psgd.PowerSGDPlus(inner, width, transposed=True, **opt),       # stored width x inner: the transpose of a tall matrix
                         "head": psgd.PowerSGDPlus(vocab, width, grad_dtype="bfloat16", **opt)}
        self.G = {"gate_up": torch.empty((2, nodes, inner, width), dtype=torch.bfloat16, device=device),
                  "down": torch.empty((1, nodes, width, inner), device=device),
                  "head": torch.empty((1, nodes, vocab, width), dtype=torch.bfloat16, device=device)}

    def node_step(self, node, tokens, targets):
        """One node's forward and backward pass; its weight gradients go to slot `node` of the stacks.  Returns its loss (on the device)."""
        W = {k: v.to(torch.bfloat16) for k, v in self.X.items()}
        x = self.embedding[tokens]
        n1, f1 = rms_norm(x)
        kept_in = psgd.pack_activation(n1)                                                # for two weight gradients, 8 bits
        h, kept_gate, kept_up = psgd.swiglu_forward(n1 @ W["gate_up"][0].T, n1 @ W["gate_up"][1].T)
        y = x + h @ W["down"][0].T
        n2, f2 = rms_norm(y)
        del n1, h
        out = psgd.linear_cross_entropy_grad(n2, W["head"][0], targets, d_weight=self.G["head"][0, node])
        dy = rms_norm_backward(out.d_hidden, y, f2).to(torch.bfloat16)
        dh = dy @ W["down"][0]
        d_gate, d_up, h_again = psgd.swiglu_backward(dh, kept_gate, kept_up, recompute=True)
        psgd.weight_gradient(dy, psgd.pack_activation(h_again), out=self.G["down"][0, node])
        psgd.weight_gradient(d_gate, kept_in, out=self.G["gate_up"][0, node])
        psgd.weight_gradient(d_up, kept_in, out=self.G["gate_up"][1, node])
        return out.loss

    def step(self, tokens, targets, eta, mu=0.9):
        """tokens, targets [nodes, T] int64.  Returns the mean loss over the nodes (on the device)."""
        loss = torch.stack([self.node_step(i, tokens[i], targets[i]) for i in range(self.nodes)]).mean()
        for k, c in self.compress.items():
            c.step(self.G[k])
            c.msgd_update(self.X[k], self.mom[k], eta, mu)
        return loss


def train(steps=60, nodes=2, vocab=2000, width=256, inner=512, tokens=1024, rank=8, eta=0.5, seed=0, log=print):
    model = Model(vocab, width, inner, nodes, rank, seed)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 1)
    follow = torch.randperm(vocab, generator=g, device="cuda")
    losses = []
    for t in range(steps):
        x = torch.randint(vocab, (nodes, tokens), generator=g, device="cuda")
        losses.append(float(model.step(x, follow[x], eta)))
        if log and (t % 10 == 0 or t == steps - 1):
            log(f"step {t:4d}  loss {losses[-1]:.4f}  (log vocabulary {math.log(vocab):.4f})")
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    for name, default in (("steps", 60), ("nodes", 2), ("vocab", 2000), ("width", 256), ("inner", 512), ("tokens", 1024), ("rank", 8)):
        ap.add_argument("--" + name, type=int, default=default)
    ap.add_argument("--eta", type=float, default=0.5)
    a = ap.parse_args()
    train(**vars(a))
