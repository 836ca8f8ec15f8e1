#!/usr/bin/env python
"""A small decoder layer trained from a teacher's top logits, with compressed gradients, on one GPU with simulated nodes.

Per node and step: norm, queries / keys / values with rotary positions, causal attention (plain torch), residual, norm, gated unit, residual, norm, and the last
layer's distance from the teacher without its logits.  The norms add the residual and keep their result in 8 bits for the weight gradients
(layer_norm_forward), the gradients come back through layer_norm_backward, rotary_backward, swiglu_backward, linear_distillation_grad and weight_gradient, the
latter two straight into the compressor's stacks; PowerSGD+ compresses those of all nodes and momentum SGD applies the reconstruction.

The teacher is synthetic: for every token it lists a few next tokens with fixed logits.

  python examples/distillation.py [--steps 40] [--nodes 2] [--vocab 1000] [--width 128] [--heads 4] [--inner 256] [--length 64] [--batch 8] [--rank 8]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2509_11254_b200 as psgd


def attention(q, k, v):
    """Causal softmax attention of [B, heads, S, D], float32; returns (result, probabilities)."""
    s = q @ k.transpose(2, 3) / math.sqrt(q.shape[3])
    s = s.masked_fill(torch.ones_like(s[0, 0], dtype=torch.bool).triu(1), -math.inf)
    p = torch.softmax(s, 3)
    return p @ v, p


def attention_backward(d, p, q, k, v):
    ds = p * (d @ v.transpose(2, 3) - (d * (p @ v)).sum(3, keepdim=True)) / math.sqrt(q.shape[3])
    return ds @ k, ds.transpose(2, 3) @ q, p.transpose(2, 3) @ d


class Student:
    """embedding -> x + o(attention(n1(x))) -> x + down(silu(gate(n2(x))) up(n2(x))) -> n3 -> vocabulary; the embedding is not trained."""

    def __init__(self, vocab, width, heads, inner, nodes, rank, seed=0, device="cuda"):
        g = torch.Generator(device=device)
        g.manual_seed(seed)

        def normal(*shape, scale):
            return torch.randn(shape, generator=g, device=device) * scale

        self.heads, self.nodes, self.width = heads, nodes, width
        self.embedding = normal(vocab, width, scale=1.0).to(torch.bfloat16)
        # float32 weights and momentum, stacked as the compressor stacks matrices of one shape: queries, keys and values over each other; gate and up
        self.X = {"qkv": normal(1, 3 * width, width, scale=width ** -0.5), "o": normal(1, width, width, scale=0.5 * width ** -0.5),
                  "gate_up": normal(2, inner, width, scale=width ** -0.5), "down": normal(1, width, inner, scale=0.5 * inner ** -0.5), "head": normal(1, vocab, width, scale=0.02)}
        self.norms = torch.ones(3, width, device=device)
        self.mom = {k: torch.zeros_like(v) for k, v in self.X.items()}
        opt = dict(r=rank, N=nodes, refresh_period=20, seed=seed, device=device)
        self.compress = {"qkv": psgd.PowerSGDPlus(3 * width, width, **opt), "o": psgd.PowerSGDPlus(width, width, **opt), "gate_up": psgd.PowerSGDPlus(inner, width, count=2, **opt),
                         "down": psgd.PowerSGDPlus(inner, width, transposed=True, **opt), "head": psgd.PowerSGDPlus(vocab, width, grad_dtype="bfloat16", **opt)}
        self.G = {k: torch.empty((v.shape[0], nodes, *v.shape[1:]), dtype=torch.bfloat16 if k == "head" else torch.float32, device=device) for k, v in self.X.items()}
        self.d_norms = torch.empty((nodes, 3, width), device=device)
        self.frequencies = psgd.rotary_frequencies(width // heads, device=device)

    def node_step(self, node, tokens, teacher_logits, teacher_index, temperature):
        """One node's forward and backward pass; its weight gradients go to slot `node` of the stacks.  tokens [B, S].  Returns its loss (on the device)."""
        B, S = tokens.shape
        T, H, D = B * S, self.heads, self.width // self.heads
        W = {k: v.to(torch.bfloat16) for k, v in self.X.items()}
        positions = torch.arange(S, device=tokens.device).repeat(B)
        x = self.embedding[tokens.reshape(-1)]

        def split(t):                               # [T, H, D] -> [B, H, S, D]
            return t.reshape(B, S, H, D).transpose(1, 2).float()

        def join(t):                                # and back
            return t.transpose(1, 2).reshape(T, H, D).to(torch.bfloat16)

        n1 = psgd.layer_norm_forward(x, self.norms[0], center=False, keep=True)
        qkv = (n1.y @ W["qkv"][0].T).view(T, 3, H, D)
        q, k = psgd.rotary_forward(qkv[:, 0], qkv[:, 1], positions, self.frequencies)
        q, k, v = split(q), split(k), split(qkv[:, 2])
        o, p = attention(q, k, v)
        o = join(o).view(T, -1)
        kept_o = psgd.pack_activation(o)
        n2 = psgd.layer_norm_forward(o @ W["o"][0].T, self.norms[1], residual=x, center=False, keep=True)
        h, kept_gate, kept_up = psgd.swiglu_forward(n2.y @ W["gate_up"][0].T, n2.y @ W["gate_up"][1].T)
        n3 = psgd.layer_norm_forward(h @ W["down"][0].T, self.norms[2], residual=n2.x, center=False)

        out = psgd.linear_distillation_grad(n3.y, W["head"][0], teacher_logits, teacher_index, temperature, d_weight=self.G["head"][0, node])

        g3 = psgd.layer_norm_backward(out.d_hidden, n3.x, self.norms[2], None, n3.rstd)
        d_gate, d_up, h = psgd.swiglu_backward(g3.d_x @ W["down"][0], kept_gate, kept_up, recompute=True)
        psgd.weight_gradient(g3.d_x, psgd.pack_activation(h), out=self.G["down"][0, node])
        psgd.weight_gradient(d_gate, n2.kept, out=self.G["gate_up"][0, node])
        psgd.weight_gradient(d_up, n2.kept, out=self.G["gate_up"][1, node])
        g2 = psgd.layer_norm_backward(d_gate @ W["gate_up"][0] + d_up @ W["gate_up"][1], n2.x, self.norms[1], None, n2.rstd, d_x=g3.d_x)
        psgd.weight_gradient(g2.d_x, kept_o, out=self.G["o"][0, node])
        dq, dk, dv = attention_backward(split((g2.d_x @ W["o"][0]).view(T, H, D)), p, q, k, v)
        d_qkv = torch.empty_like(qkv)
        d_qkv[:, 0], d_qkv[:, 1], d_qkv[:, 2] = join(dq), join(dk), join(dv)
        psgd.rotary_backward(d_qkv[:, 0], d_qkv[:, 1], positions, self.frequencies, in_place=True)
        d_qkv = d_qkv.view(T, -1)
        psgd.weight_gradient(d_qkv, n1.kept, out=self.G["qkv"][0, node])
        g1 = psgd.layer_norm_backward(d_qkv @ W["qkv"][0], x, self.norms[0], None, n1.rstd, d_x=g2.d_x)
        self.d_norms[node] = torch.stack([g1.d_weight, g2.d_weight, g3.d_weight])
        return out.loss

    def step(self, tokens, teacher_logits, teacher_index, eta, mu=0.9, temperature=2.0):
        """tokens [nodes, B, S], the teacher's [nodes, B * S, K].  Returns the mean loss over the nodes (on the device)."""
        loss = torch.stack([self.node_step(i, tokens[i], teacher_logits[i], teacher_index[i], temperature) for i in range(self.nodes)]).mean()
        for k, c in self.compress.items():
            c.step(self.G[k])
            c.msgd_update(self.X[k], self.mom[k], eta, mu)
        self.norms -= eta * self.d_norms.mean(0)
        return loss


class Teacher:
    """Lists `top` next tokens for every token, with logits of its own."""

    def __init__(self, vocab, top=8, seed=1, device="cuda"):
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.index = torch.stack([(torch.randperm(vocab, generator=g, device=device)) for _ in range(top)], 1)
        self.logits = torch.sort(2 * torch.randn(vocab, top, generator=g, device=device), dim=1, descending=True).values

    def __call__(self, tokens):
        return self.logits[tokens], self.index[tokens]


def train(steps=40, nodes=2, vocab=1000, width=128, heads=4, inner=256, length=64, batch=8, rank=8, eta=0.2, seed=0, log=print):
    student, teacher = Student(vocab, width, heads, inner, nodes, rank, seed), Teacher(vocab)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 1)
    losses = []
    for t in range(steps):
        tokens = torch.randint(vocab, (nodes, batch, length), generator=g, device="cuda")
        losses.append(float(student.step(tokens, *teacher(tokens.view(nodes, -1)), eta)))
        if log and (t % 10 == 0 or t == steps - 1):
            log(f"step {t:4d}  distance from the teacher {losses[-1]:.4f}")
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    for name, default in (("steps", 40), ("nodes", 2), ("vocab", 1000), ("width", 128), ("heads", 4), ("inner", 256), ("length", 64), ("batch", 8), ("rank", 8)):
        ap.add_argument("--" + name, type=int, default=default)
    ap.add_argument("--eta", type=float, default=0.2)
    train(**vars(ap.parse_args()))
