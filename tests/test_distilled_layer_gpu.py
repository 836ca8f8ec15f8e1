"""The operators together, as they are used: the example's decoder layer, trained from a teacher's top logits."""
import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t

    if not t.cuda.is_available():
        pytest.skip("no CUDA device")
    return t


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "distillation.py")
    spec = importlib.util.spec_from_file_location("distillation_example", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def reference(torch, s, tokens, z, index, tau):
    """The same function of the same bfloat16 weights in float64 with autograd: (loss, {name: gradient})."""
    W = {k: v.to(torch.bfloat16).double().requires_grad_() for k, v in s.X.items()}
    norms = s.norms.double().requires_grad_()
    B, S = tokens.shape
    H, D = s.heads, s.width // s.heads

    def norm(x, i):
        return x / torch.sqrt(x.square().mean(1, keepdim=True) + 1e-5) * norms[i]

    def turn(x):                                    # [B, S, H, D]
        angle = torch.arange(S, device=x.device).double()[:, None] * s.frequencies
        c, n = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
        u, v = x[..., :D // 2], x[..., D // 2:]
        return torch.cat([u * c - v * n, u * n + v * c], 3)

    x = s.embedding[tokens.reshape(-1)].double()
    q, k, v = (norm(x, 0) @ W["qkv"][0].T).view(B, S, 3, H, D).unbind(2)
    q, k, v = (t.transpose(1, 2) for t in (turn(q), turn(k), v))
    a = (q @ k.transpose(2, 3) / math.sqrt(D)).masked_fill(torch.ones(S, S, dtype=torch.bool, device=x.device).triu(1), -math.inf)
    x = x + (torch.softmax(a, 3) @ v).transpose(1, 2).reshape(B * S, -1) @ W["o"][0].T
    n = norm(x, 1)
    x = x + (torch.nn.functional.silu(n @ W["gate_up"][0].T) * (n @ W["gate_up"][1].T)) @ W["down"][0].T
    log_p = torch.log_softmax(norm(x, 2) @ W["head"][0].T / tau, 1).gather(1, index)
    log_q = torch.log_softmax(z.double() / tau, 1)
    loss = (tau ** 2 * (log_q.exp() * (log_q - log_p)).sum(1)).mean()
    loss.backward()
    return loss.detach(), {**{k: v.grad for k, v in W.items()}, "norms": norms.grad}


def test_layer_gradients(torch, example):
    """Every gradient of the layer against float64.  In Frobenius norm: values are rounded to bfloat16 about a dozen times on the way to the furthest weight (2^-9 rms at most each,
    12 of them 7e-3 if they are independent, and amplified at most a few times by the softmax), and an 8-bit activation is off by at most 1/63 of its group's largest
    value in uniform steps, 1/220 of it rms, 2 % of values a quarter as large as it: 5 % bounds them together."""
    s = example.Student(vocab=500, width=96, heads=3, inner=200, nodes=1, rank=4)
    s.norms += 0.2 * torch.randn(s.norms.shape, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    s.X["head"] *= 10
    tokens = torch.randint(500, (5, 37), generator=torch.Generator(device="cuda").manual_seed(4), device="cuda")
    z, index = example.Teacher(500)(tokens.view(-1))
    loss = s.node_step(0, tokens, z, index, 2.0)
    want, grads = reference(torch, s, tokens, z, index, 2.0)
    assert abs(float(loss) - float(want)) <= 2e-2 * float(want)
    got = {**{k: g[:, 0] for k, g in s.G.items()}, "norms": s.d_norms[0]}
    for k, g in grads.items():
        off = float((got[k].double() - g).norm() / g.norm())
        assert off < 0.05, (k, off)


def test_example_runs(torch, example):
    losses = example.train(steps=4, vocab=300, width=64, heads=2, inner=120, length=33, batch=3, log=None)
    assert len(losses) == 4 and all(math.isfinite(v) and v > 0 for v in losses)


def test_distillation_right_behind_the_kernel_that_writes_its_input(torch, example):
    """The product's loads begin before the kernel in front of it ends: a norm writes the hidden states into memory that held others just before, a hundred times, few tokens
    and many, the same bits as with a pause between the two."""
    import paper_2509_11254_b200 as ops

    g = torch.Generator(device="cuda").manual_seed(7)
    for T, V, D, K in ((1, 3000, 256, 4), (90, 2000, 768, 20), (2100, 900, 512, 7)):
        w = (torch.randn(V, D, generator=g, device="cuda") * 0.1).bfloat16()
        xs = [torch.randn(T, D, generator=g, device="cuda").bfloat16() for _ in range(4)]
        one = torch.ones(D, device="cuda")
        z, index = torch.randn(T, K, generator=g, device="cuda"), torch.randint(V, (T, K), generator=g, device="cuda")
        want = []
        for x in xs:
            y = ops.layer_norm_forward(x, one).y
            torch.cuda.synchronize()
            want.append([*ops.linear_distillation_grad(y, w, z, index), *ops.linear_distillation(y, w, z, index, 2.0)])
            torch.cuda.synchronize()
        del y
        for i in range(100):
            y = ops.layer_norm_forward(xs[i % 4], one).y             # (the allocator hands out the memory of the last round)
            got = ops.linear_distillation_grad(y, w, z, index)
            y = ops.layer_norm_forward(xs[i % 4], one).y
            got = [*got, *ops.linear_distillation(y, w, z, index, 2.0)]
            for a, b in zip(got, want[i % 4]):
                assert torch.equal(a, b), (T, i)
            del y, got
