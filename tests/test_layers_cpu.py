"""Host-only checks of layer norm and rotary positions: workspaces, refusals, frequencies, without touching a GPU."""
import ctypes as C
import math

import pytest


@pytest.fixture(scope="module")
def L():
    from paper_2509_11254_b200 import binding, build

    build.build_library()
    return binding.lib()


P = 1 << 20          # stands for device addresses; nothing below gets as far as using one
FAR = 1 << 30


def norm_forward(L, x=P, ldx=64, xt=1, r=None, ldr=0, w=P, b=None, wt=0, eps=1e-5, center=1, T=8, F=64, s=None, lds=0, y=FAR, ldy=64, yt=1, mean=P, rstd=P, q=None, scales=None):
    return L.psgd_norm_forward(x, ldx, xt, r, ldr, w, b, wt, eps, center, T, F, s, lds, y, ldy, yt, mean, rstd, q, scales, None)


def norm_backward(L, dy=P, lddy=64, dyt=1, x=P, ldx=64, xt=1, w=P, wt=0, mean=P, rstd=P, add=None, lda=0, T=8, F=64, dx=FAR, lddx=64, dw=P, db=None, ws=P, nb=0):
    return L.psgd_norm_backward(dy, lddy, dyt, x, ldx, xt, w, wt, mean, rstd, add, lda, T, F, dx, lddx, dw, db, ws, nb, None)


def rotary(L, q=P, qt=256, qh=64, H=4, oq=FAR, oqt=256, oqh=64, k=None, kt=0, kh=0, K=0, okk=None, okt=0, okh=0, pos=P, f=P, T=8, D=64, R=64, layout=0, dtype=1):
    return L.psgd_rotary(q, qt, qh, H, oq, oqt, oqh, k, kt, kh, K, okk, okt, okh, pos, f, T, D, R, layout, 0, 1.0, dtype, None)


def test_norm_refuses_before_any_launch(L):
    f = lambda **kw: norm_forward(L, **kw)
    assert f(T=-1) == -1 and f(F=0) == -1 and f(T=1 << 31) == -1 and f(F=1 << 31) == -1 and f(ldx=63) == -1 and f(ldy=63) == -1
    assert f(xt=7) == -1 and f(yt=0) == -1 and f(wt=2) == -1 and f(eps=-1.0) == -1 and f(eps=float("nan")) == -1
    assert f(x=None) == -2 and f(w=None) == -2 and f(y=None) == -2 and f(rstd=None) == -2 and f(mean=None) == -2 and f(r=2 * FAR, ldr=64) == -2 and f(q=P, scales=None) == -2
    assert f(r=2 * FAR, ldr=63, s=3 * FAR, lds=64) == -1 and f(r=2 * FAR, ldr=64, s=3 * FAR, lds=63) == -1 and f(q=P + 8, scales=P) == -1
    assert f(y=P) == -1 and f(y=P + 1022) == -1 and f(r=FAR, ldr=64, s=3 * FAR, lds=64) == -1 and f(r=2 * FAR, ldr=64, s=P, lds=64) == -1 and f(r=2 * FAR, ldr=64, s=FAR, lds=64) == -1
    assert f(T=0, x=None, y=None) == 0
    g = lambda **kw: norm_backward(L, **kw)
    assert g(T=-1) == -1 and g(F=0) == -1 and g(dyt=0) == -1 and g(xt=3) == -1 and g(wt=-1) == -1 and g(lddy=63) == -1 and g(ldx=63) == -1 and g(lddx=63) == -1 and g(add=2 * FAR, lda=63) == -1
    assert g(dy=None) == -2 and g(x=None) == -2 and g(w=None) == -2 and g(rstd=None) == -2 and g(dx=None) == -2 and g(dw=None) == -2 and g(ws=None) == -2 and g(ws=P + 16) == -1
    assert g(dx=P) == -1 and g(add=FAR, lda=64) == -1 and g() == -3 and g(mean=None) == -3


def test_norm_workspace(L):
    n = C.c_size_t()
    for T, F in ((1, 1), (4096, 768), (16384, 2048), (1 << 20, 8192), (100000, 30000)):
        assert L.psgd_norm_workspace(T, F, C.byref(n)) == 0
        # two sums per column of every CTA, at most eight CTAs per multiprocessor; two floats per row where rows are wide
        assert 8 * F <= n.value <= 8 * 148 * 8 * F + 8 * T + 4096
    assert L.psgd_norm_workspace(0, 5, C.byref(n)) == 0 and n.value > 0
    assert L.psgd_norm_workspace(-1, 5, C.byref(n)) == -1 and L.psgd_norm_workspace(5, 0, C.byref(n)) == -1 and L.psgd_norm_workspace(5, 5, None) == -2


def test_rotary_refuses_before_any_launch(L):
    f = lambda **kw: rotary(L, **kw)
    assert f(T=-1) == -1 and f(H=-1) == -1 and f(K=-1) == -1 and f(D=0) == -1 and f(H=1 << 17) == -1 and f(H=1 << 16, D=1 << 16, R=64) == -1
    assert f(R=0) == -1 and f(R=63) == -1 and f(R=66) == -1 and f(D=8192, R=4098) == -1 and f(layout=2) == -1 and f(dtype=2) == -1 and f(qt=-1) == -1 and f(okh=-1) == -1
    assert f(q=None) == -2 and f(oq=None) == -2 and f(pos=None) == -2 and f(f=None) == -2 and f(K=1) == -2
    assert f(T=0, q=None) == 0 and f(H=0, q=None) == 0
    # an output's values one on another, over an input other than its own, over its own with other strides, over the other output
    assert f(oqh=63) == -1 and f(oqt=255) == -1 and f(oqh=0) == -1 and f(oq=P + 64) == -1 and f(oq=P, oqt=512) == -1 and f(oq=P, oqt=64, oqh=512) == -1
    k = dict(k=2 * FAR, kt=256, kh=64, K=4, okk=3 * FAR, okt=256, okh=64)
    assert f(**{**k, "okk": P}) == -1 and f(**{**k, "okk": FAR}) == -1 and f(**{**k, "k": FAR}) == -1 and f(**{**k, "okk": FAR + 2 * 64}) == -1


def test_python_refuses_host_tensors():
    import torch

    import paper_2509_11254_b200 as p

    x, w, at = torch.zeros(4, 8), torch.ones(8), torch.arange(4)
    f = p.rotary_frequencies(8, device="cpu")
    for call in (lambda: p.layer_norm_forward(x, w), lambda: p.layer_norm_backward(x, x, w, None, at), lambda: p.rotary_forward(x.view(4, 1, 8), None, at, f),
                 lambda: p.rotary_backward(x.view(4, 1, 8), None, at, f)):
        with pytest.raises(p.PSGDError):
            call()


def test_frequencies():
    """By the number of turns over the length of the training: fast pairs stay, slow ones are divided by the factor, a straight line between."""
    import torch

    import paper_2509_11254_b200 as p

    f = p.rotary_frequencies(64, device="cpu")
    assert f.dtype == torch.float64 and f.shape == (32,)
    want = torch.exp(-math.log(10000.0) * torch.arange(32, dtype=torch.float64) / 32)
    assert torch.allclose(f, want, rtol=1e-14)
    assert torch.allclose(p.rotary_frequencies(64, factor=8.0, device="cpu"), want / 8, rtol=1e-14)
    g = p.rotary_frequencies(64, factor=8.0, original_length=4096, low=2.0, high=20.0, device="cpu")
    turns = 4096 * want / (2 * math.pi)
    assert torch.allclose(g[turns >= 20], want[turns >= 20], rtol=1e-14) and torch.allclose(g[turns <= 2], want[turns <= 2] / 8, rtol=1e-14)
    mid = (turns > 2) & (turns < 20)
    assert int(mid.sum()) >= 3
    share = (g[mid] / want[mid] - 1 / 8) / (1 - 1 / 8)
    assert torch.allclose(share, (turns[mid] - 2) / 18, rtol=1e-12) and bool((g[1:] < g[:-1]).all())
    for bad in (dict(rotated=0), dict(rotated=7), dict(rotated=8, base=0.0), dict(rotated=8, factor=0.0), dict(rotated=8, factor=float("inf")), dict(rotated=8, original_length=0),
                dict(rotated=8, original_length=10, low=4.0, high=4.0)):
        with pytest.raises(p.PSGDError):
            p.rotary_frequencies(device="cpu", **bad)


# ---- distillation -------------------------------------------------------------------------------------------------
def test_distillation_refuses_before_any_launch(L):
    n = C.c_size_t()
    for bad in ((-1, 10, 10, 4), (10, 0, 10, 4), (10, 10, 0, 4), (10, 10, 10, 0), (10, 10, 10, 1025), (1 << 31, 10, 10, 4)):
        assert L.psgd_distill_workspace(*bad, 1, C.byref(n)) == -1
    assert L.psgd_distill_workspace(8, 8, 8, 4, 1, None) == -2

    def f(H=P, ldh=64, W=P, ldw=64, z=P, ldl=4, dt=0, i=P, ldi=4, K=4, tau=1.0, T=8, V=16, D=64, loss=P, ws=P, nb=0):
        a = L.psgd_distill_loss(H, ldh, W, ldw, z, ldl, dt, i, ldi, K, tau, None, T, V, D, loss, P, P, None, ws, nb, None)
        b = L.psgd_distill_grad(H, ldh, W, ldw, z, ldl, dt, i, ldi, K, tau, None, T, V, D, loss, P, P, 2 * FAR, D, 3 * FAR, D, None, ws, nb, None)
        assert a == b
        return a

    assert f() == -3 and f(H=None) == -2 and f(W=None) == -2 and f(z=None) == -2 and f(i=None) == -2 and f(loss=None) == -2 and f(ws=None) == -2
    assert f(H=P + 8) == -1 and f(ldh=63) == -1 and f(ldl=3) == -1 and f(ldi=3) == -1 and f(dt=5) == -1 and f(K=0) == -1 and f(K=1025, ldl=2000, ldi=2000) == -1
    assert f(tau=0.0) == -1 and f(tau=float("nan")) == -1 and f(tau=float("inf")) == -1 and f(tau=-1.0) == -1 and f(T=-1) == -1 and f(V=0) == -1 and f(D=0) == -1


def test_distillation_workspace(L):
    """Beyond the cross entropy's: 8 bytes per token, and for the tokens of a piece 16 bytes per entry, 4 per token and 4 per 32 tokens and 32 columns; a piece has at most 2^29 logits
    (with gradients) or 2^32 (loss alone), or 1024 tokens."""
    a, b = C.c_size_t(), C.c_size_t()
    for T, V, D, K, grad in ((1, 32000, 768, 8, 0), (777, 50257, 768, 50, 0), (4096, 32000, 768, 64, 1), (1 << 20, 131072, 1024, 32, 1), (1 << 22, 131072, 1024, 64, 0), (1 << 20, 1000, 64, 1024, 1)):
        assert L.psgd_distill_workspace(T, V, D, K, grad, C.byref(a)) == 0 and L.psgd_xent_workspace(T, V, D, grad, C.byref(b)) == 0
        piece = min(T, max(1024, (1 << (29 if grad else 32)) // V) + 256)
        blocks = (piece + 31) // 32
        assert b.value <= a.value <= b.value + 8 * T + piece * (12 * K + 4) + blocks * (128 * K + 4 * (V // 32 + 2)) + 4096
