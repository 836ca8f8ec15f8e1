"""The training operators (cross entropy of the last layer, 8-bit activations, gated unit) against their definitions in 64 bits.

Tolerances.  Every bound below is elementwise and follows from how the result is formed:
  * a sum of products on the tensor cores, K terms: 16 products enter one float32 addition, which may truncate, so
    |error| <= (K / 16 + 8) * 2^-23 * sum |a| |b|;
  * a value rounded to bfloat16 (8 significant bits): 2^-8 of its size; the gradient of a logit is rounded once that way and carries the rounding of the
    stored exponents, ln(2) / 2048 < 3.4e-4 of p, and 2^-12 for the evaluation of p in float32;
  * exp and log of float32 arguments up to 64 in size: 2^-18 absolute in the log-sum-exp, sums of up to 2^18 terms included.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

BF16 = 2.0 ** -8          # unit roundoff: 8 significant bits, round to nearest
GROUP = 32


@pytest.fixture(scope="module")
def torch():
    import torch as t

    if not t.cuda.is_available():
        pytest.skip("no CUDA device")
    return t


@pytest.fixture(scope="module")
def ops():
    import paper_2509_11254_b200 as p

    return p


def gen(torch, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def sum_bound(K):
    return (K / 16 + 8) * 2.0 ** -23


def within(got, ref, bound):
    """Largest error over its bound."""
    d = (got.double() - ref).abs()
    assert bool((d <= bound).all()), f"worst error / bound {float((d / bound.clamp(min=1e-300)).max()):.3g}"


# ---- cross entropy ------------------------------------------------------------------------------------------------
def xent_reference(torch, h, w, labels, tw, ignore):
    """Everything in 64 bits: loss, token_loss, lse, d_hidden, d_weight and the sums the bounds are made of."""
    h, w = h.double(), w.double()
    T, V = h.shape[0], w.shape[0]
    l = h @ w.T
    lse = torch.logsumexp(l, 1) if T else torch.zeros(0, dtype=torch.float64, device=h.device)
    valid = labels != ignore
    rows = torch.nonzero(valid)[:, 0]
    cols = labels[rows]
    token = torch.zeros(T, dtype=torch.float64, device=h.device)
    token[rows] = lse[rows] - l[rows, cols]
    wt = torch.zeros(T, dtype=torch.float64, device=h.device)
    wt[rows] = 1.0 if tw is None else tw[rows].double()
    Z = float(wt.sum())
    wt = wt / Z if Z else wt * 0
    p = torch.exp(l - lse[:, None])
    d = p.clone()
    d[rows, cols] -= 1
    d = d * wt[:, None]
    mag = p.clone()
    mag[rows, cols] += 1
    mag = mag * wt.abs()[:, None]
    size = h.abs() @ w.abs().T
    return dict(loss=(wt * token).sum(), token=token, lse=lse, dh=d @ w, dw=d.T @ h, wt=wt,
                dl=d.abs(), mag=mag, size=size.amax(1) if V else size, h=h, w=w)


def check_xent(torch, ops, h, w, labels, tw=None, ignore=-100, out=None, ref=None):
    T, D = h.shape
    V = w.shape[0]
    ref = ref or xent_reference(torch, h, w, labels, tw, ignore)
    l_err = sum_bound(D) * ref["size"] + 2.0 ** -18                      # error of a logit and of the log-sum-exp, per row
    t_err = 2 * l_err + 2.0 ** -22 * ref["lse"].abs()
    kw = dict(token_weight=tw, ignore_index=ignore)
    only = ops.linear_cross_entropy(h, w, labels, **kw)
    full = ops.linear_cross_entropy_grad(h, w, labels, **kw, **(out or {}))
    for r in (only, full):
        within(r.lse, ref["lse"], l_err + 2.0 ** -22 * ref["lse"].abs())
        within(r.token_loss, ref["token"], t_err)
        assert bool((r.token_loss[labels == ignore] == 0).all())
        within(r.loss, ref["loss"], (ref["wt"].abs() * t_err).sum() + 2.0 ** -22 * ref["loss"].abs() + 1e-12)
    # gradient of a logit: one rounding to bfloat16 of w (p - [v = y]), and the relative error of p
    p_err = 3.4e-4 + 2.0 ** -12 + 2 * l_err.max() if T else 0.0
    each = BF16 * ref["dl"] + p_err * ref["mag"]
    near = (ref["dl"] + each)
    assert full.d_hidden.dtype == torch.bfloat16 and full.d_weight.dtype == torch.bfloat16
    within(full.d_hidden, ref["dh"], (each + sum_bound(V) * near) @ ref["w"].abs() * (1 + BF16) + (BF16 + 2.0 ** -22) * ref["dh"].abs() + 1e-30)
    within(full.d_weight, ref["dw"], (each + sum_bound(T) * near).T @ ref["h"].abs() * (1 + BF16) + (BF16 + 2.0 ** -22) * ref["dw"].abs() + 1e-30)
    return full


def xent_inputs(torch, T, V, D, seed, spread=1.5, ignored=0.2):
    g = gen(torch, seed)
    h = torch.randn(T, D, generator=g, device="cuda").to(torch.bfloat16)
    w = (torch.randn(V, D, generator=g, device="cuda") * (spread / math.sqrt(D))).to(torch.bfloat16)
    labels = torch.randint(V, (T,), generator=g, device="cuda")
    labels[torch.rand(T, generator=g, device="cuda") < ignored] = -100
    return h, w, labels


XENT_SHAPES = [(1, 1, 8), (1, 2, 16), (2, 33, 64), (1, 1000, 72), (63, 100, 40), (64, 128, 64), (129, 129, 200), (128, 257, 128), (257, 256, 520), (300, 4099, 136),
               (31, 50257, 768), (1, 32000, 768), (513, 2050, 264), (1030, 777, 768), (2047, 1025, 8)]


@pytest.mark.parametrize("T,V,D", XENT_SHAPES)
@pytest.mark.parametrize("weighted", [False, True])
def test_xent_matches_definition(torch, ops, T, V, D, weighted):
    h, w, labels = xent_inputs(torch, T, V, D, seed=T * 7 + V + D)
    tw = torch.rand(T, generator=gen(torch, 5), device="cuda") * 2 - 0.25 if weighted else None
    check_xent(torch, ops, h, w, labels, tw)


@pytest.mark.parametrize("T,V,D", [(5, 7, 37), (130, 300, 101), (20, 129, 1)])
def test_xent_odd_widths(torch, ops, T, V, D):
    check_xent(torch, ops, *xent_inputs(torch, T, V, D, seed=3))


def test_xent_in_pieces(torch, ops):
    """More logits than the workspace holds at a time: two pieces of tokens, the weight gradient summed over them."""
    T, V, D = 2300, 131072 - 5, 72
    h, w, labels = xent_inputs(torch, T, V, D, seed=11)
    a = check_xent(torch, ops, h, w, labels)
    b = ops.linear_cross_entropy_grad(h, w, labels)
    assert torch.equal(a.d_weight, b.d_weight) and torch.equal(a.d_hidden, b.d_hidden) and torch.equal(a.loss, b.loss)


@pytest.mark.parametrize("T,V,D,weighted", [(4500, 131072 - 5, 40, True), (5000, 131072, 36, False), (9000, 131072, 8, False)])
def test_xent_in_pieces_of_many_tokens(torch, ops, T, V, D, weighted):
    """Two and three pieces; widths whose rows are and are not 16-byte aligned."""
    h, w, labels = xent_inputs(torch, T, V, D, seed=13)
    tw = torch.rand(T, generator=gen(torch, 6), device="cuda") if weighted else None
    r = ops.linear_cross_entropy_grad(h, w, labels, token_weight=tw)
    step = 1500                       # the reference in 64 bits, by tokens
    dw = torch.zeros(V, D, dtype=torch.float64, device="cuda")
    dw_size = torch.zeros_like(dw)
    valid = labels >= 0
    wt = valid.double() * (1.0 if tw is None else tw.double())
    wt = wt / wt.sum()
    loss = 0.0
    for a in range(0, T, step):
        s = slice(a, min(T, a + step))
        ref = xent_reference(torch, h[s], w, labels[s], None, -100)
        mine = valid[s].double().sum()
        scale = wt[s] * mine / valid[s].double().clamp(min=1)           # undo the reference's own mean over this range
        l_err = sum_bound(D) * ref["size"] + 2.0 ** -18
        within(r.lse[s], ref["lse"], l_err + 2.0 ** -22 * ref["lse"].abs())
        within(r.token_loss[s], ref["token"], 2 * l_err + 2.0 ** -22 * ref["lse"].abs())
        p_err = 3.4e-4 + 2.0 ** -12 + 2 * l_err.max()
        dl, each = ref["dl"] * scale[:, None], (BF16 * ref["dl"] + p_err * ref["mag"]) * scale[:, None]
        within(r.d_hidden[s], ref["dh"] * scale[:, None], (each + sum_bound(V) * (dl + each)) @ ref["w"].abs() * (1 + BF16) + (BF16 + 2.0 ** -22) * (ref["dh"] * scale[:, None]).abs() + 1e-30)
        full = torch.exp(ref["h"] @ ref["w"].T - ref["lse"][:, None])
        rows = torch.nonzero(valid[s])[:, 0]
        full[rows, labels[s][rows]] -= 1
        full *= wt[s][:, None]
        dw += full.T @ ref["h"]
        dw_size += (each + sum_bound(T) * (dl + each)).T @ ref["h"].abs()
        loss += float((wt[s] * ref["token"]).sum())
        del ref, full, dl, each
    within(r.d_weight, dw, dw_size * (1 + BF16) + (BF16 + 2.0 ** -20) * dw.abs() + 1e-30)
    assert abs(float(r.loss) - loss) < 1e-4


def test_xent_all_ignored_and_no_tokens(torch, ops):
    h, w, labels = xent_inputs(torch, 40, 300, 64, seed=1)
    labels[:] = 7
    r = ops.linear_cross_entropy_grad(h, w, labels, ignore_index=7)
    assert float(r.loss) == 0 and not r.token_loss.any() and not r.d_hidden.any() and not r.d_weight.any()
    within(r.lse, torch.logsumexp(h.double() @ w.double().T, 1), torch.full((40,), 1e-4, dtype=torch.float64, device="cuda"))
    r = ops.linear_cross_entropy_grad(h[:0], w, labels[:0])
    assert float(r.loss) == 0 and r.token_loss.shape == (0,) and r.d_hidden.shape == (0, 64) and not r.d_weight.any() and r.d_weight.shape == (300, 64)
    r = ops.linear_cross_entropy(h[:0], w, labels[:0])
    assert float(r.loss) == 0 and r.lse.shape == (0,)


def test_xent_extreme_logits(torch, ops):
    """One column far above the rest, columns thousands below, and rows whose logits are all equal."""
    T, V, D = 70, 513, 64
    h, w, labels = xent_inputs(torch, T, V, D, seed=2, ignored=0.0)
    h[:20] *= 64
    w[300] *= 16
    h[20:30] = 0
    check_xent(torch, ops, h, w, labels)
    h2 = torch.zeros_like(h)
    h2[:, 0] = 1
    w2 = torch.zeros_like(w)
    w2[:, 0] = -3e38                    # as good as minus infinity everywhere but in two columns
    w2[5, 0], w2[400, 0] = 1, 1
    r = ops.linear_cross_entropy_grad(h2, w2, torch.full_like(labels, 5))
    assert torch.allclose(r.token_loss, torch.full((T,), math.log(2.0), device="cuda"), rtol=1e-6)
    assert torch.allclose(r.d_weight[5, 0].float(), torch.tensor(-0.5, device="cuda")) and torch.allclose(r.d_weight[400, 0].float(), torch.tensor(0.5, device="cuda"))
    assert not r.d_weight[6:400].any()


def test_xent_not_finite(torch, ops):
    """A NaN or an infinity in a hidden state stays in its row (and reaches the weight gradient); an ignored row with one is left out."""
    T, V, D = 300, 700, 64
    h, w, labels = xent_inputs(torch, T, V, D, seed=4, ignored=0.0)
    h[3, 5], h[270, 6] = float("nan"), float("inf")
    r = ops.linear_cross_entropy_grad(h, w, labels)
    bad = torch.zeros(T, dtype=torch.bool, device="cuda")
    bad[3] = bad[270] = True
    assert torch.equal(torch.isnan(r.token_loss), bad) and torch.equal(torch.isnan(r.d_hidden).all(1), bad) and torch.equal(torch.isnan(r.d_hidden).any(1), bad)
    assert bool(torch.isnan(r.loss)) and bool(torch.isnan(r.d_weight).all())
    labels[3] = labels[270] = -100
    r = ops.linear_cross_entropy_grad(h, w, labels)
    keep = ~bad
    ref = xent_reference(torch, h[keep], w, labels[keep], None, -100)
    assert bool(torch.isfinite(r.loss)) and bool((r.d_hidden[bad] == 0).all()) and bool((r.token_loss[bad] == 0).all())
    assert abs(float(r.loss) - float(ref["loss"])) < 1e-4
    # 0 * NaN: the row's gradient is zero, but the hidden state it would be multiplied with is not a number
    assert bool(torch.isnan(r.d_weight[:, 5:7]).all()) and bool(torch.isfinite(r.d_weight[:, :5]).all())


def test_xent_bad_label_is_reported(torch, ops):
    T, V, D = 20, 100, 64
    h, w, labels = xent_inputs(torch, T, V, D, seed=6, ignored=0.0)
    ok = labels.clone()
    labels[4], labels[9] = V + 10, -1
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    r = ops.linear_cross_entropy_grad(h, w, labels, status=status)
    assert int(status) == ops.PSGD_W_LABEL
    assert torch.equal(torch.isnan(r.token_loss).nonzero()[:, 0].cpu(), torch.tensor([4, 9])) and bool(torch.isnan(r.loss))
    assert not r.d_hidden[4].any() and not r.d_hidden[9].any() and bool(torch.isfinite(r.d_weight).all())
    assert bool(torch.isnan(ops.linear_cross_entropy(h, w, labels).loss))
    status.zero_()
    ops.linear_cross_entropy_grad(h, w, ok, status=status)
    assert int(status) == 0


def test_xent_strides_slots_and_streams(torch, ops):
    T, V, D = 260, 520, 200
    h, w, labels = xent_inputs(torch, T, V, D, seed=8)
    ref = xent_reference(torch, h, w, labels, None, -100)
    wide_h, wide_w = torch.full((T, D + 24), float("nan"), device="cuda", dtype=torch.bfloat16), torch.full((V, D + 9), float("nan"), device="cuda", dtype=torch.bfloat16)
    wide_h[:, 8:8 + D], wide_w[:, 3:3 + D] = h, w                        # one readable in place, one not
    G = torch.full((2, 3, V, D), 7.0, device="cuda", dtype=torch.bfloat16)
    dh = torch.full((T, D + 5), 7.0, device="cuda", dtype=torch.bfloat16)
    check_xent(torch, ops, wide_h[:, 8:8 + D], wide_w[:, 3:3 + D], labels, out=dict(d_weight=G[1, 2], d_hidden=dh[:, 2:2 + D]), ref=ref)
    assert bool((dh[:, :2] == 7).all()) and bool((dh[:, 2 + D:] == 7).all()) and bool((G.view(6, -1)[:5] == 7).all())
    plain = ops.linear_cross_entropy_grad(h, w, labels)
    assert torch.equal(plain.d_weight, G[1, 2]) and torch.equal(plain.d_hidden, dh[:, 2:2 + D])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        x = h * 1
    r = ops.linear_cross_entropy_grad(x, w, labels, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    for a, b in zip(r, plain):
        assert torch.equal(a, b)


def test_xent_gradient_by_differences(torch, ops):
    """Central differences of the kernel's own loss.  A step of 2^-4 in one entry (exact in bfloat16 by choice of the entries) moves a logit by
    at most 2^-4 |x|, |x| <= 1, so the cubic term is below (2^-4)^2 / 6 per unit of gradient; the loss is good to 2^-20, over a step of 2^-3."""
    T, V, D = 6, 40, 16
    g = gen(torch, 9)
    h = (torch.randint(-8, 9, (T, D), generator=g, device="cuda") / 8).to(torch.bfloat16)
    w = (torch.randint(-8, 9, (V, D), generator=g, device="cuda") / 8).to(torch.bfloat16)
    labels = torch.randint(V, (T,), generator=g, device="cuda")
    r = ops.linear_cross_entropy_grad(h, w, labels)
    step = 2.0 ** -4
    for name, at in [("h", (0, 0)), ("h", (3, 7)), ("h", (5, 15)), ("w", (0, 0)), ("w", (int(labels[2]), 3)), ("w", (39, 15))]:
        loss = []
        for sign in (1, -1):
            a = {"h": h.clone(), "w": w.clone()}
            a[name][at] += sign * step
            loss.append(float(ops.linear_cross_entropy(a["h"], a["w"], labels).loss))
        grad = float((r.d_hidden if name == "h" else r.d_weight)[at])
        assert abs((loss[0] - loss[1]) / (2 * step) - grad) <= step ** 2 / 6 + 2.0 ** -20 / step + 0.01 * abs(grad) + 1e-4


def test_xent_repeats_bit_for_bit(torch, ops):
    h, w, labels = xent_inputs(torch, 1000, 5000, 512, seed=12)
    a, b = (ops.linear_cross_entropy_grad(h, w, labels) for _ in range(2))
    for x, y in zip(a, b):
        assert torch.equal(x, y)


# ---- 8-bit activations --------------------------------------------------------------------------------------------
def pack_reference(x):
    """x [T, F] -> (q, scale byte per group), from the definition, group by group in 64 bits."""
    T, F = x.shape
    G = -(-F // GROUP)
    q, sb = np.zeros((T, G * GROUP), np.int8), np.zeros((T, G), np.uint8)
    for t in range(T):
        for g in range(G):
            v = x[t, g * GROUP:(g + 1) * GROUP].astype(np.float64)
            if not np.isfinite(v).all():
                sb[t, g] = 255
                continue
            top = np.abs(v).max()
            e = -126
            while 127 * 2.0 ** e < top and e < 121:
                e += 1
            q[t, g * GROUP:g * GROUP + len(v)] = np.clip(np.rint(v / 2.0 ** e), -127, 127)
            sb[t, g] = e + 127
    return q, sb


@pytest.mark.parametrize("T,F", [(1, 1), (1, 31), (3, 32), (2, 33), (5, 100), (37, 256), (9, 771), (70, 1025)])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_pack_is_the_definition(torch, ops, T, F, dtype):
    g = gen(torch, T * 100 + F)
    x = (torch.randn(T, F, generator=g, device="cuda") * torch.exp(6 * torch.randn(T, 1, generator=g, device="cuda"))).to(getattr(torch, dtype))
    if F > 40:
        x[0, :32] = 0
        x[-1, 32] = 0
    kept = ops.pack_activation(x)
    q, sb = pack_reference(x.float().cpu().numpy())
    assert np.array_equal(kept.q.cpu().numpy(), q) and np.array_equal(kept.scales.cpu().numpy(), sb)
    assert kept.nbytes == q.size + sb.size
    stands = (q.astype(np.float64) * 2.0 ** (np.repeat(sb, GROUP, 1).astype(np.float64) - 127))[:, :F]
    for t in (torch.bfloat16, torch.float32):
        assert np.array_equal(kept.unpack(t).double().cpu().numpy(), stands)
    wide = torch.full((T, F + 3), 5.0, device="cuda")
    kept.unpack(out=wide[:, 1:1 + F])
    assert np.array_equal(wide[:, 1:1 + F].double().cpu().numpy(), stands) and bool((wide[:, 0] == 5).all()) and bool((wide[:, 1 + F:] == 5).all())
    # a matrix that starts at an odd address and has a row stride of its own
    odd = torch.zeros((T, F + 7), dtype=x.dtype, device="cuda")
    odd[:, 1:1 + F] = x
    again = ops.pack_activation(odd[:, 1:1 + F])
    assert torch.equal(again.q, kept.q) and torch.equal(again.scales, kept.scales)


def test_pack_edges(torch, ops):
    """Ties, the mantissa at which the scale steps up, the smallest and largest numbers, infinities and NaN."""
    x = torch.zeros(12, 64, device="cuda")
    x[0, :4] = torch.tensor([127.0, 126.5, 0.5, -1.5])
    x[1, :3] = torch.tensor([127.5, 1.0, -3.0])          # above 127: scale 2
    x[2, :2] = torch.tensor([1.984375, 0.0078125])       # 127/64 exactly
    x[3, 0] = 1.9843751
    x[4, 0] = 1e-40
    x[5, 0] = 3.4028234e38
    x[5, 33] = -3.3895314e38
    x[6, 0], x[6, 40] = float("inf"), 2.0
    x[7, 63] = float("nan")
    x[8, 0] = 2.0 ** -126
    x[9, :] = -127.0
    x[10, 3] = 2.0 ** -149
    q, sb = pack_reference(x.cpu().numpy())
    kept = ops.pack_activation(x)
    assert np.array_equal(kept.q.cpu().numpy(), q) and np.array_equal(kept.scales.cpu().numpy(), sb)
    v = kept.unpack(torch.float32)
    assert bool(torch.isnan(v[6, :32]).all()) and float(v[6, 40]) == 2.0 and bool(torch.isnan(v[7, 32:]).all()) and not v[7, :32].any()
    assert bool(torch.isfinite(v[5]).all())
    b = kept.unpack(torch.bfloat16).float()
    assert torch.equal(torch.nan_to_num(b, nan=1.0), torch.nan_to_num(v, nan=1.0))


def test_pack_beyond_32_bit_offsets(torch, ops):
    T, F = (1 << 20) + 3, 2080                           # 2.2e9 values
    x = torch.zeros((T, F), dtype=torch.bfloat16, device="cuda")
    tail = torch.randn(5, F, generator=gen(torch, 1), device="cuda").to(torch.bfloat16)
    x[-5:] = tail
    kept = ops.pack_activation(x)
    want = ops.pack_activation(tail)
    assert torch.equal(kept.q[-5:], want.q) and torch.equal(kept.scales[-5:], want.scales)
    del x
    out = kept.unpack()
    assert torch.equal(out[-5:], want.unpack()) and not out[:1000].any()


def test_no_rows(torch, ops):
    x = torch.zeros((0, 40), dtype=torch.bfloat16, device="cuda")
    kept = ops.pack_activation(x)
    assert kept.q.shape == (0, 64) and kept.unpack().shape == (0, 40)
    dw = ops.weight_gradient(torch.zeros((0, 24), dtype=torch.bfloat16, device="cuda"), kept)
    assert dw.shape == (24, 40) and not dw.any()
    h, a, b = ops.swiglu_forward(x, x)
    assert h.shape == (0, 40) and all(t.shape == (0, 40) for t in ops.swiglu_backward(x, a, b, recompute=True))


WGRAD_SHAPES = [(1, 8, 32), (1, 1, 1), (17, 33, 65), (64, 256, 256), (65, 300, 129), (300, 1000, 520), (1000, 257, 771), (4096, 768, 768), (4097, 520, 200), (9000, 300, 260),
                (129, 2048, 768), (777, 5504, 264)]


@pytest.mark.parametrize("T,O,F", WGRAD_SHAPES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_weight_gradient_matches_definition(torch, ops, T, O, F, dtype):
    g = gen(torch, T + O + F)
    x = (torch.randn(T, F, generator=g, device="cuda") * torch.exp(torch.randn(F, generator=g, device="cuda"))).to(torch.bfloat16)
    dy = (torch.randn(T, O, generator=g, device="cuda") * 1e-3).to(torch.bfloat16)
    kept = ops.pack_activation(x)
    xs, dyd = kept.unpack(torch.float32).double(), dy.double()
    ref, size = dyd.T @ xs, dyd.abs().T @ xs.abs()
    out = ops.weight_gradient(dy, kept, dtype=getattr(torch, dtype))
    within(out, ref, sum_bound(T) * size + (BF16 + 2.0 ** -20) * ref.abs() * (dtype == "bfloat16") + 1e-30)
    assert torch.equal(out, ops.weight_gradient(dy, kept, dtype=getattr(torch, dtype)))


@pytest.mark.parametrize("T,O,F", [(2049, 300, 131), (5000, 1027, 770), (9001, 70, 3), (4100, 2600, 1533)])
def test_weight_gradient_with_rows_of_odd_length(torch, ops, T, O, F):
    """Results whose rows are not 16-byte aligned, with more terms than one accumulator takes (T > 2048)."""
    g = gen(torch, T + O)
    x = torch.randn(T, F, generator=g, device="cuda").to(torch.bfloat16)
    dy = torch.randn(T, O, generator=g, device="cuda").to(torch.bfloat16)
    kept = ops.pack_activation(x)
    xs, dyd = kept.unpack(torch.float32).double(), dy.double()
    ref, size = dyd.T @ xs, dyd.abs().T @ xs.abs()
    out = ops.weight_gradient(dy, kept)
    within(out, ref, sum_bound(T) * size)
    wide = torch.full((O, F + 2), 9.0, device="cuda")                    # a result that starts at an odd place, whatever its width
    ops.weight_gradient(dy, kept, out=wide[:, 1:1 + F])
    within(wide[:, 1:1 + F], ref, sum_bound(T) * size)
    assert bool((wide[:, 0] == 9).all()) and bool((wide[:, 1 + F] == 9).all())


@pytest.mark.parametrize("T", [1, 64, 65, 130])
def test_weight_gradient_of_groups_that_are_not_numbers(torch, ops, T):
    """An infinity in the last row makes the 32 input columns of its group NaN, and no others (rows behind the last one count as zeros)."""
    O, F = 40, 200
    g = gen(torch, T)
    x = torch.randn(T, F, generator=g, device="cuda").to(torch.bfloat16)
    dy = torch.randn(T, O, generator=g, device="cuda").to(torch.bfloat16)
    x[-1, 70], x[0, 199] = float("inf"), float("nan")
    dw = ops.weight_gradient(dy, ops.pack_activation(x))
    bad = torch.zeros(F, dtype=torch.bool, device="cuda")
    bad[64:96] = bad[192:200] = True
    assert bool(torch.isnan(dw[:, bad]).all()) and bool(torch.isfinite(dw[:, ~bad]).all())


def test_weight_gradient_of_extreme_scales(torch, ops):
    """Groups at both ends of the scale's range come out exactly (one row: every entry is one product)."""
    x = torch.ones(1, 96, device="cuda")
    x[:, :32] *= 3.0e38
    x[:, 32:64] *= 2.0 ** -125
    kept = ops.pack_activation(x)
    dy = torch.tensor([[0.5, -0.25]], device="cuda", dtype=torch.bfloat16)
    assert torch.equal(ops.weight_gradient(dy, kept), dy.float().T @ kept.unpack(torch.float32))


def test_weight_gradient_slots_and_strides(torch, ops):
    T, O, F = 333, 264, 136
    g = gen(torch, 2)
    x = torch.randn(T, F, generator=g, device="cuda").to(torch.bfloat16)
    wide = torch.full((T, O + 5), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 3:3 + O] = torch.randn(T, O, generator=g, device="cuda").to(torch.bfloat16)
    dy = wide[:, 3:3 + O]
    kept = ops.pack_activation(x)
    for dt in (torch.float32, torch.bfloat16):
        G = torch.full((2, 2, O, F), 3.0, dtype=dt, device="cuda")
        want = ops.weight_gradient(dy.contiguous(), kept, dtype=dt)
        assert ops.weight_gradient(dy, kept, out=G[0, 1]).data_ptr() == G[0, 1].data_ptr()
        assert torch.equal(G[0, 1], want) and bool((G[0, 0] == 3).all()) and bool((G[1] == 3).all())
        odd = torch.full((O, F + 3), 3.0, dtype=dt, device="cuda")
        ops.weight_gradient(dy, kept, out=odd[:, 1:1 + F])
        assert torch.equal(odd[:, 1:1 + F], want) and bool((odd[:, 0] == 3).all()) and bool((odd[:, 1 + F:] == 3).all())


# ---- gated unit ---------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("T,F", [(1, 1), (2, 40), (33, 256), (7, 771), (64, 2048), (129, 1000)])
def test_swiglu_matches_definition(torch, ops, T, F):
    g = gen(torch, F)
    gate, up, dh = ((torch.randn(T, F, generator=g, device="cuda") * s).to(torch.bfloat16) for s in (3.0, 1.0, 1e-3))
    if F > 100:
        gate[0, :6] = torch.tensor([100.0, -100.0, 30.0, -30.0, 0.0, -0.0], dtype=torch.bfloat16)
    h, kg, ku = ops.swiglu_forward(gate, up)
    pg, pu = ops.pack_activation(gate), ops.pack_activation(up)
    assert torch.equal(kg.q, pg.q) and torch.equal(kg.scales, pg.scales) and torch.equal(ku.q, pu.q) and torch.equal(ku.scales, pu.scales)

    def close(got, ref, size):     # one rounding to bfloat16, float32 arithmetic and exp of arguments up to 128 before it
        within(got, ref, BF16 * ref.abs() + 2.0 ** -15 * size + 1e-38)

    sil = lambda v: v * torch.sigmoid(v)
    a, b, d = gate.double(), up.double(), dh.double()
    close(h, sil(a) * b, (sil(a) * b).abs())
    a, b = kg.unpack(torch.float32).double(), ku.unpack(torch.float32).double()
    d_gate, d_up, again = ops.swiglu_backward(dh, kg, ku, recompute=True)
    s = torch.sigmoid(a)
    close(d_gate, d * b * (s + a * s * (1 - s)), (d * b * s).abs() * (1 + (a * (1 - s)).abs()))
    close(d_up, d * sil(a), (d * sil(a)).abs())
    close(again, sil(a) * b, (sil(a) * b).abs())
    short = ops.swiglu_backward(dh, kg, ku)
    assert len(short) == 2 and torch.equal(short[0], d_gate) and torch.equal(short[1], d_up)


def test_swiglu_gradient_by_differences(torch, ops):
    """Slope of silu(g) u from the checkpoint against central differences of the definition in 64 bits (step 1e-4: error below 1e-8)."""
    gate = torch.linspace(-6, 6, 64, device="cuda").to(torch.bfloat16)[None]
    up = torch.linspace(-1, 2, 64, device="cuda").to(torch.bfloat16)[None]
    _, kg, ku = ops.swiglu_forward(gate, up)
    dh = torch.ones_like(gate)
    d_gate, d_up = ops.swiglu_backward(dh, kg, ku)
    a, b = kg.unpack(torch.float32).double(), ku.unpack(torch.float32).double()
    f = lambda x, y: x / (1 + torch.exp(-x)) * y
    e = 1e-4
    within(d_gate, (f(a + e, b) - f(a - e, b)) / (2 * e), BF16 * (b.abs() * 1.2) + 1e-5)
    within(d_up, (f(a, b + e) - f(a, b - e)) / (2 * e), BF16 * a.abs() + 1e-5)


def test_swiglu_strides_and_streams(torch, ops):
    T, F = 65, 520
    g = gen(torch, 3)
    both = torch.randn(T, 2 * F + 3, generator=g, device="cuda").to(torch.bfloat16)   # gate and up side by side, as one product writes them
    gate, up = both[:, :F], both[:, F + 3:]
    h, kg, ku = ops.swiglu_forward(gate, up)
    h2, kg2, ku2 = ops.swiglu_forward(gate.contiguous(), up.contiguous())
    assert torch.equal(h, h2) and torch.equal(kg.q, kg2.q) and torch.equal(ku.q, ku2.q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    a = ops.swiglu_backward(h, kg, ku, recompute=True, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    for x, y in zip(a, ops.swiglu_backward(h2, kg2, ku2, recompute=True)):
        assert torch.equal(x, y)


# ---- refusals -----------------------------------------------------------------------------------------------------
def test_refusals(torch, ops):
    E = ops.PSGDError
    h, w, labels = xent_inputs(torch, 8, 16, 64, seed=1)
    for bad in [dict(hidden=h.float()), dict(weight=w[:, :32]), dict(labels=labels.int()), dict(labels=labels[:4]), dict(hidden=h.cpu()), dict(weight=w.t()),
                dict(token_weight=torch.ones(8, dtype=torch.float64, device="cuda")), dict(hidden=h[None]), dict(weight=w[:0])]:
        with pytest.raises(E):
            ops.linear_cross_entropy(**{**dict(hidden=h, weight=w, labels=labels), **bad})
    for bad in [dict(d_hidden=h.float()), dict(d_weight=h), dict(d_weight=torch.zeros(16, 128, dtype=torch.bfloat16, device="cuda")[:, ::2]),
                dict(status=torch.zeros(1, device="cuda"))]:
        with pytest.raises(E):
            ops.linear_cross_entropy_grad(h, w, labels, **bad)
    kept = ops.pack_activation(h)
    with pytest.raises(E):
        ops.pack_activation(h.half())
    with pytest.raises(E):
        ops.pack_activation(h[0])
    with pytest.raises(E):
        ops.pack_activation(h[:, :0])
    with pytest.raises(E):
        ops.weight_gradient(h[:4], kept)
    with pytest.raises(E):
        ops.weight_gradient(h, h)
    with pytest.raises(E):
        ops.weight_gradient(h, kept, dtype=torch.float16)
    with pytest.raises(E):
        ops.weight_gradient(h, kept, out=torch.zeros(64, 63, device="cuda"))
    with pytest.raises(E):
        ops.swiglu_forward(h, h[:, :32])
    with pytest.raises(E):
        ops.swiglu_backward(h[:, :32], kept, kept)
    with pytest.raises(E):
        kept.unpack(torch.float16)


def test_c_entry_points_refuse(torch, ops):
    """The C calls check before anything is launched: alignment, strides, workspace size, NULL, extents."""
    import ctypes as C

    L = ops.lib()
    h, w, labels = xent_inputs(torch, 8, 16, 64, seed=1)
    n = C.c_size_t()
    assert L.psgd_xent_workspace(8, 16, 64, 1, C.byref(n)) == 0 and n.value > 0
    ws = torch.zeros(n.value, dtype=torch.uint8, device="cuda")
    f = torch.zeros(64, device="cuda")
    dh, dw = torch.full_like(h, 2.0), torch.full_like(w, 2.0)

    def call(H=h.data_ptr(), ldh=64, W=w.data_ptr(), ldw=64, lab=labels.data_ptr(), T=8, V=16, D=64, dW=dw.data_ptr(), lddw=64, wsp=ws.data_ptr(), nb=n.value):
        return L.psgd_xent_grad(H, ldh, W, ldw, lab, None, -100, T, V, D, f.data_ptr(), f.data_ptr() + 16, f.data_ptr() + 64, dh.data_ptr(), 64, dW, lddw, None, wsp, nb, None)

    assert call(H=None) == -2 and call(W=None) == -2 and call(lab=None) == -2 and call(dW=None) == -2 and call(wsp=None) == -2
    assert call(H=h.data_ptr() + 2) == -1 and call(ldh=65) == -1 and call(ldw=63) == -1 and call(lddw=32) == -1 and call(wsp=ws.data_ptr() + 16) == -1
    assert call(T=-1) == -1 and call(V=0) == -1 and call(D=0) == -1 and call(T=1 << 40) == -1
    assert call(nb=n.value - 1) == -3
    torch.cuda.synchronize()
    assert bool((dw == 2).all()) and bool((dh == 2).all()) and not f.any()
    assert call() == 0
    torch.cuda.synchronize()
    assert not bool((dw == 2).all())
    assert L.psgd_act_pack(h.data_ptr(), 32, 1, 8, 64, ws.data_ptr(), ws.data_ptr(), None) == -1
    assert L.psgd_act_pack(h.data_ptr(), 64, 2, 8, 64, ws.data_ptr(), ws.data_ptr(), None) == -1
    assert L.psgd_act_pack(h.data_ptr(), 64, 1, 8, 64, ws.data_ptr() + 1, ws.data_ptr(), None) == -1
    assert L.psgd_act_pack(None, 64, 1, 8, 64, ws.data_ptr(), ws.data_ptr(), None) == -2
    assert L.psgd_act_wgrad_workspace(8, 0, 64, C.byref(n)) == -1 and L.psgd_act_wgrad_workspace(8, 16, 64, None) == -2
    assert L.psgd_swiglu_backward(h.data_ptr(), 64, None, None, None, None, 8, 64, dh.data_ptr(), 64, dh.data_ptr(), 64, None, 0, None) == -2


@pytest.mark.parametrize("T", [1, 2, 3, 19])
@pytest.mark.parametrize("F", [1, 2, 5, 7, 8, 9, 31, 33, 250, 256, 257, 263, 505, 521, 1031])
def test_rows_of_any_alignment_equal_aligned_ones(torch, ops, T, F):
    """Every start within 16 bytes and strides that move it from row to row: the same bits as from aligned copies, and nothing around the rows changes."""
    g = gen(torch, 100 * F + T)
    wide = (F + 7) // 8 * 8
    for start, gap in [(0, 0), (1, 0), (2, 1), (3, 2), (5, 3), (6, 4), (7, 7), (8, 1), (4, 8)]:
        ld = F + gap
        flat = torch.randn(start + T * ld + 16, generator=g, device="cuda").to(torch.bfloat16)
        x, y = (flat.as_strided((T, F), (ld, 1), start), flat.as_strided((T, F), (ld, 1), start + (1 if gap else 0)))

        def aligned(t):                             # padded with zeros to whole units of 8: the same groups, the same values
            a = torch.zeros(T, wide, device="cuda", dtype=torch.bfloat16)
            a[:, :F] = t
            return a

        ax, ay = aligned(x), aligned(y)
        k, ak = ops.pack_activation(x), ops.pack_activation(ax)
        assert torch.equal(k.q, ak.q) and torch.equal(k.scales, ak.scales)
        out = torch.full((start + T * ld + 24,), 7.0, device="cuda", dtype=torch.bfloat16)
        before = out.clone()
        view = out.as_strided((T, F), (ld, 1), start)
        k.unpack(out=view)
        assert torch.equal(view, ak.unpack()[:, :F])
        view.copy_(before.as_strided((T, F), (ld, 1), start))
        assert torch.equal(out, before)
        h, kg, ku = ops.swiglu_forward(x, y)
        ah, akg, aku = ops.swiglu_forward(ax, ay)
        assert torch.equal(h, ah[:, :F]) and torch.equal(kg.q, akg.q) and torch.equal(ku.q, aku.q) and torch.equal(kg.scales, akg.scales) and torch.equal(ku.scales, aku.scales)
        for a, b in zip(ops.swiglu_backward(x, kg, ku, recompute=True), ops.swiglu_backward(ax, akg, aku, recompute=True)):
            assert torch.equal(a, b[:, :F])
        for a, b in zip(ops.swiglu_backward(y, kg, ku), ops.swiglu_backward(ay, akg, aku)):
            assert torch.equal(a, b[:, :F])
        dw, adw = ops.weight_gradient(y, k), ops.weight_gradient(ay, ak)
        assert torch.equal(dw, adw[:F, :F])


# ---- streams, graphs, long offsets --------------------------------------------------------------------------------
def test_calls_on_two_streams_at_once(torch, ops):
    sets = [xent_inputs(torch, 700, 3000, 256, seed=s) for s in (21, 22)]
    x = [torch.randn(500, 776, generator=gen(torch, s), device="cuda").to(torch.bfloat16) for s in (23, 24)]

    def work(i, stream=None):
        r = ops.linear_cross_entropy_grad(*sets[i], stream=stream)
        kept = ops.pack_activation(x[i], stream=stream)
        return [*r, ops.weight_gradient(x[i][:, :520].contiguous(), kept, stream=stream)]

    want = [work(0), work(1)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        got.append([work(i, streams[i]) for i in (0, 1)])
    torch.cuda.synchronize()
    for both in got:
        for a, b in zip(both, want):
            for u, v in zip(a, b):
                assert torch.equal(u, v)


def test_inputs_freed_before_another_stream_has_read_them(torch, ops):
    """The caller drops its inputs while the call's stream is still busy: their memory is not given to the next allocation before they are read."""
    h, w, labels = xent_inputs(torch, 300, 1100, 200, seed=25)
    x = torch.randn(300, 264, generator=gen(torch, 26), device="cuda").to(torch.bfloat16)

    def work(h, w, labels, x, stream=None):
        y, kg, ku = ops.swiglu_forward(x, x, stream=stream)
        return [*ops.linear_cross_entropy_grad(h, w, labels, stream=stream), y, *ops.swiglu_backward(x, kg, ku, recompute=True, stream=stream),
                ops.weight_gradient(x, ops.pack_activation(x, stream=stream), stream=stream)]

    want = work(h, w, labels, x)
    s = torch.cuda.Stream()
    mine = [t.clone() for t in (h, w, labels, x)]
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)               # about ten milliseconds
    got = work(*mine, stream=s)
    sizes = [(t.shape, t.dtype) for t in mine]
    del mine
    torch.cuda.current_stream().synchronize()
    others = [torch.full(shape, 3, dtype=dtype, device="cuda") for shape, dtype in sizes for _ in range(4)]
    torch.cuda.synchronize()
    assert len(others) == 16
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_calls_in_a_cuda_graph(torch, ops):
    """Captured once, replayed with other inputs in the same places."""
    h, w, labels = xent_inputs(torch, 300, 1100, 200, seed=31)
    x = torch.randn(300, 264, generator=gen(torch, 32), device="cuda").to(torch.bfloat16)

    def work():
        r = ops.linear_cross_entropy_grad(h, w, labels)
        loss = ops.linear_cross_entropy(h, w, labels).loss
        y, kg, ku = ops.swiglu_forward(x, x)
        return [*r, loss, ops.weight_gradient(r.d_hidden, ops.pack_activation(x)), *ops.swiglu_backward(y, kg, ku, recompute=True)]

    work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = work()
    h2, w2, labels2 = xent_inputs(torch, 300, 1100, 200, seed=33)
    h.copy_(h2), w.copy_(w2), labels.copy_(labels2), x.neg_()
    for t in out:
        t.fill_(7)
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(out, work()):
        assert torch.equal(a, b)


def test_xent_beyond_32_bit_offsets(torch, ops):
    """A vocabulary matrix of 2.2e9 entries; the labels lie at both ends."""
    T, V, D = 5, 540000, 4000
    g = gen(torch, 41)
    h = torch.randn(T, D, generator=g, device="cuda").to(torch.bfloat16)
    w = torch.empty(V, D, dtype=torch.bfloat16, device="cuda")
    for a in range(0, V, 60000):
        w[a:a + 60000] = (torch.randn(60000, D, generator=g, device="cuda") / math.sqrt(D)).to(torch.bfloat16)
    labels = torch.tensor([0, V - 1, V - 2, -100, V // 2], device="cuda")
    r = ops.linear_cross_entropy_grad(h, w, labels)
    z = torch.cat([h.double() @ w[a:a + 60000].double().T for a in range(0, V, 60000)], 1)
    lse = torch.logsumexp(z, 1)
    within(r.lse, lse, torch.full_like(lse, 1e-4))
    p = torch.softmax(z, 1)
    rows = torch.tensor([0, 1, 2, 4], device="cuda")
    p[rows, labels[rows]] -= 1
    p[3] = 0
    p /= 4
    for a in (0, V // 2 - 100, V - 1000):
        ref, size = p[:, a:a + 1000].T @ h.double(), p[:, a:a + 1000].abs().T @ h.double().abs()
        within(r.d_weight[a:a + 1000], ref, (2 * BF16 + 1e-3) * size)
    dh = sum(p[:, a:a + 60000] @ w[a:a + 60000].double() for a in range(0, V, 60000))
    size = sum(p[:, a:a + 60000].abs() @ w[a:a + 60000].double().abs() for a in range(0, V, 60000))
    within(r.d_hidden, dh, (2 * BF16 + 1e-3) * size)


# ---- together -----------------------------------------------------------------------------------------------------
def test_operators_feed_the_compressor(torch, ops):
    """The example: two simulated nodes, 8-bit activations, compressed gradients.  The task is a fixed map of tokens, learnt within 60 steps."""
    import importlib.util
    import os

    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "compressed_training.py")
    spec = importlib.util.spec_from_file_location("compressed_training", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses = example.train(steps=60, log=None)
    assert abs(losses[0] - math.log(2000)) < 0.2 and losses[-1] < 0.1 and all(math.isfinite(v) for v in losses)


# ---- tokens that the model is sure of -----------------------------------------------------------------------------
@pytest.mark.parametrize("base", [-60, 0, 20, 60, 100])
@pytest.mark.parametrize("V", [90, 700, 50257])
def test_xent_of_confident_tokens(torch, ops, V, base):
    """Tokens whose label has 1 - p of 1e-3 to 1e-5, at logits of any size: the label's gradient and the loss are good relative to 1 - p.

    Column 0 of the weight lifts every logit of a token by `base`, and every token has a label and a column of its own that lifts it further, so that
    d_hidden[t, own column] and d_weight[label, own column] / lift are the gradient of the label's logit alone and d_hidden[t, 0] is the
    sum of all the gradients of the token's logits, which is 0.
    Bounds: a logit is good to l_err, which moves 1 - p by 2 l_err of itself; the sum of the exponentials is 1 + (1 - p) / p and meets, beside
    the 1, at most 8 roundings of 2^-24; the gradient is rounded to bfloat16 once before and once after the product; p of the other columns by 3.4e-4 for the
    stored exponents and once to bfloat16.
    """
    T, D = 24, 64
    g = gen(torch, V + base)
    h = torch.zeros(T, D, device="cuda")
    w = torch.zeros(V, D, device="cuda")
    own = torch.arange(1, T + 1, device="cuda")
    rows = torch.arange(T, device="cuda")
    h[:, T + 1:] = torch.randn(T, D - T - 1, generator=g, device="cuda") * 0.15
    w[:, T + 1:] = torch.randn(V, D - T - 1, generator=g, device="cuda")
    labels = torch.randperm(V, generator=g, device="cuda")[:T]
    h[:, 0], w[:, 0] = base, 1
    rest = 10.0 ** -torch.linspace(3, 5, T, device="cuda")
    h[rows, own] = math.log(V) + 0.4 - torch.log(rest)
    w[labels, own] = 1
    w[labels, T + 1:] = 0                                                # the label stands at base + lift exactly
    h, w = h.to(torch.bfloat16), w.to(torch.bfloat16)
    lift = h[rows, own].double()
    ref = xent_reference(torch, h, w, labels, None, -100)
    miss = -torch.expm1(-ref["token"])                                   # 1 - p
    assert bool(((miss > 3e-6) & (miss < 3e-3)).all())
    l_err = sum_bound(D) * ref["size"]
    off = 2 * l_err * miss + 8 * 2.0 ** -24
    for r in (ops.linear_cross_entropy(h, w, labels), ops.linear_cross_entropy_grad(h, w, labels)):
        within(r.token_loss, ref["token"], off + 2.0 ** -21 * ref["token"])
        within(r.lse, ref["lse"], l_err + 2.0 ** -22 * ref["lse"].abs() + 2.0 ** -21)
    grad = -miss / T
    bound = (off * (1 + 2 * BF16) + 2 * BF16 * miss) / T
    within(r.d_hidden[rows, own], grad, bound)
    within(r.d_weight[labels, own].double() / lift, grad, bound)
    within(r.d_hidden[:, 0], torch.zeros_like(grad), (off + (2 * BF16 + 3.4e-4 + 2.0 ** -12 + 2 * l_err) * 2 * miss) / T)


# ---- waits that run out -------------------------------------------------------------------------------------------
def test_results_behind_a_wait_that_ran_out_are_nan(torch, ops, tmp_path, monkeypatch):
    """A build whose epilogue gives up every wait for an accumulator at once (the products themselves run to their end; no pair has more than two
    accumulators here, so none waits for this epilogue): every result is NaN, without a status word too, and the status word says why."""
    import ctypes as C
    import subprocess

    from paper_2509_11254_b200 import binding, build

    so = str(tmp_path / "gives_up.so")
    src = [s for s in build.SRCS if s.endswith("psgd_lm.cu")]
    subprocess.run([build.nvcc_path(), "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-Xcompiler", "-fPIC", "-shared", "-DPSGD_WARP_WAIT_LIMIT=0",
                    "-o", so, *src], check=True, capture_output=True)
    L = C.CDLL(so)
    for name, (res, args) in binding.SIGNATURES.items():
        if hasattr(L, name):
            getattr(L, name).restype, getattr(L, name).argtypes = res, args
    h, w, labels = xent_inputs(torch, 300, 700, 64, seed=3)
    x = torch.randn(100, 136, generator=gen(torch, 4), device="cuda").to(torch.bfloat16)
    dy = torch.randn(100, 264, generator=gen(torch, 5), device="cuda").to(torch.bfloat16)
    kept = ops.pack_activation(x)
    monkeypatch.setattr(binding, "_lib", L)
    only, full = ops.linear_cross_entropy(h, w, labels), ops.linear_cross_entropy_grad(h, w, labels)
    counts = labels != -100
    for r in (only, full):
        assert bool(torch.isnan(r.loss)) and bool(torch.isnan(r.lse).all()) and bool(torch.isnan(r.token_loss[counts]).all())
    assert bool(torch.isnan(full.d_hidden).all()) and bool(torch.isnan(full.d_weight).all())
    for dtype in (torch.float32, torch.bfloat16):
        assert bool(torch.isnan(ops.weight_gradient(dy, kept, dtype=dtype)).all())
    assert bool(torch.isnan(ops.weight_gradient(dy[:, :263], kept, out=torch.zeros(263, 137, device="cuda")[:, 1:])).all())
    for call in (lambda s: ops.linear_cross_entropy(h, w, labels, status=s), lambda s: ops.linear_cross_entropy_grad(h, w, labels, status=s), lambda s: ops.weight_gradient(dy, kept, status=s)):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        call(status)
        assert int(status) == ops.PSGD_W_TIMEOUT


# ---- outputs in the way of inputs ---------------------------------------------------------------------------------
def test_outputs_beside_inputs_but_not_over_them(torch, ops):
    """Gradients in the other columns of the buffers that hold the operands are right; over the operands they are refused before anything is launched."""
    T, V, D = 260, 520, 64
    h, w, labels = xent_inputs(torch, T, V, D, seed=51)
    want = ops.linear_cross_entropy_grad(h, w, labels)
    H, W = (torch.cat([t, torch.full_like(t, 7)], 1) for t in (h, w))
    got = ops.linear_cross_entropy_grad(H[:, :D], W[:, :D], labels, d_hidden=H[:, D:], d_weight=W[:, D:])
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    assert torch.equal(H[:, :D], h) and torch.equal(W[:, :D], w)
    for bad in (dict(d_hidden=h), dict(d_weight=w), dict(d_hidden=w[:T]), dict(d_weight=W[:, D:], d_hidden=W[3:3 + T, D:])):
        with pytest.raises(ops.PSGDError):
            ops.linear_cross_entropy_grad(h, w, labels, **bad)
    dy = torch.randn(T, T, generator=gen(torch, 52), device="cuda").to(torch.bfloat16)
    kept = ops.pack_activation(h)
    with pytest.raises(ops.PSGDError):
        ops.weight_gradient(dy, kept, out=dy[:, :D])


def test_loss_of_many_tokens_in_pieces(torch, ops):
    """More statistics than the workspace holds at a time: three pieces of tokens, the same bits per token as from calls that take one, and the mean over all of them."""
    T, V, D = 70001, 131072 - 5, 16
    h, w, labels = xent_inputs(torch, T, V, D, seed=61)
    labels[12345] = V - 1
    tw = torch.rand(T, generator=gen(torch, 62), device="cuda")
    r = ops.linear_cross_entropy(h, w, labels, token_weight=tw)
    for a in range(0, T, 20000):
        s = slice(a, min(T, a + 20000))
        one = ops.linear_cross_entropy(h[s], w, labels[s], token_weight=tw[s])
        assert torch.equal(r.lse[s], one.lse) and torch.equal(r.token_loss[s], one.token_loss)
    tail = slice(T - 500, T)
    z = h[tail].double() @ w.double().T
    within(r.lse[tail], torch.logsumexp(z, 1), sum_bound(D) * (h[tail].double().abs() @ w.double().abs().T).amax(1) + 2.0 ** -18 + 2.0 ** -22 * 16)
    wt = tw.double() * (labels != -100)
    loss = float((wt * r.token_loss.double()).sum() / wt.sum())
    assert abs(float(r.loss) - loss) <= 2.0 ** -23 * abs(loss) * 2


# ---- autograd -----------------------------------------------------------------------------------------------------
def test_lost_autograd_graph_is_warned_about(torch, ops):
    """Results that look differentiable and are not: a warning where an input requires a gradient, none under no_grad, none from the calls that return gradients."""
    import warnings

    h, w, labels = xent_inputs(torch, 40, 90, 64, seed=71)
    leaf = h.clone().requires_grad_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for call in (lambda: ops.linear_cross_entropy(leaf, w, labels), lambda: ops.linear_cross_entropy(h, w.clone().requires_grad_(), labels, stream=side),
                 lambda: ops.swiglu_forward(h, leaf), lambda: ops.swiglu_forward(leaf, h, stream=side)):
        with pytest.warns(UserWarning, match="no autograd graph") as seen:
            call()
        assert len(seen) == 1 and seen[0].filename == __file__
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        with torch.no_grad():
            ops.linear_cross_entropy(leaf, w, labels)
            ops.swiglu_forward(leaf, leaf)
        ops.linear_cross_entropy(h, w, labels)
        ops.swiglu_forward(h, h)
        ops.linear_cross_entropy_grad(leaf, w, labels)
        ops.pack_activation(leaf)
    torch.cuda.synchronize()


def test_two_streams_at_once_with_inputs_made_before(torch, ops):
    """Both streams find their inputs complete: nothing but the operators runs between the synchronisations."""
    sets = [xent_inputs(torch, 700, 3000, 256, seed=s) for s in (81, 82)]
    x = [torch.randn(500, 776, generator=gen(torch, s), device="cuda").to(torch.bfloat16) for s in (83, 84)]
    dy = [t[:, :520].contiguous() for t in x]

    def work(i, stream=None):
        r = ops.linear_cross_entropy_grad(*sets[i], stream=stream)
        only = ops.linear_cross_entropy(*sets[i], stream=stream)
        kept = ops.pack_activation(x[i], stream=stream)
        h, kg, ku = ops.swiglu_forward(x[i], x[i], stream=stream)
        return [*r, *only, ops.weight_gradient(dy[i], kept, stream=stream), h, *ops.swiglu_backward(h, kg, ku, recompute=True, stream=stream), kept.unpack(stream=stream)]

    want = [work(0), work(1)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[work(i, streams[i]) for i in (0, 1)] for _ in range(5)]
    torch.cuda.synchronize()
    for both in got:
        for a, b in zip(both, want):
            for u, v in zip(a, b):
                assert torch.equal(u, v)
