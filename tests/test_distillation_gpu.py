"""Distillation of the last layer from a teacher's top logits against its definition in 64 bits.

Tolerances.  Elementwise, from how the result is formed (u = 2^-24, half a step of float32):
  * a logit is a sum of D products on the tensor cores, 16 at a time into one float32 addition that may truncate: (D / 16 + 8) 2^-23 sum |h w|; divided by the temperature it and what is
    formed from it carry 2^-22 of their size, and the log-sum-exp 2^-18 of its own (sums of up to 2^18 terms, exp and log): together `le`;
  * q carries 2^-20 and 2^-22 of its exponent's size; log q and log p 2^-21 of their sizes;
  * the gradient of a logit: once rounded to bfloat16 (2^-8), the stored exponent (3.4e-4 of p), 2^-12 for the evaluation of p, and what le moves; then the
    products' sums, and one rounding to bfloat16.
"""
import math
import warnings

import pytest

pytestmark = pytest.mark.gpu

BF16 = 2.0 ** -8
U = 2.0 ** -24


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
    d = (got.double() - ref).abs()
    assert bool((d <= bound).all()), f"worst error / bound {float((d / bound.clamp(min=1e-300)).max()):.3g}"


def reference(torch, h, w, z, index, tau, tw):
    h, w, z = h.double(), w.double(), z.double() / tau
    T, V = h.shape[0], w.shape[0]
    l = h @ w.T / tau
    size = (h.abs() @ w.abs().T).amax(1) / tau
    lse = torch.logsumexp(l, 1)
    there = (index >= 0) & (z > -math.inf)
    counts = there.any(1)
    z = torch.where(there, z, -math.inf)
    z = z - torch.where(counts, z.amax(1), 0.0)[:, None]
    total = torch.exp(z).sum(1, keepdim=True)
    log_q = z - torch.log(torch.where(counts[:, None], total, 1.0))
    q = torch.exp(log_q)
    at = index.clamp(0, V - 1)
    log_p = l.gather(1, at) - lse[:, None]
    live = there & (q > 0)
    gap = torch.where(live, log_q - log_p, 0.0)
    token = tau ** 2 * (q * gap).sum(1)
    le = sum_bound(h.shape[1]) * size + 2.0 ** -22 * size + 2.0 ** -18
    zero = torch.zeros_like(q)
    q_err = 2.0 ** -20 + 2.0 ** -22 * torch.where(live, z.abs(), zero)
    t_err = tau ** 2 * (2 * le + (q * q_err * gap.abs()).sum(1) + 2.0 ** -21 * torch.where(live, q * (log_q.abs() + log_p.abs()), zero).sum(1)) * counts
    wt = torch.where(counts, torch.ones_like(lse) if tw is None else tw.double(), 0.0)
    Z = float(wt.sum())
    wt = wt / Z if Z else wt * 0
    p = torch.exp(l - lse[:, None])
    qs = torch.zeros_like(p).scatter_add_(1, at, torch.where(there, q, 0.0))
    scale = (wt * tau)[:, None]
    d = (p - qs) * scale
    p_err = 3.4e-4 + 2.0 ** -12 + 2 * le[:, None]
    each = BF16 * d.abs() + (p_err * p + (2.0 ** -19 + 2.0 ** -22 * torch.where(live, z.abs(), zero).amax(1, keepdim=True)) * qs) * scale.abs()
    return dict(loss=(wt * token).sum(), token=token, t_err=t_err, lse=lse, le=le, counts=counts, wt=wt, d=d, each=each, h=h, w=w)


def check(torch, ops, h, w, z, index, tau=1.0, tw=None, out=None, ref=None):
    T, D = h.shape
    V = w.shape[0]
    ref = ref or reference(torch, h, w, z, index, tau, tw)
    kw = dict(temperature=tau, token_weight=tw)
    only, full = ops.linear_distillation(h, w, z, index, **kw), ops.linear_distillation_grad(h, w, z, index, **kw, **(out or {}))
    for r in (only, full):
        within(r.lse, ref["lse"], ref["le"] + 2.0 ** -22 * ref["lse"].abs())
        within(r.token_loss, ref["token"], ref["t_err"] + 2 * U * ref["token"].abs())
        assert bool((r.token_loss[~ref["counts"]] == 0).all())
        within(r.loss, ref["loss"], (ref["wt"].abs() * ref["t_err"]).sum() + 2.0 ** -22 * (ref["wt"].abs() * ref["token"].abs()).sum() + 1e-12)
    near = ref["d"].abs() + ref["each"]
    assert full.d_hidden.dtype == torch.bfloat16 and full.d_weight.dtype == torch.bfloat16
    dh, dw = ref["d"] @ ref["w"], ref["d"].T @ ref["h"]
    within(full.d_hidden, dh, (ref["each"] + sum_bound(V) * near) @ ref["w"].abs() * (1 + BF16) + (BF16 + 2.0 ** -22) * dh.abs() + 1e-30)
    within(full.d_weight, dw, (ref["each"] + sum_bound(T) * near).T @ ref["h"].abs() * (1 + BF16) + (BF16 + 2.0 ** -22) * dw.abs() + 1e-30)
    return full


def inputs(torch, T, V, D, K, seed, dtype=None, spread=1.5, empty=0.2, missing=0.1):
    """Columns at random, some of them twice; entries and whole rows missing."""
    g = gen(torch, seed)
    h = torch.randn(T, D, generator=g, device="cuda").bfloat16()
    w = (torch.randn(V, D, generator=g, device="cuda") * (spread / math.sqrt(D))).bfloat16()
    z = (2 * torch.randn(T, K, generator=g, device="cuda")).to(dtype or torch.float32)
    index = torch.randint(V, (T, K), generator=g, device="cuda")
    index[torch.rand(T, K, generator=g, device="cuda") < missing] = -1
    index[torch.rand(T, generator=g, device="cuda") < empty] = -7
    return h, w, z, index


SHAPES = [(1, 1, 8, 1), (1, 2, 16, 3), (2, 33, 64, 5), (1, 1000, 72, 8), (63, 100, 40, 64), (64, 128, 64, 1), (129, 129, 200, 33), (128, 257, 128, 100), (257, 256, 520, 7), (300, 4099, 136, 65),
          (31, 50257, 768, 50), (1, 32000, 768, 8), (513, 2050, 264, 16), (1030, 777, 768, 31), (2047, 1025, 8, 2), (70, 7, 32, 40), (40, 600, 64, 1024)]


@pytest.mark.parametrize("T,V,D,K", SHAPES)
@pytest.mark.parametrize("tau,weighted,dtype", [(1.0, False, "float32"), (2.0, True, "bfloat16"), (0.5, False, "bfloat16")])
def test_distillation_matches_definition(torch, ops, T, V, D, K, tau, weighted, dtype):
    h, w, z, index = inputs(torch, T, V, D, K, T * 7 + V + D, getattr(torch, dtype))
    tw = torch.rand(T, generator=gen(torch, 5), device="cuda") * 2 - 0.25 if weighted else None
    check(torch, ops, h, w, z, index, tau, tw)


@pytest.mark.parametrize("T,V,D,K", [(5, 7, 37, 3), (130, 300, 101, 20), (20, 129, 1, 9)])
def test_distillation_odd_widths(torch, ops, T, V, D, K):
    check(torch, ops, *inputs(torch, T, V, D, K, 3))


def test_distillation_crowded_columns(torch, ops):
    """Every row lists the same 256 columns (more entries in a segment than a warp has lanes), and every row one column 100 times."""
    T, V, D = 70, 900, 64
    h, w, _, _ = inputs(torch, T, V, D, 1, 1)
    z = torch.randn(T, 256, generator=gen(torch, 2), device="cuda")
    check(torch, ops, h, w, z, (torch.arange(256, device="cuda") + 100).expand(T, 256).contiguous())
    check(torch, ops, h, w, z[:, :100], torch.full((T, 100), 333, device="cuda"))
    lone = ops.linear_distillation_grad(h, w, z[:, :1], torch.full((T, 1), 333, device="cuda"))
    many = ops.linear_distillation_grad(h, w, torch.zeros(T, 128, device="cuda"), torch.full((T, 128), 333, device="cuda"))
    # 128 equal shares of one column are that column: the same gradient up to the rounding of their sum
    within(many.d_hidden, lone.d_hidden.double(), 2 * BF16 * lone.d_hidden.double().abs() + 2.0 ** -12 * lone.d_hidden.double().abs().amax())


def test_distillation_many_segments(torch, ops):
    """More segments of 128 columns than are counted at a time; columns at both ends."""
    T, V, D, K = 40, 600011, 16, 6
    h, w, z, index = inputs(torch, T, V, D, K, 11)
    index[0] = torch.tensor([0, V - 1, V - 2, 262143, 262144, 524288], device="cuda")
    check(torch, ops, h, w, z, index, 1.5)


@pytest.mark.parametrize("T,V,D,K", [(4500, 131072 - 5, 40, 5), (9000, 131072, 8, 3)])
def test_distillation_in_pieces_of_many_tokens(torch, ops, T, V, D, K):
    """More logits than the workspace holds at a time: two and three pieces."""
    h, w, z, index = inputs(torch, T, V, D, K, 13)
    tw = torch.rand(T, generator=gen(torch, 6), device="cuda")
    r, only = ops.linear_distillation_grad(h, w, z, index, 2.0, token_weight=tw), ops.linear_distillation(h, w, z, index, 2.0, token_weight=tw)
    counts = (index >= 0).any(1)
    total = float((tw.double() * counts).sum())
    dw, dw_bound, loss = torch.zeros(V, D, dtype=torch.float64, device="cuda"), torch.zeros(V, D, dtype=torch.float64, device="cuda"), 0.0
    for a in range(0, T, 1500):
        s = slice(a, min(T, a + 1500))
        ref = reference(torch, h[s], w, z[s], index[s], 2.0, tw[s])
        share = float((tw[s].double() * counts[s]).sum()) / total              # of these rows in the mean
        d, each = ref["d"] * share, ref["each"] * share
        for t in (r, only):
            within(t.lse[s], ref["lse"], ref["le"] + 2.0 ** -22 * ref["lse"].abs())
            within(t.token_loss[s], ref["token"], ref["t_err"] + 2 * U * ref["token"].abs())
        dh = d @ ref["w"]
        within(r.d_hidden[s], dh, (each + sum_bound(V) * (d.abs() + each)) @ ref["w"].abs() * (1 + BF16) + (BF16 + 2.0 ** -22) * dh.abs() + 1e-30)
        dw += d.T @ ref["h"]
        dw_bound += (each + sum_bound(T) * (d.abs() + each)).T @ ref["h"].abs()
        loss += share * float(ref["loss"])
        del ref, d, each, dh
    within(r.d_weight, dw, dw_bound * (1 + BF16) + (BF16 + 2.0 ** -20) * dw.abs() + 1e-30)
    assert abs(float(r.loss) - loss) < 1e-4 and abs(float(only.loss) - loss) < 1e-4


def test_distillation_of_one_entry_is_the_cross_entropy(torch, ops):
    T, V, D = 300, 1000, 128
    h, w, z, index = inputs(torch, T, V, D, 1, 4, missing=0.0)
    labels = torch.where(index[:, 0] < 0, -100, index[:, 0])
    a, b = ops.linear_distillation_grad(h, w, z, index), ops.linear_cross_entropy_grad(h, w, labels)
    assert torch.equal(a.lse, b.lse)
    within(a.token_loss, b.token_loss.double(), 2.0 ** -21 * (b.token_loss.double().abs() + b.lse.double().abs()))
    within(a.loss, b.loss.double(), 2.0 ** -20 * b.loss.double().abs() + 1e-6)
    for x, y in ((a.d_hidden, b.d_hidden), (a.d_weight, b.d_weight)):          # the entry's p - 1 in another order: rarely another bfloat16
        within(x, y.double(), 2 * BF16 * y.double().abs() + 2.0 ** -10 * y.double().abs().amax())


def test_distillation_from_itself(torch, ops):
    """A teacher who lists every column with the student's own logits: no distance, no gradient beyond the logits' errors."""
    T, V, D = 50, 100, 64
    h, w, _, _ = inputs(torch, T, V, D, 1, 5)
    z = (h.double() @ w.double().T).float()
    check(torch, ops, h, w, z, torch.arange(V, device="cuda").expand(T, V).contiguous())


def test_distillation_no_entries_and_no_tokens(torch, ops):
    h, w, z, index = inputs(torch, 40, 300, 64, 5, 1)
    for z2, i2 in ((z, torch.full_like(index, -1)), (torch.full_like(z, -math.inf), index.abs())):
        r = ops.linear_distillation_grad(h, w, z2, i2)
        assert float(r.loss) == 0 and not r.token_loss.any() and not r.d_hidden.any() and not r.d_weight.any()
        within(r.lse, torch.logsumexp(h.double() @ w.double().T, 1), torch.full((40,), 1e-4, dtype=torch.float64, device="cuda"))
        assert float(ops.linear_distillation(h, w, z2, i2).loss) == 0
    r = ops.linear_distillation_grad(h[:0], w, z[:0], index[:0])
    assert float(r.loss) == 0 and r.token_loss.shape == (0,) and r.d_hidden.shape == (0, 64) and not r.d_weight.any() and r.d_weight.shape == (300, 64)
    assert float(ops.linear_distillation(h[:0], w, z[:0], index[:0]).loss) == 0


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_distillation_masks(torch, ops, dtype):
    """What stands at a masked place does not matter (NaN, infinities, columns that do not exist); the type's lowest value is a probability of 0, alone it is 1."""
    T, V, D, K = 60, 500, 64, 12
    h, w, z, index = inputs(torch, T, V, D, K, 6, getattr(torch, dtype), empty=0.0, missing=0.0)
    masked = torch.rand(T, K, generator=gen(torch, 7), device="cuda") < 0.3
    masked[:, 0] = False
    bare = index.masked_fill(masked, -1)
    want = ops.linear_distillation_grad(h, w, z, bare)
    check(torch, ops, h, w, z, bare)
    for value in (float("nan"), float("inf"), -float("inf"), 3e38):
        got = ops.linear_distillation_grad(h, w, z.masked_fill(masked, value), bare)
        for a, b in zip(got, want):
            assert torch.equal(a, b)
    got = ops.linear_distillation_grad(h, w, z.masked_fill(masked, -float("inf")), index.masked_fill(masked, 10 ** 12))
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    low = torch.finfo(z.dtype).min
    got = ops.linear_distillation_grad(h, w, z.masked_fill(masked, low), index)
    for a, b in zip(got[:3], want[:3]):
        assert torch.equal(a, b)
    lows = torch.full_like(z, low)
    check(torch, ops, h, w, torch.zeros_like(z), index)
    for a, b in zip(ops.linear_distillation_grad(h, w, lows, index), ops.linear_distillation_grad(h, w, torch.zeros_like(z), index)):
        assert torch.equal(a, b)


def test_distillation_not_finite(torch, ops):
    """A NaN or an infinity of the teacher's or of a hidden state stays in its row; a row without an entry is left out."""
    T, V, D, K = 300, 700, 64, 9
    h, w, z, index = inputs(torch, T, V, D, K, 8, empty=0.0, missing=0.0)
    h2, z2 = h.clone(), z.clone()
    h2[3, 5], z2[100, 2], z2[270, 0], z2[271] = float("nan"), float("nan"), float("inf"), float("nan")
    bad = torch.zeros(T, dtype=torch.bool, device="cuda")
    bad[[3, 100, 270, 271]] = True
    for r in (ops.linear_distillation(h2, w, z2, index), ops.linear_distillation_grad(h2, w, z2, index)):
        assert torch.equal(torch.isnan(r.token_loss), bad) and bool(torch.isnan(r.loss))
    assert torch.equal(torch.isnan(r.d_hidden).all(1), bad) and torch.equal(torch.isnan(r.d_hidden).any(1), bad)
    i2 = index.clone()
    i2[bad] = -1
    r = ops.linear_distillation_grad(h2, w, z2, i2)
    keep = ~bad
    ref = reference(torch, h[keep], w, z[keep], index[keep], 1.0, None)
    assert abs(float(r.loss) - float(ref["loss"])) < 1e-4 and bool((r.d_hidden[bad] == 0).all()) and bool((r.token_loss[bad] == 0).all())


def test_distillation_extreme_logits(torch, ops):
    """Columns far above and thousands below, rows of equal logits; a listed column of probability 0 is infinitely far, unless the teacher's is 0 too."""
    T, V, D, K = 70, 513, 64, 10
    h, w, z, index = inputs(torch, T, V, D, K, 2, empty=0.0)
    h[:20] *= 64
    w[300] *= 16
    h[20:30] = 0
    check(torch, ops, h, w, z, index, 1.0)
    check(torch, ops, h, w, z * 30, index, 4.0)
    h2, w2 = torch.zeros_like(h), torch.zeros_like(w)
    h2[:, 0] = 1
    w2[:, 0] = -3e38
    w2[5, 0] = w2[400, 0] = 1
    r = ops.linear_distillation_grad(h2, w2, torch.zeros(T, 2, device="cuda"), torch.tensor([[5, 400]], device="cuda").expand(T, 2).contiguous())
    assert not r.token_loss.any() and not r.d_weight.any()
    r = ops.linear_distillation(h2 * 4, w2 * 1, torch.tensor([[0.0, -1e6]], device="cuda").expand(T, 2).contiguous(), torch.tensor([[5, 6]], device="cuda").expand(T, 2).contiguous())
    assert torch.allclose(r.token_loss, torch.full((T,), math.log(2.0), device="cuda"), rtol=1e-6)


def test_distillation_bad_index_is_reported(torch, ops):
    T, V, D, K = 20, 100, 64, 4
    h, w, z, index = inputs(torch, T, V, D, K, 6, empty=0.0, missing=0.0)
    ok = index.clone()
    index[4, 2], index[9, 0] = V, 1 << 40
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    r = ops.linear_distillation_grad(h, w, z, index, status=status)
    assert int(status) == ops.PSGD_W_LABEL
    assert torch.equal(torch.isnan(r.token_loss).nonzero()[:, 0].cpu(), torch.tensor([4, 9])) and bool(torch.isnan(r.loss))
    assert not r.d_hidden[4].any() and not r.d_hidden[9].any() and bool(torch.isfinite(r.d_weight).all())
    assert bool(torch.isnan(ops.linear_distillation(h, w, z, index).loss))
    status.zero_()
    ops.linear_distillation_grad(h, w, z, ok, status=status)
    assert int(status) == 0


def test_distillation_strides_slots_and_streams(torch, ops):
    T, V, D, K = 260, 520, 200, 11
    h, w, z, index = inputs(torch, T, V, D, K, 8)
    ref = reference(torch, h, w, z, index, 1.0, None)
    nan = float("nan")
    wide_h, wide_w = torch.full((T, D + 24), nan, device="cuda", dtype=torch.bfloat16), torch.full((V, D + 9), nan, device="cuda", dtype=torch.bfloat16)
    wide_h[:, 8:8 + D], wide_w[:, 3:3 + D] = h, w
    wide_z, wide_i = torch.full((T, K + 5), nan, device="cuda"), torch.full((T, K + 3), 1 << 50, device="cuda")
    wide_z[:, 2:2 + K], wide_i[:, 1:1 + K] = z, index
    G = torch.full((2, 3, V, D), 7.0, device="cuda", dtype=torch.bfloat16)
    dh = torch.full((T, D + 5), 7.0, device="cuda", dtype=torch.bfloat16)
    check(torch, ops, wide_h[:, 8:8 + D], wide_w[:, 3:3 + D], wide_z[:, 2:2 + K], wide_i[:, 1:1 + K], out=dict(d_weight=G[1, 2], d_hidden=dh[:, 2:2 + D]), ref=ref)
    assert bool((dh[:, :2] == 7).all()) and bool((dh[:, 2 + D:] == 7).all()) and bool((G.view(6, -1)[:5] == 7).all())
    plain = ops.linear_distillation_grad(h, w, z, index)
    assert torch.equal(plain.d_weight, G[1, 2]) and torch.equal(plain.d_hidden, dh[:, 2:2 + D])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        x = h * 1
    r = ops.linear_distillation_grad(x, w, z, index, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    for a, b in zip(r, plain):
        assert torch.equal(a, b)
    for bad in (dict(d_hidden=h), dict(d_weight=w)):
        with pytest.raises(ops.PSGDError):
            ops.linear_distillation_grad(h, w, z, index, **bad)


def test_distillation_gradient_by_differences(torch, ops):
    """Central differences of the kernel's own loss, as for the cross entropy: a step of 2^-4 in one entry moves a logit over the temperature by at most 2^-4; the gradient carries the
    temperature once, the loss twice."""
    T, V, D, K, tau = 6, 40, 16, 5, 2.0
    g = gen(torch, 9)
    h = (torch.randint(-8, 9, (T, D), generator=g, device="cuda") / 8).bfloat16()
    w = (torch.randint(-8, 9, (V, D), generator=g, device="cuda") / 8).bfloat16()
    z, index = torch.randn(T, K, generator=g, device="cuda"), torch.randint(V, (T, K), generator=g, device="cuda")
    r = ops.linear_distillation_grad(h, w, z, index, tau)
    step = 2.0 ** -4
    for which, at in [("h", (0, 0)), ("h", (3, 7)), ("h", (5, 15)), ("w", (0, 0)), ("w", (int(index[2, 1]), 3)), ("w", (39, 15))]:
        loss = []
        for sign in (1, -1):
            a = {"h": h.clone(), "w": w.clone()}
            a[which][at] += sign * step
            loss.append(float(ops.linear_distillation(a["h"], a["w"], z, index, tau).loss))
        grad = float((r.d_hidden if which == "h" else r.d_weight)[at])
        assert abs((loss[0] - loss[1]) / (2 * step) - grad) <= tau * step ** 2 / 6 + tau ** 2 * 2.0 ** -20 / step + 0.01 * abs(grad) + 1e-4


@pytest.mark.parametrize("base", [-60, 0, 60])
def test_distillation_of_tokens_that_both_are_sure_of(torch, ops, base):
    """Teacher and student both within 1e-3 to 1e-5 of certainty about one column, at logits of any size: the distance and the column's gradient are good relative to that.

    Every token has a column of its own that lifts it, so d_hidden[t, own column] is the gradient of that column's logit alone.  Bounds: a logit is good to l_err,
    which moves 1 - p by 2 l_err of itself; sums and e_p, e_q meet at most 10 roundings of 2^-24, the teacher's exponentials 2^-20 of their size; two roundings to bfloat16.
    """
    T, D, V, K = 24, 64, 700, 6
    g = gen(torch, 70 + base)
    h, w = torch.zeros(T, D, device="cuda"), torch.zeros(V, D, device="cuda")
    own, rows = torch.arange(1, T + 1, device="cuda"), torch.arange(T, device="cuda")
    h[:, T + 1:] = torch.randn(T, D - T - 1, generator=g, device="cuda") * 0.15
    w[:, T + 1:] = torch.randn(V, D - T - 1, generator=g, device="cuda")
    sure = torch.randperm(V, generator=g, device="cuda")[:T]
    h[:, 0], w[:, 0] = base, 1
    rest = 10.0 ** -torch.linspace(3, 5, T, device="cuda")
    h[rows, own] = math.log(V) + 0.4 - torch.log(rest)
    w[sure, own] = 1
    w[sure, T + 1:] = 0
    h, w = h.bfloat16(), w.bfloat16()
    index = torch.stack([sure] + [(sure + 1 + 7 * k) % V for k in range(K - 1)], 1)
    z = torch.log(rest.flip(0))[:, None] - math.log(K - 1) + torch.randn(T, K, generator=g, device="cuda") * 0.3
    z[:, 0] = 0
    ref = reference(torch, h, w, z, index, 1.0, None)
    hd, wd = h.double(), w.double()
    miss_p = -torch.expm1(hd[rows] @ wd.T - ref["lse"][:, None])[rows, sure]
    zd = z.double()
    miss_q = torch.exp(zd[:, 1:]).sum(1) / (1 + torch.exp(zd[:, 1:]).sum(1))
    assert bool(((miss_p > 3e-6) & (miss_p < 3e-3) & (miss_q > 3e-6) & (miss_q < 3e-3)).all())
    l_err = sum_bound(D) * (hd.abs() @ wd.abs().T).amax(1)
    off = 2 * l_err * miss_p + 10 * U + 2.0 ** -20 * (miss_p + miss_q)
    r = ops.linear_distillation_grad(h, w, z, index)
    grad = miss_q - miss_p                                               # p - q
    within(r.d_hidden[rows, own] * T, grad, off * (1 + 2 * BF16) + (2 * BF16 + 2.0 ** -20) * grad.abs())
    # the distance: near 1 log q - log p is miss_p - miss_q; the others' terms q (log q - log p) with q up to 1e-3, their logs of size 20
    others = torch.exp(zd[:, 1:]).sum(1)
    for t in (r, ops.linear_distillation(h, w, z, index)):
        within(t.token_loss, ref["token"], off + others * (2 * l_err + (20 + abs(base)) * 2.0 ** -20) + 2.0 ** -21 * ref["token"].abs())


# ---- streams, graphs, warnings, waits -----------------------------------------------------------------------------
def test_distillation_repeats_bit_for_bit(torch, ops):
    args = inputs(torch, 1000, 5000, 512, 64, 12)
    a, b = (ops.linear_distillation_grad(*args) for _ in range(2))
    for x, y in zip(a, b):
        assert torch.equal(x, y)


def test_distillation_in_a_cuda_graph(torch, ops):
    args = inputs(torch, 300, 1100, 200, 20, 31)

    def work():
        return [*ops.linear_distillation_grad(*args), *ops.linear_distillation(*args, 2.0)]

    work()
    torch.cuda.synchronize()
    graphs, outs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()], []
    for i, g in enumerate(graphs):
        with torch.cuda.graph(g, pool=graphs[0].pool() if i else None):
            outs.append(work())
    for t, u in zip(args, inputs(torch, 300, 1100, 200, 20, 33)):
        t.copy_(u)
    want = work()
    for g, out in zip(graphs, outs):
        for t in out:
            t.fill_(7)
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b)


def test_distillation_on_two_streams_and_with_inputs_freed(torch, ops):
    sets = [inputs(torch, 700, 3000, 256, 30, s) for s in (21, 22)]
    want = [ops.linear_distillation_grad(*s) for s in sets]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[ops.linear_distillation_grad(*sets[i], stream=streams[i]) for i in (0, 1)] for _ in range(5)]
    torch.cuda.synchronize()
    for both in got:
        for a, b in zip(both, want):
            for u, v in zip(a, b):
                assert torch.equal(u, v)
    mine = [t.clone() for t in sets[0]]
    streams[0].wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(streams[0]):
        torch.cuda._sleep(20_000_000)
    late = ops.linear_distillation_grad(*mine, stream=streams[0])
    sizes = [(t.shape, t.dtype) for t in mine]
    del mine
    torch.cuda.current_stream().synchronize()
    others = [torch.full(shape, 3, dtype=dtype, device="cuda") for shape, dtype in sizes for _ in range(4)]
    torch.cuda.synchronize()
    assert len(others) == 16
    for a, b in zip(late, want[0]):
        assert torch.equal(a, b)


def test_distillation_warns_and_refuses(torch, ops):
    h, w, z, index = inputs(torch, 40, 90, 64, 5, 71)
    leaf = h.clone().requires_grad_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for call in (lambda: ops.linear_distillation(leaf, w, z, index), lambda: ops.linear_distillation(h, w.clone().requires_grad_(), z, index, stream=side)):
        with pytest.warns(UserWarning, match="linear_distillation: the results have no autograd graph") as seen:
            call()
        assert len(seen) == 1 and seen[0].filename == __file__
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        ops.linear_distillation_grad(leaf, w, z, index)
        with torch.no_grad():
            ops.linear_distillation(leaf, w, z, index)
    torch.cuda.synchronize()
    bad = [lambda: ops.linear_distillation(h, w, z[:, :4], index), lambda: ops.linear_distillation(h, w, z[:39], index[:39]), lambda: ops.linear_distillation(h, w, z, index.int()),
           lambda: ops.linear_distillation(h, w, z.half(), index), lambda: ops.linear_distillation(h, w, z, index, 0.0), lambda: ops.linear_distillation(h, w, z, index, -1.0),
           lambda: ops.linear_distillation(h, w, z, index, float("nan")), lambda: ops.linear_distillation(h, w, z.cpu(), index), lambda: ops.linear_distillation(h, w, z, index.cpu()),
           lambda: ops.linear_distillation(h, w, z.expand(2, 40, 5)[0].T, index), lambda: ops.linear_distillation(h, w, z[:, :0], index[:, :0]),
           lambda: ops.linear_distillation_grad(h, w, torch.zeros(40, 1025, device="cuda"), torch.zeros(40, 1025, dtype=torch.int64, device="cuda")),
           lambda: ops.linear_distillation_grad(h.float(), w, z, index), lambda: ops.linear_distillation_grad(h, w, z, index, token_weight=z[:, 0])]
    for call in bad:
        with pytest.raises(ops.PSGDError):
            call()


def test_distillation_refuses_gradients_over_its_lists(torch, ops):
    h, w, z, index = inputs(torch, 40, 90, 64, 64, 72)
    z = z.bfloat16().contiguous()
    over = index.view(torch.bfloat16)                  # (40, 256)
    for out in ({"d_hidden": z}, {"d_hidden": over[:, 64:128]}, {"d_weight": torch.as_strided(over, (90, 64), (64, 1))}):
        for status in (None, torch.zeros(1, dtype=torch.int32, device="cuda")):
            with pytest.raises(ops.PSGDError):
                ops.linear_distillation_grad(h, w, z, index, status=status, **out)


@pytest.mark.parametrize("T", [1, 2])
@pytest.mark.parametrize("V,D,K", [(1, 8, 1), (33, 1, 3), (127, 37, 5), (128, 64, 40), (129, 100, 7), (5000, 768, 64), (700, 2051, 300), (300, 16384, 9), (300, 16392, 9), (4000, 4096, 16), (4001, 8, 1024)])
def test_distillation_of_one_token(torch, ops, T, V, D, K):
    """The loss alone goes without tiles (up to a width of 16384), the gradients and two tokens by them; every kind of row end, a vocabulary that ends inside a segment."""
    h, w, z, index = inputs(torch, T, V, D, K, T + V + D, spread=1.0, empty=0.0)
    check(torch, ops, h, w, z, index, 1.5)
    wide_h, wide_w = torch.full((T, D + 24), float("nan"), device="cuda", dtype=torch.bfloat16), torch.full((V, (D + 7) // 8 * 8 + 8), float("nan"), device="cuda", dtype=torch.bfloat16)
    wide_h[:, 8:8 + D], wide_w[:, 8:8 + D] = h, w                        # NaN on both sides of every row
    a, b = ops.linear_distillation(h, w, z, index), ops.linear_distillation(wide_h[:, 8:8 + D], wide_w[:, 8:8 + D], z, index)
    for u, v in zip(a, b):
        assert torch.equal(u, v)


def test_distillation_behind_a_wait_that_ran_out_is_nan(torch, ops, tmp_path, monkeypatch):
    """A build whose epilogue gives up every wait for an accumulator at once (no pair has more than two accumulators here, so nothing waits for the epilogue in turn): every
    result is NaN, and the status word says why.  (Calls with a status word take the long way, through the library that is put in its place.)"""
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
    h, w, z, index = inputs(torch, 300, 700, 64, 9, 3)
    monkeypatch.setattr(binding, "_lib", L)
    counts = (index >= 0).any(1)
    for call in (ops.linear_distillation, ops.linear_distillation_grad):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        r = call(h, w, z, index, 2.0, status=status)
        assert int(status) == ops.PSGD_W_TIMEOUT
        assert bool(torch.isnan(r.loss)) and bool(torch.isnan(r.lse).all()) and bool(torch.isnan(r.token_loss[counts]).all())
    assert bool(torch.isnan(r.d_hidden).all()) and bool(torch.isnan(r.d_weight).all())
