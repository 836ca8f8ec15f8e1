"""Layer norm, rotary positions and distillation where calls are unusual: frequencies that are not finite, tensors that autograd has saved, rows beyond registers in numbers,
long lists over many tokens.  Bounds count roundings as in the operators' other tests, u = 2^-24."""
import math

import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF_STEP = {"bfloat16": 2.0 ** -8, "float32": U}


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


def within(got, ref, bound):
    d = (got.double() - ref).abs()
    assert bool((d <= bound).all()), f"worst error / bound {float((d / bound.clamp(min=1e-300)).max()):.3g}"


# ---- rotary positions ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("R", [32, 34])
def test_rotary_frequencies_that_are_not_finite(torch, ops, layout, dtype, R):
    """A frequency that is NaN or infinite has no angle at any position: its pair is NaN in every token, even at position 0, and no other value changes."""
    g = gen(torch, R)
    q, k = (torch.randn(6, heads, 40, generator=g, device="cuda").to(getattr(torch, dtype)) for heads in (3, 1))
    positions = torch.tensor([0, 1, 2, -5, 1 << 20, 7], device="cuda")
    f = ops.rotary_frequencies(R)
    odd = f.clone()
    odd[3], odd[9], odd[R // 2 - 1] = math.nan, math.inf, -math.inf
    bad = torch.zeros(40, dtype=torch.bool, device="cuda")
    for i in (3, 9, R // 2 - 1):
        bad[[i, i + R // 2] if layout == "half" else [2 * i, 2 * i + 1]] = True
    for call in (ops.rotary_forward, ops.rotary_backward):
        for in_place in (False, True):
            got = call(q.clone(), k.clone(), positions, odd, layout=layout, in_place=in_place)
            for x, y in zip(got, call(q, k, positions, f, layout=layout)):
                assert bool(torch.isnan(x[..., bad]).all()) and torch.equal(x[..., ~bad], y[..., ~bad])


@pytest.mark.parametrize("other_stream", [False, True])
def test_rotary_in_place_is_seen_by_autograd(torch, ops, other_stream):
    """What another operator has saved for its gradients and is turned in place raises there, as behind any operator that works in place; calls that write nothing into their
    inputs, or that are refused, leave them as they are."""
    g = gen(torch, 1)
    side = torch.cuda.Stream() if other_stream else None
    positions, f = torch.arange(5, device="cuda"), ops.rotary_frequencies(16)
    for call in (ops.rotary_forward, ops.rotary_backward):
        for which in (0, 1):
            both = [torch.randn(5, heads, 24, generator=g, device="cuda") for heads in (4, 2)]
            leaf = torch.randn_like(both[which]).requires_grad_()
            y = (leaf * both[which]).sum()
            before = [t._version for t in both]
            call(*both, positions, f, stream=side)
            assert [t._version for t in both] == before
            call(*both, positions, f, in_place=True, stream=side)
            assert all(t._version > v for t, v in zip(both, before))
            torch.cuda.synchronize()
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                y.backward()
    packed = torch.randn(5, 6, 24, generator=g, device="cuda")
    before = packed._version
    ops.rotary_forward(packed[:, :4], packed[:, 4:], positions, f, in_place=True, stream=side)
    assert packed._version > before                    # (a view's base)
    before = packed._version
    with pytest.raises(ops.PSGDError):
        ops.rotary_forward(packed[:, :4], packed[:, 3:], positions, f, in_place=True, stream=side)
    assert packed._version == before
    with torch.inference_mode():
        x = torch.randn(5, 4, 24, generator=g, device="cuda")
    want = ops.rotary_forward(x, None, positions, f)[0]
    assert torch.equal(ops.rotary_forward(x, None, positions, f, in_place=True, stream=side)[0].clone(), want)      # (has no version)
    torch.cuda.synchronize()


def test_results_in_the_callers_tensors_are_seen_by_autograd(torch, ops):
    """`out`, `d_hidden` and `d_weight` are tensors of the caller's: what has saved them for its gradients has to know."""
    T, D, V, K = 40, 64, 90, 5
    g = gen(torch, 2)
    h, w = torch.randn(T, D, generator=g, device="cuda").bfloat16(), torch.randn(V, D, generator=g, device="cuda").bfloat16()
    z, index = torch.randn(T, K, generator=g, device="cuda"), torch.randint(V, (T, K), generator=g, device="cuda")
    kept = ops.pack_activation(h)
    G = torch.zeros(2, V, D, device="cuda", dtype=torch.bfloat16)      # a stack, of which a slot is written
    for side in (None, torch.cuda.Stream()):
        for shape, write in (((T, D), lambda t: ops.linear_distillation_grad(h, w, z, index, d_hidden=t, stream=side)), ((V, D), lambda t: ops.linear_distillation_grad(h, w, z, index, d_weight=t, stream=side)),
                             ((T, D), lambda t: ops.linear_cross_entropy_grad(h, w, index[:, 0].contiguous(), d_hidden=t, stream=side)),
                             ((V, D), lambda t: ops.linear_cross_entropy_grad(h, w, index[:, 0].contiguous(), d_weight=t, stream=side)),
                             ((D, D), lambda t: ops.weight_gradient(h, kept, out=t, stream=side)), ((T, D), lambda t: kept.unpack(out=t, stream=side))):
            torch.cuda.synchronize()
            t = torch.zeros(shape, device="cuda", dtype=torch.bfloat16)
            y = (torch.ones_like(t).requires_grad_() * t).sum()
            write(t)
            torch.cuda.synchronize()
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                y.backward()
        before = G._version
        ops.linear_distillation_grad(h, w, z, index, d_weight=G[1], stream=side)
        assert G._version > before
        with torch.inference_mode():
            t = torch.zeros(T, D, device="cuda", dtype=torch.bfloat16)
        kept.unpack(out=t, stream=side)                # (has no version)
    torch.cuda.synchronize()


def test_rotary_angles_carry_the_precision_of_float32(torch, ops):
    """(1, 0) turned is (cos a, sin a), without a rounding of its own.  The angle's distance from the nearest quarter of a turn, at most 1/8, is held in float32: within 2^-28 of a
    turn; beside it four roundings of position * frequency in float64 (the reference makes some of them), and one unit in the last place of the sine and the cosine (2^-24
    where they are largest)."""
    g = gen(torch, 3)
    T, R = 4096, 64
    positions = torch.randint(1 << 17, (T,), generator=g, device="cuda")
    f = ops.rotary_frequencies(R)
    x = torch.zeros(T, 1, R, device="cuda")
    x[..., :R // 2] = 1
    angle = positions.double()[:, None] * f
    bound = 2 * math.pi * 2.0 ** -28 + 4 * angle.abs() * 2.0 ** -53 + 2.0 ** -24
    for call, way in ((ops.rotary_forward, 1), (ops.rotary_backward, -1)):
        got = call(x, None, positions, f)[0][:, 0]
        within(got[:, :R // 2], torch.cos(angle), bound)
        within(got[:, R // 2:], way * torch.sin(angle), bound)
    # whole quarters, and the angles beside the places where the nearest quarter changes (1/8, 3/8, 5/8, 7/8 of a turn)
    steps = torch.arange(-64, 65, device="cuda")
    eighth = torch.tensor([2 * math.pi / 1024], dtype=torch.float64, device="cuda")
    at = torch.cat([steps + 128 * i for i in range(-9, 10)])
    x = torch.zeros(len(at), 1, 2, device="cuda")
    x[..., 0] = 1
    got = ops.rotary_forward(x, None, at, eighth)[0][:, 0]
    turn = at.double() / 1024 * 2 * math.pi
    bound = torch.full_like(turn, 2 * math.pi * 2.0 ** -28 + 2.0 ** -24) + 4 * turn.abs() * 2.0 ** -53
    within(got[:, 0], torch.cos(turn), bound)
    within(got[:, 1], torch.sin(turn), bound)
    quarter = at % 256 == 0
    assert int(quarter.sum()) >= 9
    whole = torch.stack([torch.cos(turn), torch.sin(turn)], 1)[quarter].round().float()
    assert bool(((got[quarter] - whole).abs() <= 2.0 ** -40).all())


# ---- layer norm ---------------------------------------------------------------------------------------------------
def check_norm(torch, ops, T, F, x_type, y_type=None, extra=False, center=True, bias=True, rows=500):
    """Both directions against 64 bits, a few hundred rows at a time; a sum over F values passes each through at most 40 + F / 4096 additions, one over T rows through at
    most T / 128 + 65."""
    dtype, out_type = getattr(torch, x_type), getattr(torch, y_type or x_type)
    g = gen(torch, T + F)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    w, b = 1 + 0.3 * normal(F), 0.2 * normal(F) if bias else None
    x, dy = (normal(T, F) + 0.3 * normal(F)).to(dtype), (1e-2 * normal(T, F)).to(out_type)
    r, d_x = (normal(T, F).to(dtype), (1e-2 * normal(T, F)).to(dtype)) if extra else (None, None)
    n = ops.layer_norm_forward(x, w, b, residual=r, center=center, keep=True, dtype=out_type)
    d = ops.layer_norm_backward(dy, n.x, w, n.mean, n.rstd, d_x=d_x, bias=bias)
    assert n.y.dtype == out_type and d.d_x.dtype == dtype
    again = ops.pack_activation(n.y)
    assert torch.equal(n.kept.q, again.q) and torch.equal(n.kept.scales, again.scales)
    depth, wd, bd = 40 + F / 4096, w.double(), b.double() if bias else 0.0
    dw, dw_size, db, db_size = (torch.zeros(F, dtype=torch.float64, device="cuda") for _ in range(4))
    for a in range(0, T, rows):
        p = slice(a, a + rows)
        s = x[p] if r is None else (x[p].float() + r[p].float()).to(dtype)
        assert torch.equal(n.x[p], s)
        s = s.double()
        mean = s.mean(1, keepdim=True) if center else torch.zeros_like(s[:, :1])
        em = (depth + 1) * U * s.abs().mean(1, keepdim=True) if center else 0.0 * mean
        v = s - mean
        var = v.square().mean(1, keepdim=True) + 1e-5
        rstd = var.rsqrt()
        er = ((depth + 4) * U + em ** 2 / var + 4 * U) / 2 + 2.0 ** -22
        if center:
            within(n.mean[p, None], mean, em + U * mean.abs() + 1e-40)
        within(n.rstd[p, None], rstd, er * rstd)
        y = v * rstd * wd + bd
        step = HALF_STEP[y_type or x_type]
        within(n.y[p], y, (em * rstd + (er + 6 * U) * (v * rstd).abs()) * wd.abs() * (1 + 1e-3) * (1 + step) + (step + 2 * U) * y.abs() + 1e-38)
        # the gradients of the statistics that the forward pass returned
        f, m = n.rstd[p, None].double(), n.mean[p, None].double() if center else 0.0
        xh, e = (s - m) * f, dy[p].double()
        dw += (e * xh).sum(0)
        dw_size += (e * xh).abs().sum(0)
        db += e.sum(0)
        db_size += e.abs().sum(0)
        e = e * wd
        c1, c2 = e.mean(1, keepdim=True) if center else 0.0, (e * xh).mean(1, keepdim=True)
        e1, e2 = (depth + 3) * U * e.abs().mean(1, keepdim=True), (depth + 6) * U * (e * xh).abs().mean(1, keepdim=True)
        dx = f * (e - c1 - xh * c2)
        bound = f * (8 * U * (e.abs() + (xh * c2).abs() + abs(c1)) + e1 + xh.abs() * e2)
        if d_x is not None:
            dx = dx + d_x[p].double()
            bound = bound + U * (dx.abs() + d_x[p].double().abs())
        step = HALF_STEP[x_type]
        within(d.d_x[p], dx, bound * (1 + step) + (step + 2 * U) * dx.abs() + 1e-38)
    within(d.d_weight, dw, (T / 128 + 68) * U * dw_size + 1e-38)
    if bias:
        within(d.d_bias, db, (T / 128 + 65) * U * db_size + 1e-38)


@pytest.mark.parametrize("T,F,x_type,y_type,extra", [(2000, 4099, "float32", None, True), (1500, 4099, "float32", "bfloat16", False), (700, 10001, "float32", None, False),
                                                     (700, 10001, "float32", "bfloat16", True), (1300, 16640, "bfloat16", None, True), (700, 16391, "bfloat16", None, False), (700, 12800, "float32", None, True),
                                                     (1200, 12288, "float32", "bfloat16", True), (650, 16640, "float32", None, False), (60, 131072, "bfloat16", None, True)])
@pytest.mark.parametrize("center", [True, False])
def test_norm_many_rows_beyond_registers(torch, ops, T, F, x_type, y_type, extra, center):
    """More rows than CTAs where a CTA walks over its row several times: every one takes a second row and a third, and the columns' sums go over several."""
    check_norm(torch, ops, T, F, x_type, y_type, extra, center, bias=center)


@pytest.mark.parametrize("T,F,gap", [(1300, 5003, 3), (700, 4100, 2)])
def test_norm_many_rows_beyond_registers_that_lie_unlike(torch, ops, T, F, gap):
    """Bfloat16 rows whose operands lie at different places within 16 bytes: the same values as those of copies that lie alike, to one rounding of the result."""
    g = gen(torch, F)
    x, dy = (torch.randn(T, F + gap, generator=g, device="cuda").bfloat16()[:, 1:F + 1] for _ in range(2))
    r = torch.randn(T, F, generator=g, device="cuda").bfloat16()
    w, b = 1 + 0.3 * torch.randn(F, generator=g, device="cuda"), 0.2 * torch.randn(F, generator=g, device="cuda")
    n, m = (ops.layer_norm_forward(t, w, b, residual=r, keep=True) for t in (x, x.contiguous()))
    d, e = (ops.layer_norm_backward(t, n.x, w, n.mean, n.rstd, d_x=r, bias=True) for t in (dy, dy.contiguous()))
    assert torch.equal(n.x, m.x)
    for a, c in ((n.y, m.y), (d.d_x, e.d_x)):
        within(a, c.double(), 2 * 2.0 ** -8 * c.double().abs() + 1e-5)
    depth = 40 + F / 4096
    within(n.mean, m.mean.double(), 2 * (depth + 2) * U * n.x.double().abs().mean(1))
    within(n.rstd, m.rstd.double(), ((depth + 8) * U + 2.0 ** -21) * m.rstd.double())
    xh = ((n.x.double() - n.mean.double()[:, None]) * n.rstd.double()[:, None] * dy.double()).abs().sum(0)
    within(d.d_weight, e.d_weight.double(), 2 * (T / 128 + 68) * U * xh)
    within(d.d_bias, e.d_bias.double(), 2 * (T / 128 + 65) * U * dy.double().abs().sum(0))


@pytest.mark.parametrize("T,F,term", [(4000, 262144, 1.0041199), (8000, 131072, 1.2795105)])
def test_norm_sums_over_many_wide_rows(torch, ops, T, F, term):
    """Sums over rows pass every value through at most T / 128 + 65 additions however wide the rows are.  Equal terms are the worst of sums, since all additions of a stretch round
    the same way; with these two, one running sum of a thread's rows (1000 and 889 of them) would be off by 2.6 and 1.7 times the bound."""
    x, dy = torch.ones(T, F, device="cuda"), torch.full((T, F), term, device="cuda")
    # without centring and with a rstd of 1, dy xh is dy
    d = ops.layer_norm_backward(dy, x, torch.ones(F, device="cuda"), None, torch.ones(T, device="cuda"), bias=True)
    want = torch.full((F,), T * float(dy[0, 0]), dtype=torch.float64, device="cuda")
    for got in (d.d_bias, d.d_weight):
        within(got, want, (T / 128 + 65) * U * want)


# ---- distillation -------------------------------------------------------------------------------------------------
def test_distillation_of_long_lists_over_many_tokens(torch, ops):
    """More entries than the workspace holds at a time, with and without gradients, over a vocabulary of less than one tile."""
    from test_distillation_gpu import check

    T, V, D, K = 70003, 100, 16, 1024
    g = gen(torch, 4)
    h, w = torch.randn(T, D, generator=g, device="cuda").bfloat16(), (0.3 * torch.randn(V, D, generator=g, device="cuda")).bfloat16()
    z, index = torch.randn(T, K, generator=g, device="cuda").bfloat16(), torch.randint(-3, V, (T, K), generator=g, device="cuda")
    index[::5] = -1
    check(torch, ops, h, w, z, index, 2.0, torch.rand(T, generator=g, device="cuda"))


def test_calls_warn_about_every_gradient_that_is_lost(torch, ops):
    """Not only the student's: a teacher whose logits are part of a graph, weights of the tokens, frequencies that are learned."""
    import warnings

    g = gen(torch, 5)
    h, w = torch.randn(8, 64, generator=g, device="cuda").bfloat16(), torch.randn(90, 64, generator=g, device="cuda").bfloat16()
    z, index = torch.randn(8, 5, generator=g, device="cuda"), torch.randint(90, (8, 5), generator=g, device="cuda")
    tw, labels = torch.rand(8, generator=g, device="cuda"), index[:, 0].contiguous()
    q, at, f = torch.randn(8, 2, 16, generator=g, device="cuda"), torch.arange(8, device="cuda"), ops.rotary_frequencies(16)
    live = lambda t: t.clone().requires_grad_()  # noqa: E731
    side = torch.cuda.Stream()
    calls = [(ops.linear_distillation, (h, w, live(z), index), {}), (ops.linear_distillation, (h, w, z, index), {"token_weight": live(tw)}),
             (ops.linear_cross_entropy, (h, w, labels), {"token_weight": live(tw)}), (ops.rotary_forward, (q, None, at, live(f)), {})]
    for call, args, kw in calls:
        want = None
        for stream in (None, side):
            torch.cuda.synchronize()
            with pytest.warns(UserWarning, match=f"{call.__name__}: the results have no autograd graph") as seen:
                got = call(*args, **kw, stream=stream)
            assert len(seen) == 1 and seen[0].filename == __file__
            torch.cuda.synchronize()
            with warnings.catch_warnings():
                warnings.simplefilter("error")
                with torch.no_grad():
                    want = call(*args, **kw, stream=stream)
            torch.cuda.synchronize()
            assert all(a is b or torch.equal(a, b) for a, b in zip(got, want))
