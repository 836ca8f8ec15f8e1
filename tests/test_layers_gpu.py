"""Layer norm and rotary positions, forward and backward, against their definitions in 64 bits.

Tolerances.  Every bound is elementwise and counts roundings, u = 2^-24 of float32 (half a step):
  * a sum over a row of F values passes every value through at most `depth` = 40 + F / 4096 additions (eight in a thread's unit, its units, five of a warp, at most
    sixteen warps): |error| <= depth u sum |terms|;
  * the mean is off by em = (depth + 1) u mean|s|; the squares about it by (depth + 4) u of their sum, and a mean that is off by em adds em^2 to their mean; a reciprocal root
    halves a relative error and adds 2^-22 of its own;
  * a value rounded to bfloat16 once: 2^-8 of its size; to float32: u;
  * sums over T rows: a thread adds at most T / 128 + 1 rows, then at most 60 more partial sums meet;
  * an angle is within 2^-25 + 2^-31 of a turn and four roundings of position * frequency in float64 (the reference makes some of them); sine and cosine of it 2^-22.
"""
import ctypes as C
import math
import warnings

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


def name(dtype):
    return str(dtype).replace("torch.", "")


def within(got, ref, bound):
    d = (got.double() - ref).abs()
    assert bool((d <= bound).all()), f"worst error / bound {float((d / bound.clamp(min=1e-300)).max()):.3g}"


# ---- layer norm ---------------------------------------------------------------------------------------------------
def norm_inputs(torch, T, F, seed, dtype, residual=True, offset=0.3):
    g = gen(torch, seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    channel = torch.exp(0.5 * normal(F))
    x = (normal(T, F) * channel + offset * normal(F)).to(dtype)
    r = (normal(T, F) * channel.flip(0)).to(dtype) if residual else None
    return x, r, 1 + 0.3 * normal(F), 0.2 * normal(F)


def check_forward(torch, ops, x, w, b, r, eps, center, keep, dtype):
    T, F = x.shape
    out = ops.layer_norm_forward(x, w, b, residual=r, eps=eps, center=center, keep=keep, dtype=dtype)
    s = x if r is None else (x.float() + r.float()).to(x.dtype)
    assert out.y.dtype == (dtype or x.dtype) and (out.x is x if r is None else torch.equal(out.x, s))
    s, wd, bd = s.double(), w.double(), b.double() if b is not None else 0.0
    depth = 40 + F / 4096
    mean = s.mean(1) if center else torch.zeros(T, dtype=torch.float64, device="cuda")
    em = (depth + 1) * U * s.abs().mean(1) if center else 0.0 * mean
    d = s - mean[:, None]
    var = d.square().mean(1) + eps
    rstd = var.rsqrt()
    er = ((depth + 4) * U + em ** 2 / var + 4 * U) / 2 + 2.0 ** -22
    if center:
        within(out.mean, mean, em + U * mean.abs() + 1e-40)
    else:
        assert out.mean is None
    within(out.rstd, rstd, er * rstd)
    xh = d * rstd[:, None]
    y = xh * wd + bd
    bound = ((em * rstd)[:, None] + (er[:, None] + 6 * U) * xh.abs()) * wd.abs() * (1 + 1e-3)
    within(out.y, y, bound * (1 + HALF_STEP[name(out.y.dtype)]) + (HALF_STEP[name(out.y.dtype)] + 2 * U) * y.abs() + 1e-38)
    if keep:
        again = ops.pack_activation(out.y)
        assert torch.equal(out.kept.q, again.q) and torch.equal(out.kept.scales, again.scales)
    else:
        assert out.kept is None
    return out


def check_backward(torch, ops, fwd, w, dy, d_x, bias, center):
    """Against the formula with the statistics that the forward pass returned."""
    x = fwd.x
    T, F = x.shape
    got = ops.layer_norm_backward(dy, x, w, fwd.mean, fwd.rstd, d_x=d_x, bias=bias)
    assert got.d_x.dtype == x.dtype and got.d_weight.dtype == torch.float32 and (got.d_bias is not None) == bias
    depth = 40 + F / 4096
    s, wd, g, f = x.double(), w.double(), dy.double(), fwd.rstd.double()[:, None]
    m = fwd.mean.double()[:, None] if center else 0.0
    xh = (s - m) * f
    dw, size_w = (g * xh).sum(0), (g * xh).abs().sum(0)
    db, size_b = g.sum(0), g.abs().sum(0)
    g = g * wd
    c1, c2 = (g.mean(1, keepdim=True) if center else 0.0), (g * xh).mean(1, keepdim=True)
    e1, e2 = (depth + 3) * U * g.abs().mean(1, keepdim=True), (depth + 6) * U * (g * xh).abs().mean(1, keepdim=True)
    dx = f * (g - c1 - xh * c2)
    bound = f * (8 * U * (g.abs() + (xh * c2).abs() + abs(c1)) + e1 + xh.abs() * e2)
    if d_x is not None:
        dx = dx + d_x.double()
        bound = bound + U * (dx.abs() + d_x.double().abs())
    step = HALF_STEP[name(x.dtype)]
    within(got.d_x, dx, bound * (1 + step) + (step + 2 * U) * dx.abs() + 1e-38)
    rows = T / 128 + 64
    within(got.d_weight, dw, (rows + 4) * U * size_w + 1e-38)
    if bias:
        within(got.d_bias, db, (rows + 1) * U * size_b + 1e-38)
    return got


NORM_SHAPES = [(1, 1), (1, 8), (2, 7), (3, 33), (5, 100), (1, 768), (37, 256), (9, 771), (300, 768), (130, 1025), (33, 2048), (20, 2050), (40, 2056), (17, 4096), (9, 5504), (6, 8192),
               (5, 8200), (3, 10001), (2, 20000), (3001, 40), (5000, 24), (1537, 515)]
TYPES = [("bfloat16", None), ("float32", None), ("float32", "bfloat16")]


@pytest.mark.parametrize("T,F", NORM_SHAPES)
@pytest.mark.parametrize("x_type,y_type", TYPES)
@pytest.mark.parametrize("center", [True, False])
def test_norm_matches_definition(torch, ops, T, F, x_type, y_type, center):
    dtype, out_type = getattr(torch, x_type), getattr(torch, y_type) if y_type else None
    kind = T + F                                       # (which of the optional parts come along)
    x, r, w, b = norm_inputs(torch, T, F, T * 7 + F, dtype, residual=kind % 3 != 0)
    b = b if center else None
    if kind % 4 == 0:
        w, b = w.bfloat16(), b.bfloat16() if b is not None else None
    fwd = check_forward(torch, ops, x, w, b, r, 1e-5, center, kind % 2 == 0, out_type)
    g = gen(torch, kind)
    dy = (torch.randn(T, F, generator=g, device="cuda") * 1e-2).to(out_type or dtype)
    d_x = (torch.randn(T, F, generator=g, device="cuda") * 1e-2).to(dtype) if kind % 3 == 1 else None
    check_backward(torch, ops, fwd, w, dy, d_x, center, center)


@pytest.mark.parametrize("F", [64, 771, 2048, 8200])
def test_norm_of_rows_with_a_large_mean_and_of_constant_rows(torch, ops, F):
    """A mean 10^4 times the deviations costs no more than its own rounding; rows of one value have a variance of exactly their eps."""
    g = gen(torch, F)
    x = torch.randn(40, F, generator=g, device="cuda") + 1e4
    x[7] = 3.0
    x[8] = 0.0
    w, b = torch.ones(F, device="cuda"), torch.full((F,), 0.5, device="cuda")
    for center in (True, False):
        fwd = check_forward(torch, ops, x, w, b if center else None, None, 1e-5, center, True, None)
        check_backward(torch, ops, fwd, w, torch.randn(40, F, generator=g, device="cuda"), None, True, center)
    out = ops.layer_norm_forward(x, w, b)
    within(out.rstd[7:9], torch.full((2,), 1e-5 ** -0.5, dtype=torch.float64, device="cuda"), torch.full((2,), 2.0 ** -22 * 317, dtype=torch.float64, device="cuda"))
    assert bool((out.y[7:9] == 0.5).all())


def test_norm_eps_zero_and_tiny_rows(torch, ops):
    x = torch.randn(5, 96, generator=gen(torch, 1), device="cuda") * 1e-12
    check_forward(torch, ops, x, torch.ones(96, device="cuda"), None, None, 0.0, True, False, None)
    check_forward(torch, ops, x * 1e24, torch.ones(96, device="cuda"), None, None, 0.0, False, False, None)


@pytest.mark.parametrize("F", [768, 771, 8200])
def test_norm_not_finite(torch, ops, F):
    """A NaN or an infinity stays in its row, and reaches the sums over rows (of its column alone in d_bias' case: not at all)."""
    x, _, w, b = norm_inputs(torch, 20, F, 3, torch.bfloat16, residual=False)
    clean = ops.layer_norm_forward(x, w, b, keep=True)
    x2 = x.clone()
    x2[3, 5], x2[11, F - 1] = float("nan"), float("inf")
    out = ops.layer_norm_forward(x2, w, b, keep=True)
    bad = torch.zeros(20, dtype=torch.bool, device="cuda")
    bad[3] = bad[11] = True
    assert bool(torch.isnan(out.y[bad]).all()) and torch.equal(out.y[~bad], clean.y[~bad])
    assert bool((out.kept.scales[bad] == 255).all()) and torch.equal(out.kept.q[~bad], clean.kept.q[~bad])
    dy = torch.randn(20, F, generator=gen(torch, 4), device="cuda").bfloat16()
    d, c = ops.layer_norm_backward(dy, x2, w, out.mean, out.rstd, bias=True), ops.layer_norm_backward(dy, x, w, clean.mean, clean.rstd, bias=True)
    assert bool(torch.isnan(d.d_x[bad]).all()) and torch.equal(d.d_x[~bad], c.d_x[~bad]) and bool(torch.isnan(d.d_weight).all()) and torch.equal(d.d_bias, c.d_bias)


@pytest.mark.parametrize("F", [64, 100, 771, 2048])
@pytest.mark.parametrize("x_type", ["bfloat16", "float32"])
def test_norm_rows_of_any_stride(torch, ops, F, x_type):
    """Parts of wider matrices, aligned and not; NaN around them."""
    T, dtype = 37, getattr(torch, x_type)
    x, r, w, b = norm_inputs(torch, T, F, F, dtype)
    dy, d_x = (torch.randn(T, F, generator=gen(torch, s), device="cuda").to(dtype) for s in (5, 6))
    for start, gap in ((0, 0), (8, 24), (1, 3), (3, 8)):
        def part(t):
            wide = torch.full((T, F + start + gap), float("nan"), dtype=t.dtype, device="cuda")
            wide[:, start:start + F] = t
            return wide[:, start:start + F]

        fwd = check_forward(torch, ops, part(x), w, b, part(r), 1e-5, True, True, None)
        check_backward(torch, ops, fwd, w, part(dy), part(d_x), True, True)
        plain = ops.layer_norm_forward(part(x), w, b)
        check_backward(torch, ops, plain, w, part(dy), None, False, True)


def test_norm_writes_its_rows_only(torch, ops):
    """C entry points with strides of their own: what lies between the rows stays."""
    from paper_2509_11254_b200 import binding

    L = binding.lib()
    T, bad = 11, 7.0
    for F in (64, 101, 8203):
        x, r, w, b = norm_inputs(torch, T, F, F, torch.bfloat16)
        dy = torch.randn(T, F, generator=gen(torch, 1), device="cuda").bfloat16()
        want = ops.layer_norm_forward(x, w, b, residual=r)
        grad = ops.layer_norm_backward(dy, want.x, w, want.mean, want.rstd, bias=True)
        for gap in (8, 5):
            s, y, dx = (torch.full((T, F + gap), bad, dtype=torch.bfloat16, device="cuda") for _ in range(3))
            f, sums = torch.empty(2, T, device="cuda"), torch.empty(2, F, device="cuda")
            n = C.c_size_t()
            assert L.psgd_norm_workspace(T, F, C.byref(n)) == 0
            ws = torch.empty(n.value, dtype=torch.uint8, device="cuda")
            at = torch.cuda.current_stream().cuda_stream
            assert L.psgd_norm_forward(x.data_ptr(), F, 1, r.data_ptr(), F, w.data_ptr(), b.data_ptr(), 0, 1e-5, 1, T, F, s.data_ptr(), F + gap, y.data_ptr(), F + gap, 1,
                                       f[1].data_ptr(), f[0].data_ptr(), None, None, at) == 0
            assert L.psgd_norm_backward(dy.data_ptr(), F, 1, s.data_ptr(), F + gap, 1, w.data_ptr(), 0, f[1].data_ptr(), f[0].data_ptr(), None, 0, T, F, dx.data_ptr(), F + gap,
                                        sums.data_ptr(), sums[1].data_ptr(), ws.data_ptr(), n.value, at) == 0
            assert torch.equal(s[:, :F], want.x)
            for t, ref in ((y, want.y), (dx, grad.d_x)):
                within(t[:, :F], ref.double(), 2 * 2.0 ** -8 * ref.double().abs() + 1e-6)          # (another split of the rows: another rounding)
            for t in (s, y, dx):
                assert bool((t[:, F:] == bad).all())


def test_norm_no_rows(torch, ops):
    x, w = torch.zeros(0, 40, device="cuda"), torch.ones(40, device="cuda")
    out = ops.layer_norm_forward(x, w, w, residual=x, keep=True)
    assert out.y.shape == (0, 40) and out.mean.shape == (0,) and out.kept.q.shape == (0, 64)
    d = ops.layer_norm_backward(x, x, w, out.mean, out.rstd, d_x=x, bias=True)
    assert d.d_x.shape == (0, 40) and not d.d_weight.any() and not d.d_bias.any() and d.d_weight.shape == (40,)


def test_norm_beyond_32_bit_offsets(torch, ops):
    T, F = (1 << 20) + 3, 2080                           # 2.2e9 values
    x = torch.zeros((T, F), dtype=torch.bfloat16, device="cuda")
    tail, _, w, b = norm_inputs(torch, 5, F, 1, torch.bfloat16, residual=False)
    x[-5:] = tail
    out, want = ops.layer_norm_forward(x, w, b, keep=True), ops.layer_norm_forward(tail, w, b, keep=True)
    assert torch.equal(out.y[-5:], want.y) and torch.equal(out.kept.q[-5:], want.kept.q) and torch.equal(out.rstd[-5:], want.rstd)
    mean, rstd = out.mean, out.rstd
    del out
    dy = x
    d, e = ops.layer_norm_backward(dy, x, w, mean, rstd, bias=True), ops.layer_norm_backward(tail, tail, w, want.mean, want.rstd, bias=True)
    assert torch.equal(d.d_x[-5:], e.d_x) and not d.d_x[:1000].any()
    within(d.d_bias, e.d_bias.double(), 16 * U * tail.double().abs().sum(0))
    xh = ((tail.double() - want.mean.double()[:, None]) * want.rstd.double()[:, None]).abs()
    within(d.d_weight, e.d_weight.double(), 32 * U * (tail.double().abs() * xh).sum(0))


def test_norm_gradient_by_differences(torch, ops):
    """Central differences of the kernel's own forward pass, float32.  loss = sum(dy y), its rounding at most 2^-20 of sum |dy y| ~ 200: 2e-4 over a step of 2^-4."""
    T, F = 3, 40
    x, r, w, b = norm_inputs(torch, T, F, 9, torch.float32)
    dy = torch.randn(T, F, generator=gen(torch, 2), device="cuda")
    for center in (True, False):
        def loss(x, r, w, b):
            return float((ops.layer_norm_forward(x, w, b, residual=r, center=center).y.double() * dy.double()).sum())

        fwd = ops.layer_norm_forward(x, w, b, residual=r, center=center)
        d = ops.layer_norm_backward(dy, fwd.x, w, fwd.mean, fwd.rstd, bias=True)
        args = [x, r, w, b]
        for which, grad in ((0, d.d_x), (1, d.d_x), (2, d.d_weight), (3, d.d_bias)):
            for at in ((0, 0), (1, 17), (2, 39)) if which < 2 else ((0,), (17,), (39,)):
                def moved(by):
                    a = [t.clone() for t in args]
                    a[which][at] += by
                    return loss(*a)

                h = 2.0 ** -4
                first, half = (moved(h) - moved(-h)) / (2 * h), (moved(h / 2) - moved(-h / 2)) / h
                want = half + (half - first) / 3           # the quadratic term taken out, as large as what it took out for the rest
                assert abs(float(grad[at]) - want) <= abs(half - first) + 2e-2 * h + 1e-3 * abs(want), (which, at)


# ---- rotary positions ---------------------------------------------------------------------------------------------
def turned(torch, x, positions, f, layout, scale, way=1):
    """The definition in 64 bits and what its bound is made of: (values, size of what each is the sum of, error of the angle)."""
    n = f.numel()
    angle = positions.double()[:, None] * f
    c, s = (scale * torch.cos(angle))[:, None], (way * scale * torch.sin(angle))[:, None]
    x = x.double()
    a, b = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    out, size = x.clone(), torch.zeros_like(x)
    u, v = x[..., a], x[..., b]
    out[..., a], out[..., b] = u * c - v * s, u * s + v * c
    off = (2 * math.pi * (2.0 ** -25 + 2.0 ** -31) + 4 * angle.abs() * 2.0 ** -53 + 2.0 ** -22 + 4 * U)[:, None]
    size[..., a] = size[..., b] = abs(scale) * (u.abs() + v.abs()) * off
    return out, size


def check_rotary(torch, ops, q, k, positions, f, layout="half", scale=1.0, **kw):
    out = []
    for call, way in ((ops.rotary_forward, 1), (ops.rotary_backward, -1)):
        got = call(q.clone() if kw.get("in_place") else q, k.clone() if kw.get("in_place") and k is not None else k, positions, f, layout=layout, scale=scale, **kw)
        for t, x in zip(got, (q, k)):
            if x is None:
                assert t is None
                continue
            ref, size = turned(torch, x, positions, f, layout, scale, way)
            step = HALF_STEP[name(x.dtype)]
            assert t.dtype == x.dtype and t.shape == x.shape
            within(t, ref, size * (1 + step) + step * ref.abs() + 1e-38)
            n = 2 * f.numel()
            assert torch.equal(t[..., n:], x[..., n:])
        out.append(got)
    return out


ROTARY_SHAPES = [(1, 1, 0, 2, 2), (1, 12, 12, 64, 64), (3, 2, 1, 6, 2), (7, 5, 1, 80, 20), (33, 4, 2, 128, 128), (257, 3, 3, 96, 64), (65, 9, 3, 80, 48), (1000, 2, 1, 34, 34), (19, 1, 1, 256, 16),
                 (4, 70, 70, 128, 128), (5, 2, 2, 130, 128), (2100, 8, 2, 64, 32), (2, 3, 1, 4096, 4096)]


@pytest.mark.parametrize("T,H,K,D,R", ROTARY_SHAPES)
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_rotary_matches_definition(torch, ops, T, H, K, D, R, layout, dtype):
    g = gen(torch, T + D + R)
    packed = torch.randn(T, H + 2 * K, D, generator=g, device="cuda").to(getattr(torch, dtype))
    q, k = packed[:, :H], packed[:, H:H + K] if K else None
    positions = torch.randint(1 << 17, (T,), generator=g, device="cuda")
    f = ops.rotary_frequencies(R, factor=4.0, original_length=8192)
    a = check_rotary(torch, ops, q, k, positions, f, layout, 1.25)
    b = check_rotary(torch, ops, q, k, positions, f, layout, 1.25, in_place=True)
    for x, y in zip(a, b):
        for s, t in zip(x, y):
            assert s is None and t is None or torch.equal(s, t)


def test_rotary_of_far_positions(torch, ops):
    """Negative ones, 2^20 and 2^40, the same position twice; bases whose fastest pair makes more than a turn per position."""
    g = gen(torch, 3)
    positions = torch.tensor([0, 1, -1, 1 << 20, -(1 << 20), 12345678, 12345678, 1 << 31, (1 << 31) - 1], device="cuda")
    q = torch.randn(len(positions), 3, 64, generator=g, device="cuda")
    f = ops.rotary_frequencies(64)
    (forward, _), (back, _) = check_rotary(torch, ops, q, None, positions, f)
    assert torch.equal(forward[0], q[0]) and torch.equal(forward[1, 0], check_rotary(torch, ops, q[1:2], None, positions[1:2], f)[0][0][0, 0])
    check_rotary(torch, ops, q, None, positions, f * 37.5)
    # frequencies whose turns are exact: 2^-20 and 1/4 of a turn, far beyond what float64 positions times radians could tell apart
    f = torch.tensor([2 * math.pi / 4], dtype=torch.float64, device="cuda")
    far = torch.tensor([(1 << 40) + 1, (1 << 40) + 2], device="cuda")
    x = torch.tensor([[[1.0, 0.0]], [[1.0, 0.0]]], device="cuda")
    out = ops.rotary_forward(x, None, far, f)[0]
    assert torch.allclose(out[:, 0], torch.tensor([[0.0, 1.0], [-1.0, 0.0]], device="cuda"), atol=2.0 ** -10)


def test_rotary_is_undone_by_its_backward(torch, ops):
    """<turned q, y> = <q, y turned back>, and turning back what was turned gives q: two rotations' bounds in float32."""
    g = gen(torch, 4)
    q, y = (torch.randn(50, 6, 80, generator=g, device="cuda") for _ in range(2))
    positions = torch.randint(5000, (50,), generator=g, device="cuda")
    f = ops.rotary_frequencies(48)
    for layout in ("half", "interleaved"):
        t = ops.rotary_forward(q, y, positions, f, layout=layout)
        back = ops.rotary_backward(t[0], y, positions, f, layout=layout)
        within(back[0], q.double(), 4e-6 * (q.double().abs() + q.double().abs().amax(2, keepdim=True)))
        left, right = (t[0].double() * y.double()).sum(), (q.double() * back[1].double()).sum()
        assert abs(float(left - right)) <= 2e-6 * float((q.double().abs() * y.double().abs()).sum()) + 1e-2


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_rotary_strides(torch, ops, dtype):
    """Heads before tokens, gaps, odd offsets, values used several times."""
    g = gen(torch, 5)
    T, H, D = 21, 4, 64
    f, positions = ops.rotary_frequencies(32), torch.arange(T, device="cuda") * 7
    base = torch.randn(H, T, D, generator=g, device="cuda").to(getattr(torch, dtype))
    check_rotary(torch, ops, base.transpose(0, 1), base[:2].transpose(0, 1), positions, f)
    wide = torch.randn(T, H, D + 9, generator=g, device="cuda").to(getattr(torch, dtype))
    check_rotary(torch, ops, wide[:, :, 1:D + 1], wide[:, 1:3, 3:D + 3], positions, f, "interleaved")
    shared = wide[:, :1, :D].expand(T, H, D)
    check_rotary(torch, ops, shared, shared, positions, f)
    before = wide.clone()
    ops.rotary_forward(wide[:, :2, 4:D + 4], wide[:, 3:, 4:D + 4], positions, f, in_place=True)
    assert torch.equal(wide[:, 2], before[:, 2]) and torch.equal(wide[..., :4], before[..., :4]) and torch.equal(wide[..., D + 4:], before[..., D + 4:])
    assert torch.equal(wide[:, :2, 4:D + 4], ops.rotary_forward(before[:, :2, 4:D + 4], None, positions, f)[0])
    for bad in (lambda: ops.rotary_forward(shared, None, positions, f, in_place=True), lambda: ops.rotary_forward(wide[:, :2], wide[:, 1:3], positions, f, in_place=True)):
        with pytest.raises(ops.PSGDError):
            bad()


def test_rotary_edges(torch, ops):
    f, none = ops.rotary_frequencies(8), torch.zeros(0, dtype=torch.int64, device="cuda")
    q = torch.randn(0, 3, 16, device="cuda")
    assert ops.rotary_forward(q, q, none, f)[1].shape == (0, 3, 16)
    x = torch.randn(4, 2, 16, device="cuda")
    at = torch.arange(4, device="cuda")
    out = ops.rotary_forward(x, x[:, :0], at, f)
    assert out[1].shape == (4, 0, 16) and torch.equal(out[0], ops.rotary_forward(x, None, at, f)[0])
    assert torch.equal(ops.rotary_forward(x[:, :0], x, at, f)[1], out[0])
    y = x.clone()
    y[2, 1, 3], y[3, 0, 15] = float("nan"), float("inf")
    got = ops.rotary_forward(y, None, at, f)[0]
    bad = torch.isnan(got)
    assert int(bad.sum()) == 2 and bool(bad[2, 1, 3]) and bool(bad[2, 1, 7]) and float(got[3, 0, 15]) == float("inf")
    assert torch.equal(torch.nan_to_num(got, nan=0.0, posinf=0.0)[:2], out[0][:2])


def test_rotary_beyond_32_bit_offsets(torch, ops):
    T, H, D = (1 << 19) + 1, 36, 128                     # 2.4e9 values
    q = torch.zeros((T, H, D), dtype=torch.bfloat16, device="cuda")
    tail = torch.randn(3, H, D, generator=gen(torch, 1), device="cuda").bfloat16()
    q[-3:] = tail
    positions = torch.arange(T, device="cuda")
    f = ops.rotary_frequencies(D)
    out = ops.rotary_forward(q, None, positions, f)[0]
    assert torch.equal(out[-3:], ops.rotary_forward(tail, None, positions[-3:].contiguous(), f)[0]) and not out[:1000].any()
    ops.rotary_forward(q, None, positions, f, in_place=True)
    assert torch.equal(q[-3:], out[-3:])


# ---- together, streams, graphs ------------------------------------------------------------------------------------
def layer_step(ops, x, r, w, b, dy, positions, f, stream=None):
    """A norm, its 8-bit result, the result as queries and keys, and the way back."""
    kw = dict(stream=stream)
    n = ops.layer_norm_forward(x, w, b, residual=r, keep=True, **kw)
    T, F = x.shape
    heads = n.y.view(T, F // 32, 32)
    q, k = ops.rotary_forward(heads[:, :5], heads[:, 5:], positions, f, **kw)
    dq, dk = ops.rotary_backward(q, k, positions, f, **kw)
    d = ops.layer_norm_backward(dy, n.x, w, n.mean, n.rstd, d_x=r, bias=True, **kw)
    return [n.y, n.x, n.mean, n.rstd, n.kept.unpack(**kw), q, k, dq, dk, *d, ops.weight_gradient(dy, n.kept, **kw)]


def layer_inputs(torch, ops, T, seed):
    x, r, w, b = norm_inputs(torch, T, 768, seed, torch.bfloat16)
    return x, r, w, b, torch.randn(T, 768, generator=gen(torch, seed + 1), device="cuda").bfloat16(), torch.arange(T, device="cuda"), ops.rotary_frequencies(32)


def test_layer_calls_repeat_bit_for_bit(torch, ops):
    args = layer_inputs(torch, ops, 3000, 1)
    for a, b in zip(layer_step(ops, *args), layer_step(ops, *args)):
        assert torch.equal(a, b)


def test_layer_calls_in_a_cuda_graph(torch, ops):
    """Captured once, replayed with other inputs in the same places; two graphs that share a pool."""
    args = layer_inputs(torch, ops, 300, 3)
    layer_step(ops, *args)
    torch.cuda.synchronize()
    graphs, outs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()], []
    for i, g in enumerate(graphs):
        with torch.cuda.graph(g, pool=graphs[0].pool() if i else None):
            outs.append(layer_step(ops, *args))
    for t, u in zip(args[:6], layer_inputs(torch, ops, 300, 5)):
        t.copy_(u)
    want = layer_step(ops, *args)
    for g, out in zip(graphs, outs):
        for t in out:
            t.fill_(7)
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b)


def test_layer_calls_on_two_streams_at_once(torch, ops):
    sets = [layer_inputs(torch, ops, 1500, s) for s in (11, 12)]
    want = [layer_step(ops, *s) for s in sets]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[layer_step(ops, *sets[i], stream=streams[i]) for i in (0, 1)] for _ in range(5)]
    torch.cuda.synchronize()
    for both in got:
        for a, b in zip(both, want):
            for u, v in zip(a, b):
                assert torch.equal(u, v)


def test_layer_inputs_freed_before_another_stream_has_read_them(torch, ops):
    args = layer_inputs(torch, ops, 700, 21)
    want = layer_step(ops, *args)
    s = torch.cuda.Stream()
    mine = [t.clone() for t in args]
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
    got = layer_step(ops, *mine, stream=s)
    sizes = [(t.shape, t.dtype) for t in mine]
    del mine
    torch.cuda.current_stream().synchronize()
    others = [torch.full(shape, 3, dtype=dtype, device="cuda") for shape, dtype in sizes for _ in range(4)]
    torch.cuda.synchronize()
    assert len(others) == 4 * len(sizes)
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_layer_calls_warn_about_a_lost_graph(torch, ops):
    x, r, w, b, dy, positions, f = layer_inputs(torch, ops, 8, 31)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    leaf, weight = x.clone().requires_grad_(), w.clone().requires_grad_()
    heads = leaf.view(8, 24, 32)
    for call in (lambda: ops.layer_norm_forward(leaf, w), lambda: ops.layer_norm_forward(x, weight, b, stream=side), lambda: ops.layer_norm_forward(x, w, residual=leaf),
                 lambda: ops.rotary_forward(heads, None, positions, f), lambda: ops.rotary_forward(heads.detach(), heads, positions, f, stream=side)):
        with pytest.warns(UserWarning, match="no autograd graph") as seen:
            call()
        assert len(seen) == 1 and seen[0].filename == __file__
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        with torch.no_grad():
            ops.layer_norm_forward(leaf, weight)
        n = ops.layer_norm_forward(x, w)
        ops.layer_norm_backward(dy, leaf, weight, n.mean, n.rstd)
        ops.rotary_backward(heads, None, positions, f)
    torch.cuda.synchronize()


def test_layer_calls_refuse(torch, ops):
    x, r, w, b, dy, positions, f = layer_inputs(torch, ops, 8, 41)
    n = ops.layer_norm_forward(x, w, b)
    q = x.view(8, 24, 32)
    bad = [lambda: ops.layer_norm_forward(x.half(), w), lambda: ops.layer_norm_forward(x, w[:5]), lambda: ops.layer_norm_forward(x, w.double()), lambda: ops.layer_norm_forward(x, w, b.bfloat16()),
           lambda: ops.layer_norm_forward(x, w, residual=r.float()), lambda: ops.layer_norm_forward(x, w, residual=r[:4]), lambda: ops.layer_norm_forward(x, w, dtype=torch.float32),
           lambda: ops.layer_norm_forward(x, w, eps=-1.0), lambda: ops.layer_norm_forward(x, w, eps=float("nan")), lambda: ops.layer_norm_forward(x.T, w), lambda: ops.layer_norm_forward(x, None),
           lambda: ops.layer_norm_forward(x.cpu(), w), lambda: ops.layer_norm_backward(dy.float(), x, w, n.mean, n.rstd), lambda: ops.layer_norm_backward(dy, x, w, n.mean, n.rstd[:3]),
           lambda: ops.layer_norm_backward(dy, x, w, n.mean, None), lambda: ops.layer_norm_backward(dy[:3], x, w, n.mean, n.rstd), lambda: ops.layer_norm_backward(dy, x, w, n.mean, n.rstd, d_x=r.float()),
           lambda: ops.rotary_forward(x, None, positions, f), lambda: ops.rotary_forward(q, q.float(), positions, f), lambda: ops.rotary_forward(q, q[:4], positions, f),
           lambda: ops.rotary_forward(q, None, positions.int(), f), lambda: ops.rotary_forward(q, None, positions[:4], f), lambda: ops.rotary_forward(q, None, positions, f.float()),
           lambda: ops.rotary_forward(q, None, positions, ops.rotary_frequencies(34)), lambda: ops.rotary_forward(q, None, positions, f[:0]), lambda: ops.rotary_forward(q, None, positions, f, layout="pairs"),
           lambda: ops.rotary_forward(q.transpose(1, 2), None, positions, f), lambda: ops.rotary_forward(q[..., :1], None, positions, f), lambda: ops.rotary_forward(q, None, positions, f.view(4, 4))]
    for call in bad:
        with pytest.raises(ops.PSGDError):
            call()


@pytest.mark.parametrize("T", [1, 2, 9])
@pytest.mark.parametrize("F", [1, 2, 3, 7, 8, 9, 31, 255, 256, 257, 263, 511, 1000, 1537, 2057, 5003])
def test_norm_rows_of_every_alignment(torch, ops, T, F):
    """Every start within 16 bytes, strides that move it from row to row (down to rows of one value side by side), NaN everywhere else in the buffers."""
    w, b = 1 + 0.3 * torch.randn(F, generator=gen(torch, 1), device="cuda"), 0.2 * torch.randn(F, generator=gen(torch, 2), device="cuda")
    for start, gap in ((0, 0), (1, 0), (2, 1), (3, 2), (5, 3), (7, 7), (4, 8)):
        def part(seed):
            flat = torch.full((start + T * (F + gap) + 16,), float("nan"), device="cuda", dtype=torch.bfloat16)
            t = flat.as_strided((T, F), (F + gap, 1), start)
            t.copy_(torch.randn(T, F, generator=gen(torch, seed), device="cuda"))
            return t

        x, r, dy, d_x = (part(s) for s in (3, 4, 5, 6))
        fwd = check_forward(torch, ops, x, w, b, r, 1e-5, True, True, None)
        check_backward(torch, ops, fwd, w, dy, d_x, True, True)
        fwd = check_forward(torch, ops, x, w, None, None, 1e-5, False, False, None)
        check_backward(torch, ops, fwd, w, dy, None, False, False)


@pytest.mark.parametrize("T,F", [(700, 40), (2500, 2051), (1201, 2047), (700, 5003), (300, 12345), (40, 16371), (17, 16383)])
def test_norm_many_rows_of_odd_widths(torch, ops, T, F):
    """Every thread takes several rows, that begin at eight places within 16 bytes."""
    x, r, w, b = norm_inputs(torch, T, F, F, torch.bfloat16)
    dy, d_x = (torch.randn(T, F, generator=gen(torch, s), device="cuda").bfloat16() for s in (5, 6))
    fwd = check_forward(torch, ops, x, w, b, r, 1e-5, True, True, None)
    check_backward(torch, ops, fwd, w, dy, d_x, True, True)
    fwd = check_forward(torch, ops, x, w, None, None, 1e-5, False, False, None)
    check_backward(torch, ops, fwd, w, dy, None, False, False)


@pytest.mark.parametrize("T,F", [(1, 5), (9, 3), (1, 771), (20, 771), (1, 2051), (9, 2051), (30, 2056), (13, 4099), (2060, 2051)])
def test_norm_operands_that_begin_alike(torch, ops, T, F):
    """C entry points, all operands at one place within 16 bytes: the same values as those of aligned copies, and nothing else read or written."""
    from paper_2509_11254_b200 import binding

    L = binding.lib()
    x, r, w, b = norm_inputs(torch, T, F, F, torch.bfloat16)
    dy, add = (torch.randn(T, F, generator=gen(torch, s), device="cuda").bfloat16() for s in (1, 2))
    want = ops.layer_norm_forward(x, w, b, residual=r, keep=True)
    grad = ops.layer_norm_backward(dy, want.x, w, want.mean, want.rstd, d_x=add, bias=True)
    for start, gap in ((0, 0), (1, 0), (3, 5), (7, 8), (4, 1)):
        def part(t=None):
            flat = torch.full((start + T * (F + gap) + 16,), float("nan"), device="cuda", dtype=torch.bfloat16)
            view = flat.as_strided((T, F), (F + gap, 1), start)
            if t is not None:
                view.copy_(t)
            return flat, view

        (_, xv), (_, rv), (_, dv), (_, av), (fs, s), (fy, y), (fd, dx) = part(x), part(r), part(dy), part(add), part(), part(), part()
        f, sums = torch.empty(2, T, device="cuda"), torch.empty(2, F, device="cuda")
        q, scales = torch.empty_like(want.kept.q), torch.empty_like(want.kept.scales)
        n = C.c_size_t()
        assert L.psgd_norm_workspace(T, F, C.byref(n)) == 0
        ws = torch.empty(n.value, dtype=torch.uint8, device="cuda")
        at, ld = torch.cuda.current_stream().cuda_stream, F + gap
        assert L.psgd_norm_forward(xv.data_ptr(), ld, 1, rv.data_ptr(), ld, w.data_ptr(), b.data_ptr(), 0, 1e-5, 1, T, F, s.data_ptr(), ld, y.data_ptr(), ld, 1,
                                   f[1].data_ptr(), f[0].data_ptr(), q.data_ptr(), scales.data_ptr(), at) == 0
        again = ops.pack_activation(y.contiguous())
        assert torch.equal(q, again.q) and torch.equal(scales, again.scales)
        assert L.psgd_norm_backward(dv.data_ptr(), ld, 1, s.data_ptr(), ld, 1, w.data_ptr(), 0, f[1].data_ptr(), f[0].data_ptr(), av.data_ptr(), ld, T, F, dx.data_ptr(), ld,
                                    sums.data_ptr(), sums[1].data_ptr(), ws.data_ptr(), n.value, at) == 0
        assert torch.equal(s, want.x)
        for t, ref in ((y, want.y), (dx, grad.d_x)):
            within(t, ref.double(), 2 * 2.0 ** -8 * ref.double().abs() + 1e-5)             # another order of the sums: another rounding of the result, one step of two halves
        for t, ref, size in ((sums[0], grad.d_weight, dy.double().abs().sum(0) * 8), (sums[1], grad.d_bias, dy.double().abs().sum(0))):
            within(t, ref.double(), 200 * U * size + 1e-6)
        for flat in (fs, fy, fd):
            assert int(torch.isnan(flat).sum()) == flat.numel() - T * F


def test_norm_sums_of_bfloat16_are_rounded_once(torch, ops):
    """x + residual over all exponents: subnormal numbers, zeros of either sign, overflow, infinities, ties between two neighbours."""
    g = gen(torch, 1)
    bits = torch.randint(-(1 << 15), 1 << 15, (2, 64, 2048), generator=g, device="cuda", dtype=torch.int32).to(torch.int16)
    x, r = bits.view(torch.bfloat16)
    r[::2] = (x[::2].float() * (torch.randint(-9, 10, x[::2].shape, generator=g, device="cuda") / 512)).bfloat16()      # near enough for ties
    r[0, :4], x[0, :4] = torch.tensor([0.0, -0.0, 0.0, -0.0]).bfloat16(), torch.tensor([0.0, 0.0, -0.0, -0.0]).bfloat16()
    w = torch.ones(2048, device="cuda")
    for F in (2048, 2047):
        got, want = ops.layer_norm_forward(x[:, :F], w[:F], residual=r[:, :F]).x, (x[:, :F].float() + r[:, :F].float()).bfloat16()
        nan = torch.isnan(want)
        assert torch.equal(torch.isnan(got), nan) and torch.equal(got.view(torch.int16)[~nan], want.contiguous().view(torch.int16)[~nan])


# ---- the plain call and the long way ------------------------------------------------------------------------------
def test_plain_calls_equal_the_others(torch, ops, monkeypatch):
    """The same bits and the same refusals whether the call is made by _call.so or by the Python functions behind it, over types, optional parts, strides and single rows."""
    from paper_2509_11254_b200 import layers, training

    class Never:                                       # answers None to everything
        def __getattr__(self, name):
            return lambda *a: None

    took = []

    def both(call):
        monkeypatch.undo()
        module = training._plain()

        class Watch:
            def __getattr__(self, name):
                def f(*a):
                    r = getattr(module, name)(*a)
                    took.append(r is not None)
                    return r
                return f

        out = []
        for stand_in in (Watch(), Never()):
            monkeypatch.setattr(layers, "_plain", lambda: stand_in)
            monkeypatch.setattr(training, "_plain", lambda: stand_in)
            try:
                out.append(call())
            except ops.PSGDError as e:
                out.append(str(e))
        monkeypatch.undo()
        a, b = out
        assert type(a) is type(b)
        if isinstance(a, str):
            assert a == b
            return
        for u, v in zip(a, b):
            if u is None or v is None:
                assert u is v
            elif isinstance(u, ops.ActivationCheckpoint):
                assert u.shape == v.shape and torch.equal(u.q, v.q) and torch.equal(u.scales, v.scales)
            else:
                assert u.dtype == v.dtype and u.shape == v.shape and u.stride() == v.stride() and torch.equal(u, v)

    for T, F in ((1, 1), (1, 40), (7, 96), (5, 101), (3, 1)):
        for dtype in (torch.bfloat16, torch.float32):
            x, r, w, b = norm_inputs(torch, T, F, 3, dtype)
            wide = torch.zeros(T, F + 8, dtype=dtype, device="cuda")
            wide[:, :F] = x
            n = ops.layer_norm_forward(x, w, b)
            both(lambda: ops.layer_norm_forward(x, w, b))
            both(lambda: ops.layer_norm_forward(wide[:, :F], w.bfloat16(), None, residual=r, center=False, keep=True))
            both(lambda: ops.layer_norm_backward(r, x, w, n.mean, n.rstd))
            both(lambda: ops.layer_norm_backward(r, wide[:, :F], w, None, n.rstd, d_x=x, bias=True))
            both(lambda: ops.layer_norm_backward(r.bfloat16(), x, w, n.mean, n.rstd))
            both(lambda: ops.layer_norm_forward(x, w[:-1], b))
            both(lambda: ops.layer_norm_forward(x, w, b, residual=r[:, 1:]))
    q = torch.randn(9, 6, 32, device="cuda")
    at, f = torch.arange(9, device="cuda"), ops.rotary_frequencies(16)
    for t in (q, q[:, 1:5], q.transpose(0, 1).contiguous().transpose(0, 1), q[:, :1].expand(9, 6, 32), q[:1], q[:, :1]):
        at_t = at[:t.shape[0]]
        both(lambda: ops.rotary_forward(t, None, at_t, f))
        both(lambda: ops.rotary_backward(t, t, at_t, f, layout="interleaved", scale=0.5))
        both(lambda: ops.rotary_forward(t.clone(), t.clone(), at_t, f, in_place=True))
    both(lambda: ops.rotary_forward(q, None, at, f, in_place=True)[:0])
    both(lambda: ops.rotary_forward(q[:, :1].expand(9, 6, 32), None, at, f, in_place=True))
    both(lambda: ops.rotary_forward(q, q.double(), at, f))
    for T in (1, 6):
        h, w = torch.randn(T, 64, device="cuda").bfloat16(), torch.randn(90, 64, device="cuda").bfloat16()
        z, i = torch.randn(T, 5, device="cuda"), torch.randint(90, (T, 5), device="cuda")
        both(lambda: ops.linear_distillation(h, w, z, i, 2.0))
        both(lambda: ops.linear_distillation_grad(h, w, z.bfloat16(), i, token_weight=torch.ones(T, device="cuda")))
        both(lambda: ops.linear_distillation_grad(h[:, 1:41], w[:, 1:41], z, i))
        both(lambda: ops.linear_distillation(h, w, z, i, 0.0))
    assert sum(took) > 60 and len(took) - sum(took) > 20       # both ways were taken
