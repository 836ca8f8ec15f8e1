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


