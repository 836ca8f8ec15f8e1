"""Training operators between a layer's matrix products: layer norm and rotary positions, forward and backward.

  layer_norm_forward, layer_norm_backward                layer norm (or without centring: root mean square norm) of a residual sum, its result kept in 8 bits on
                                                         request for weight_gradient, and its gradients
  rotary_frequencies, rotary_forward, rotary_backward    rotary positions of queries and keys, and of their gradients

The arithmetic runs in the CUDA library (psgd_norm_*, psgd_rotary of include/psgd.h).  As with the other training operators every call is stream-ordered on
`stream` (default: the current stream), does not synchronise, can be captured in a CUDA graph and takes no part in autograd: gradients are results of calls of
their own, and layer_norm_forward and rotary_forward warn where an input requires one.

The plain call (tensors on the current device, the current stream, nothing to refuse or to warn about) goes through _call.so, whose functions answer None where
it is not one.
"""
from __future__ import annotations

import math
from collections import namedtuple

import torch

from .binding import PSGDError, lib
from .training import _BF16, _BOTH, _DTYPES, ActivationCheckpoint, _check, _empty, _here, _matrix, _name, _no_graph, _plain, _there, _vector, _workspace_bytes, _written

LayerNorm = namedtuple("LayerNorm", "y x mean rstd kept")
LayerNormGrad = namedtuple("LayerNormGrad", "d_x d_weight d_bias")

_LAYOUTS = {"half": 0, "interleaved": 1}
_empty_like = torch.empty_like


def _like(x, rows, cols):
    """A new matrix of x's shape and type whose rows lie one after the other (the shortest way to it where x's own do)."""
    return _empty_like(x) if x.stride() == (cols, 1) else _empty((rows, cols), dtype=x.dtype, device=x.device)


# ---- layer norm ---------------------------------------------------------------------------------------------------
def _param(t, name, n, device, dtype=None):
    """(address, dtype code) of a vector over the columns, float32 or bfloat16 (or `dtype`)."""
    code = _DTYPES.get(t.dtype) if isinstance(t, torch.Tensor) else None
    if code is None or (dtype is not None and t.dtype != dtype) or t.shape != (n,) or not t.is_contiguous() or t.get_device() != device.index:
        raise PSGDError(f"{name} must be a contiguous {'float32 or bfloat16' if dtype is None else _name(dtype)} tensor of {n} elements on {device}")
    return t.data_ptr(), code


def layer_norm_forward(x, weight, bias=None, residual=None, eps=1e-5, center=True, keep=False, dtype=None, stream=None):
    """y = (s - mean(s)) / sqrt(mean((s - mean(s))^2) + eps) * weight + bias over the rows of s = x + residual, [T, F].

    center=False leaves the mean in (root mean square norm).  x and residual are bfloat16 or float32, alike; s is rounded to that type.  weight and bias [F] are
    float32 or bfloat16, alike; bias and residual may be None.  y has x's type, or `dtype` (bfloat16 beside a float32 x).
    Returns (y, x, mean, rstd, kept): x is s (the very tensor `x` without a residual), which the backward pass reads; mean (None without centring) and rstd float32 [T];
    kept the 8-bit checkpoint of y, what pack_activation(y) makes, where `keep` asks for it.
    """
    if stream is None and dtype is None:
        r = _plain().norm_forward(x, weight, bias, residual, eps, center, keep)
        if type(r) is tuple:
            y, s, mean, rstd, buf = r
            return LayerNorm(y, s, mean, rstd, ActivationCheckpoint(*x.shape, x.device, buf) if keep else None)
        if r is not None:
            _check(r)
    T, F, ldx = _matrix(x, "x", _BOTH)
    dev = x.device
    at_w, w_type = _param(weight, "weight", F, dev)
    at_b = _param(bias, "bias", F, dev, weight.dtype)[0] if bias is not None else None
    ldr = _matrix(residual, "residual", (x.dtype,), (T, F), dev)[2] if residual is not None else 0
    dtype = x.dtype if dtype is None else dtype
    if dtype not in (x.dtype, _BF16):
        raise PSGDError(f"dtype must be {_name(x.dtype)} or bfloat16, not {dtype}")
    if not eps >= 0:
        raise PSGDError(f"eps must not be negative: {eps}")
    _no_graph("layer_norm_forward", (x, weight, bias, residual), "layer_norm_backward makes the gradients", 3)
    at = _here(dev, stream)
    if at is None:
        with _there(dev, stream, x, weight, bias, residual), torch.no_grad():
            return layer_norm_forward(x, weight, bias, residual, eps, center, keep, dtype)
    y = _like(x, T, F) if dtype == x.dtype else _empty((T, F), dtype=dtype, device=dev)
    s = _like(x, T, F) if residual is not None else None
    rstd = _empty(T, dtype=torch.float32, device=dev)
    mean = _empty_like(rstd) if center else None
    kept = ActivationCheckpoint(T, F, dev) if keep else None
    _check(lib().psgd_norm_forward(x.data_ptr(), ldx, _DTYPES[x.dtype], residual.data_ptr() if residual is not None else None, ldr, at_w, at_b, w_type, eps, int(center), T, F,
                                   s.data_ptr() if s is not None else None, F, y.data_ptr(), F, _DTYPES[dtype], mean.data_ptr() if center else None, rstd.data_ptr(),
                                   kept._q if keep else None, kept._s if keep else None, at))
    return LayerNorm(y, x if s is None else s, mean, rstd, kept)


def layer_norm_backward(dy, x, weight, mean, rstd, d_x=None, bias=False, stream=None):
    """Gradients of layer_norm_forward from dy [T, F] (y's type) and the forward pass's x, mean (None: without centring) and rstd.

    `d_x` [T, F] (x's type): what reaches x from elsewhere, as around the layers of a residual path; it is added.  Returns (d_x, d_weight, d_bias): d_x in x's type is
    the gradient of x and of the residual alike, d_weight and d_bias (None unless `bias`) float32 [F], summed in a fixed order.
    """
    if stream is None:
        r = _plain().norm_backward(dy, x, weight, mean, rstd, d_x, bias)
        if type(r) is tuple:
            return LayerNormGrad(*r)
        if r is not None:
            _check(r)
    T, F, ldx = _matrix(x, "x", _BOTH)
    dev = x.device
    lddy = _matrix(dy, "dy", (_BF16,) if x.dtype == _BF16 else _BOTH, (T, F), dev)[2]
    at_w, w_type = _param(weight, "weight", F, dev)
    at_mean = _vector(mean, "mean", torch.float32, T, dev) if mean is not None else None
    at_rstd = _vector(rstd, "rstd", torch.float32, T, dev)
    lda = _matrix(d_x, "d_x", (x.dtype,), (T, F), dev)[2] if d_x is not None else 0
    at = _here(dev, stream)
    if at is None:
        with _there(dev, stream, dy, x, weight, mean, rstd, d_x):
            return layer_norm_backward(dy, x, weight, mean, rstd, d_x, bias)
    nbytes = _workspace_bytes("psgd_norm_workspace", T, F, dev.index)
    ws = _empty(nbytes, dtype=torch.uint8, device=dev)
    out = _like(x, T, F)
    dw = _empty(F, dtype=torch.float32, device=dev)
    db = _empty_like(dw) if bias else None
    _check(lib().psgd_norm_backward(dy.data_ptr(), lddy, _DTYPES[dy.dtype], x.data_ptr(), ldx, _DTYPES[x.dtype], at_w, w_type, at_mean, at_rstd,
                                    d_x.data_ptr() if d_x is not None else None, lda, T, F, out.data_ptr(), F, dw.data_ptr(), db.data_ptr() if bias else None,
                                    ws.data_ptr(), nbytes, at))
    return LayerNormGrad(out, dw, db)


# ---- rotary positions ---------------------------------------------------------------------------------------------
def rotary_frequencies(rotated, base=10000.0, factor=1.0, original_length=None, low=1.0, high=4.0, device="cuda"):
    """Radians per position of the rotated/2 pairs, float64: f_i = base^(-2i/rotated), slowed down for contexts `factor` times as long.

    Without `original_length` every frequency is divided by `factor` (positions interpolated).  With it, the length that the model was trained on, by parts: a pair that makes
    at least `high` turns over that length keeps its frequency, one that makes at most `low` is divided by `factor`, between them the share of the former
    grows linearly with the number of turns.
    """
    if rotated < 2 or rotated % 2:
        raise PSGDError(f"rotated must be even and at least 2, not {rotated}")
    if not (base > 0 and factor > 0 and math.isfinite(base) and math.isfinite(factor)) or (original_length is not None and not (original_length > 0 and low < high)):
        raise PSGDError("base, factor and original_length must be positive, low less than high")
    f = []
    for i in range(0, rotated, 2):
        fast = base ** (-i / rotated)
        share = 0.0 if original_length is None else min(1.0, max(0.0, (original_length * fast / (2 * math.pi) - low) / (high - low)))
        f.append(fast * (share + (1.0 - share) / factor))
    return torch.tensor(f, dtype=torch.float64, device=device)


def _heads(t, name, like=None):
    """(T, heads, head, token stride, head stride) of a CUDA tensor [T, heads, head] with unit stride within a head."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise PSGDError(f"{name} must be a CUDA tensor")
    if t.dtype not in _DTYPES or (like is not None and t.dtype != like.dtype):
        raise PSGDError(f"{name} must be {'float32 or bfloat16' if like is None else _name(like.dtype)}, not {_name(t.dtype)}")
    if t.ndim != 3 or (like is not None and (t.shape[0] != like.shape[0] or t.shape[2] != like.shape[2])):
        raise PSGDError(f"{name} must have shape {'(tokens, heads, head)' if like is None else (like.shape[0], 'heads', like.shape[2])}, not {tuple(t.shape)}")
    if like is not None and t.get_device() != like.get_device():
        raise PSGDError(f"{name} is on {t.device}, expected {like.device}")
    T, H, D = t.shape
    token, head, one = t.stride()
    if D < 2 or one != 1:
        raise PSGDError(f"{name} must have heads of at least two values with unit stride")
    return T, H, D, token, head


def _heads_like(t):
    """A new tensor of t's shape and type without gaps, tokens and heads in t's order, and its strides."""
    out = _empty_like(t)
    token, head, one = out.stride()
    if one != 1:                                    # (values used several times in an order that mixes)
        out = _empty(t.shape, dtype=t.dtype, device=t.device)
        token, head, one = out.stride()
    return out, token, head


def _rotary(backward, q, k, positions, frequencies, layout, scale, in_place, stream):
    if stream is None and layout in _LAYOUTS:
        r = _plain().rotary(backward, q, k, positions, frequencies, _LAYOUTS[layout], scale, in_place)
        if type(r) is tuple:
            return r
        if r is not None:
            _check(r)
    T, H, D, qt, qh = _heads(q, "dq" if backward else "q")
    dev = q.device
    _, K, _, kt, kh = _heads(k, "dk" if backward else "k", q) if k is not None else (T, 0, D, 0, 0)
    if layout not in _LAYOUTS:
        raise PSGDError(f"layout must be one of {', '.join(_LAYOUTS)}, not {layout!r}")
    at_positions = _vector(positions, "positions", torch.int64, T, dev)
    if not isinstance(frequencies, torch.Tensor) or not 1 <= frequencies.numel() <= D // 2:
        raise PSGDError(f"frequencies must be a tensor of 1 to {D // 2} values")
    R = 2 * frequencies.numel()
    at_frequencies = _vector(frequencies, "frequencies", torch.float64, R // 2, dev)
    if not backward:
        _no_graph("rotary_forward", (q, k, frequencies), "rotary_backward makes the gradients", 4)
    at = _here(dev, stream)
    if at is None:
        with _there(dev, stream, q, k, positions, frequencies), torch.no_grad():
            return _rotary(backward, q, k, positions, frequencies, layout, scale, in_place, None)
    if in_place:
        oq, ok, oqt, oqh, okt, okh = q, k, qt, qh, kt, kh
    else:
        oq, oqt, oqh = _heads_like(q)
        ok, okt, okh = _heads_like(k) if k is not None else (None, 0, 0)
    none = k is None or K == 0
    _check(lib().psgd_rotary(q.data_ptr(), qt, qh, H, oq.data_ptr(), oqt, oqh, None if none else k.data_ptr(), kt, kh, K, None if none else ok.data_ptr(), okt, okh,
                             at_positions, at_frequencies, T, D, R, _LAYOUTS[layout], int(backward), scale, _DTYPES[q.dtype], at))
    if in_place:
        _written(q, k)
    return oq, ok


def rotary_forward(q, k, positions, frequencies, layout="half", scale=1.0, in_place=False, stream=None):
    """Queries q [T, heads, head] and keys k [T, key heads, head] (or None) with the pairs of every head turned by position * frequency; returns (q, k).

    bfloat16 or float32 with unit stride within a head; tokens and heads may have any strides (parts of one projection's result, tokens or heads first).  positions [T]
    int64; frequencies [R/2] float64 radians per position (rotary_frequencies), R <= head: the values behind the first R pass through.  layout "half": pairs
    (i, i + R/2); "interleaved": (2i, 2i + 1).  `scale` multiplies what is turned.  Angles are formed in 64 bits, so that far positions keep theirs.
    in_place: q and k themselves are overwritten (which autograd is told of, as by any operator that works in place), else the results are new tensors without gaps,
    tokens and heads in the order in which the inputs have them.
    """
    return _rotary(False, q, k, positions, frequencies, layout, scale, in_place, stream)


def rotary_backward(dq, dk, positions, frequencies, layout="half", scale=1.0, in_place=False, stream=None):
    """The gradients of rotary_forward's inputs from those of its results: the same with the angles turned back."""
    return _rotary(True, dq, dk, positions, frequencies, layout, scale, in_place, stream)
