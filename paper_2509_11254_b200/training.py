"""Training operators around the compressor: where the weight gradients that it takes come from.

  linear_cross_entropy, linear_cross_entropy_grad    softmax cross entropy of the last layer without its logits, and its gradients
  pack_activation, ActivationCheckpoint.unpack       activations kept in 8 bits between the forward and the backward pass
  weight_gradient                                    a linear layer's weight gradient from the 8-bit checkpoint of its input
  swiglu_forward, swiglu_backward                    the gated unit of a feed-forward block, its inputs kept in 8 bits

Weight gradients can be written straight into a slot of a compressor's gradient stack G [count, N, m, n] (`d_weight=G[c, i]`,
`out=G[c, i]`).  The arithmetic runs in the CUDA library (psgd_xent_*, psgd_act_*, psgd_swiglu_* of include/psgd.h); this module checks
arguments and hands over pointers.  Every call is stream-ordered on `stream` (default: the current stream) and does not
synchronise.  `status`, an int32 tensor with one element, collects the library's warning bits (PSGD_W_TIMEOUT, PSGD_W_LABEL).
"""
from __future__ import annotations

import contextlib
import ctypes as C
from collections import namedtuple

import torch

from .binding import PSGDError, _check, lib

PSGD_W_LABEL = 8
GROUP = 32
_DTYPES = {torch.float32: 0, torch.bfloat16: 1}

CrossEntropy = namedtuple("CrossEntropy", "loss token_loss lse")
CrossEntropyGrad = namedtuple("CrossEntropyGrad", "loss token_loss lse d_hidden d_weight")


# ---- arguments ----------------------------------------------------------------------------------------------------
def _matrix(t, name, dtypes=(torch.bfloat16,), shape=None, device=None):
    """A CUDA matrix with unit column stride; returns it."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise PSGDError(f"{name} must be a CUDA tensor")
    if t.dtype not in dtypes:
        raise PSGDError(f"{name} must be {' or '.join(str(d).replace('torch.', '') for d in dtypes)}, not {str(t.dtype).replace('torch.', '')}")
    if t.dim() != 2 or (shape is not None and tuple(t.shape) != tuple(shape)):
        raise PSGDError(f"{name} must have shape {tuple(shape) if shape is not None else '(rows, columns)'}, not {tuple(t.shape)}")
    if t.shape[1] < 1:
        raise PSGDError(f"{name} has no columns")
    if t.stride(1) != 1 and t.shape[1] > 1 or (t.shape[0] > 1 and t.stride(0) < t.shape[1]):
        raise PSGDError(f"{name} must have unit column stride and rows that do not overlap")
    if device is not None and t.device != device:
        raise PSGDError(f"{name} is on {t.device}, expected {device}")
    return t


def _vector(t, name, dtype, n, device):
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype != dtype or t.shape != (n,) or not t.is_contiguous() or t.device != device:
        raise PSGDError(f"{name} must be a contiguous {str(dtype).replace('torch.', '')} tensor of {n} elements on {device}")
    return t


def _status(t, device):
    return _vector(t, "status", torch.int32, 1, device).data_ptr() if t is not None else None


def _ld(t):
    """Row stride in elements (of a single row: its length)."""
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _operand(t):
    """`t` itself where the tensor cores' loads can read it in place (16-byte aligned rows), else a copy with padded rows."""
    if t.data_ptr() % 16 == 0 and (t.shape[0] <= 1 or t.stride(0) % 8 == 0):
        return t
    rows, cols = t.shape
    return torch.empty((rows, -(-cols // 8) * 8), dtype=t.dtype, device=t.device)[:, :cols].copy_(t)


@contextlib.contextmanager
def _on_other(device, stream):
    with torch.cuda.device(device), torch.cuda.stream(stream):
        yield C.c_void_p(stream.cuda_stream)


class _OnCurrent:
    """The common case without the cost of switching: the tensor's device is current and so is its stream."""

    def __init__(self, stream):
        self.ptr = C.c_void_p(stream)

    def __enter__(self):
        return self.ptr

    def __exit__(self, *a):
        return False


def _on(device, stream):
    """Makes `device` and `stream` current, so that what is allocated inside belongs to that stream."""
    if stream is None:
        if device.index == torch.cuda.current_device():
            return _OnCurrent(torch.cuda.current_stream(device).cuda_stream)
        stream = torch.cuda.current_stream(device)
    return _on_other(device, stream)


# ---- cross entropy ------------------------------------------------------------------------------------------------
def _xent(grad, hidden, weight, labels, token_weight, ignore_index, d_hidden, d_weight, status, stream):
    _matrix(hidden, "hidden")
    T, D = hidden.shape
    dev = hidden.device
    _matrix(weight, "weight", device=dev)
    if weight.shape[1] != D or weight.shape[0] < 1:
        raise PSGDError(f"weight must have shape (vocabulary, {D}), not {tuple(weight.shape)}")
    V = weight.shape[0]
    _vector(labels, "labels", torch.int64, T, dev)
    if token_weight is not None:
        _vector(token_weight, "token_weight", torch.float32, T, dev)
    if d_hidden is not None:
        _matrix(d_hidden, "d_hidden", shape=(T, D), device=dev)
    if d_weight is not None:
        _matrix(d_weight, "d_weight", shape=(V, D), device=dev)
    st = _status(status, dev)
    L = lib()
    nbytes = C.c_size_t()
    with _on(dev, stream) as s:
        _check(L.psgd_xent_workspace(T, V, D, int(grad), C.byref(nbytes)))
        hidden, weight = _operand(hidden), _operand(weight)
        ws = torch.empty((nbytes.value,), dtype=torch.uint8, device=dev)
        rows = torch.empty((2, T), dtype=torch.float32, device=dev)
        loss = torch.empty((), dtype=torch.float32, device=dev)
        token_loss, lse = rows[0], rows[1]
        args = [hidden.data_ptr(), _ld(hidden), weight.data_ptr(), _ld(weight), labels.data_ptr(), token_weight.data_ptr() if token_weight is not None else None,
                ignore_index, T, V, D, loss.data_ptr(), token_loss.data_ptr(), lse.data_ptr()]
        if not grad:
            _check(L.psgd_xent_loss(*args, st, ws.data_ptr(), nbytes.value, s))
            return CrossEntropy(loss, token_loss, lse)
        if d_hidden is None:
            d_hidden = torch.empty((T, D), dtype=torch.bfloat16, device=dev)
        if d_weight is None:
            d_weight = torch.empty((V, D), dtype=torch.bfloat16, device=dev)
        _check(L.psgd_xent_grad(*args, d_hidden.data_ptr(), _ld(d_hidden), d_weight.data_ptr(), _ld(d_weight), st, ws.data_ptr(), nbytes.value, s))
        return CrossEntropyGrad(loss, token_loss, lse, d_hidden, d_weight)


def linear_cross_entropy(hidden, weight, labels, token_weight=None, ignore_index=-100, status=None, stream=None):
    """Softmax cross entropy of logits hidden @ weight.T, which are never stored.

    hidden [T, D] and weight [V, D] bfloat16, labels [T] int64, token_weight [T] float32 or None.  Returns (loss, token_loss, lse):
    the weighted mean over the rows whose label is not `ignore_index` (0 if there is none), the loss of every row (0 where
    ignored) and every row's log-sum-exp, float32.  A label outside 0..V-1 gives NaN and sets PSGD_W_LABEL.
    """
    return _xent(False, hidden, weight, labels, token_weight, ignore_index, None, None, status, stream)


def linear_cross_entropy_grad(hidden, weight, labels, token_weight=None, ignore_index=-100, d_hidden=None, d_weight=None, status=None, stream=None):
    """The same with the gradients of the loss: returns (loss, token_loss, lse, d_hidden [T, D], d_weight [V, D]), the gradients bfloat16.

    d_hidden, d_weight: where to write them (matrices with unit column stride), for instance a slot of a gradient stack.
    """
    return _xent(True, hidden, weight, labels, token_weight, ignore_index, d_hidden, d_weight, status, stream)


# ---- 8-bit activations --------------------------------------------------------------------------------------------
class ActivationCheckpoint:
    """A matrix [T, F] kept in 8 bits: `q` [T, 32 G] int8 and one power-of-two scale byte per row and group of 32 values, `scales` [T, G]."""

    __slots__ = ("q", "scales", "shape")

    def __init__(self, T, F, device):
        G = -(-F // GROUP)
        self.shape = (T, F)
        self.q = torch.empty((T, G * GROUP), dtype=torch.int8, device=device)
        self.scales = torch.empty((T, G), dtype=torch.uint8, device=device)

    @property
    def device(self):
        return self.q.device

    @property
    def nbytes(self):
        return self.q.numel() + self.scales.numel()

    def unpack(self, dtype=torch.bfloat16, out=None, stream=None):
        """The values that the checkpoint stands for (exact in either type), [T, F]."""
        if out is None and dtype not in _DTYPES:
            raise PSGDError("dtype must be float32 or bfloat16")
        if out is not None:
            _matrix(out, "out", tuple(_DTYPES), self.shape, self.device)
        with _on(self.device, stream) as s:
            if out is None:
                out = torch.empty(self.shape, dtype=dtype, device=self.device)
            _check(lib().psgd_act_unpack(self.q.data_ptr(), self.scales.data_ptr(), *self.shape, out.data_ptr(), _ld(out), _DTYPES[out.dtype], s))
        return out


def pack_activation(x, stream=None):
    """x [T, F] (bfloat16 or float32) in 8 bits: an ActivationCheckpoint."""
    _matrix(x, "x", tuple(_DTYPES))
    T, F = x.shape
    with _on(x.device, stream) as s:
        kept = ActivationCheckpoint(T, F, x.device)
        _check(lib().psgd_act_pack(x.data_ptr(), _ld(x), _DTYPES[x.dtype], T, F, kept.q.data_ptr(), kept.scales.data_ptr(), s))
    return kept


def _kept(c, name, device=None, shape=None):
    if not isinstance(c, ActivationCheckpoint):
        raise PSGDError(f"{name} must be an ActivationCheckpoint")
    if (device is not None and c.device != device) or (shape is not None and tuple(c.shape) != tuple(shape)):
        raise PSGDError(f"{name} does not match the other arguments' shape or device")
    return c


def weight_gradient(dy, kept, dtype=torch.float32, out=None, status=None, stream=None):
    """dy.T @ x for dy [T, O] bfloat16 and the checkpoint of x [T, F]: the weight gradient [O, F] of y = x W.T.

    float32 sums of exact products, written as `dtype` (float32 or bfloat16) or into `out` (for instance a slot of a gradient stack).
    """
    _matrix(dy, "dy")
    T, O = dy.shape
    dev = dy.device
    _kept(kept, "kept", dev)
    if kept.shape[0] != T:
        raise PSGDError(f"dy has {T} rows, the checkpoint {kept.shape[0]}")
    F = kept.shape[1]
    if out is not None:
        _matrix(out, "out", tuple(_DTYPES), (O, F), dev)
    elif dtype not in _DTYPES:
        raise PSGDError("dtype must be float32 or bfloat16")
    st = _status(status, dev)
    L = lib()
    nbytes = C.c_size_t()
    with _on(dev, stream) as s:
        _check(L.psgd_act_wgrad_workspace(T, O, F, C.byref(nbytes)))
        dy = _operand(dy)
        ws = torch.empty((nbytes.value,), dtype=torch.uint8, device=dev)
        if out is None:
            out = torch.empty((O, F), dtype=dtype, device=dev)
        _check(L.psgd_act_wgrad(dy.data_ptr(), _ld(dy), kept.q.data_ptr(), kept.scales.data_ptr(), T, O, F, out.data_ptr(), _ld(out), _DTYPES[out.dtype], st,
                                ws.data_ptr(), nbytes.value, s))
    return out


def swiglu_forward(gate, up, stream=None):
    """h = silu(gate) * up, [T, F] bfloat16.  Returns (h, checkpoint of gate, checkpoint of up), made in one pass."""
    _matrix(gate, "gate")
    T, F = gate.shape
    dev = gate.device
    _matrix(up, "up", shape=(T, F), device=dev)
    with _on(dev, stream) as s:
        h = torch.empty((T, F), dtype=torch.bfloat16, device=dev)
        kg, ku = ActivationCheckpoint(T, F, dev), ActivationCheckpoint(T, F, dev)
        _check(lib().psgd_swiglu_forward(gate.data_ptr(), _ld(gate), up.data_ptr(), _ld(up), T, F, h.data_ptr(), F, kg.q.data_ptr(), kg.scales.data_ptr(),
                                         ku.q.data_ptr(), ku.scales.data_ptr(), s))
    return h, kg, ku


def swiglu_backward(dh, gate, up, recompute=False, stream=None):
    """Gradients (d_gate, d_up) of h = silu(gate) * up from dh [T, F] bfloat16 and the two checkpoints; with `recompute` also h again."""
    _matrix(dh, "dh")
    T, F = dh.shape
    dev = dh.device
    _kept(gate, "gate", dev, (T, F))
    _kept(up, "up", dev, (T, F))
    with _on(dev, stream) as s:
        out = [torch.empty((T, F), dtype=torch.bfloat16, device=dev) for _ in range(3 if recompute else 2)]
        _check(lib().psgd_swiglu_backward(dh.data_ptr(), _ld(dh), gate.q.data_ptr(), gate.scales.data_ptr(), up.q.data_ptr(), up.scales.data_ptr(), T, F,
                                          out[0].data_ptr(), F, out[1].data_ptr(), F, out[2].data_ptr() if recompute else None, F, s))
    return tuple(out)
