"""Training operators around the compressor: where the weight gradients that it takes come from.

  linear_cross_entropy, linear_cross_entropy_grad    softmax cross entropy of the last layer without its logits, and its gradients
  linear_distillation, linear_distillation_grad      the last layer's distance from a teacher's top logits, likewise
  pack_activation, ActivationCheckpoint.unpack       activations kept in 8 bits between the forward and the backward pass
  weight_gradient                                    a linear layer's weight gradient from the 8-bit checkpoint of its input
  swiglu_forward, swiglu_backward                    the gated unit of a feed-forward block, its inputs kept in 8 bits

Weight gradients can be written straight into a slot of a compressor's gradient stack G [count, N, m, n] (`out=G[c, i]`, float32 or bfloat16;
`d_weight=G[c, i]` of the last layer, a bfloat16 stack: `grad_dtype="bfloat16"`).  The arithmetic runs in the CUDA library (psgd_xent_*, psgd_distill_*, psgd_act_*, psgd_swiglu_* of include/psgd.h); this module checks
arguments and hands over pointers.  Every call is stream-ordered on `stream` (default: the current stream) and does not
synchronise.  `status`, an int32 tensor with one element, collects the library's warning bits (PSGD_W_TIMEOUT, PSGD_W_LABEL); what a wait
that ran out should have produced is NaN, with or without `status`.

None of these calls takes part in autograd: gradients are results of their own (d_hidden, d_weight, swiglu_backward, weight_gradient), and what a call returns has no
graph behind it.  linear_cross_entropy, linear_distillation and swiglu_forward, whose results could be taken for differentiable ones, warn where an input requires a gradient.
Tensors of the caller's that a call writes results into (`out`, `d_hidden`, `d_weight`) count for autograd as changed in place.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import warnings
from collections import namedtuple
from functools import lru_cache

import torch

from . import binding
from .binding import PSGDError, lib

PSGD_W_LABEL = 8
GROUP = 32
_MOST_ENTRIES = 1024           # of a token's teacher
_BF16 = torch.bfloat16
_DTYPES = {torch.float32: 0, torch.bfloat16: 1}
_BOTH = tuple(_DTYPES)

CrossEntropy = namedtuple("CrossEntropy", "loss token_loss lse")
CrossEntropyGrad = namedtuple("CrossEntropyGrad", "loss token_loss lse d_hidden d_weight")
Distillation = namedtuple("Distillation", "loss token_loss lse")
DistillationGrad = namedtuple("DistillationGrad", "loss token_loss lse d_hidden d_weight")

_empty = torch.empty


def _check(code):
    """Raises PSGDError for a call that failed; these calls have no handle, the library keeps the text of a CUDA error per thread."""
    if code != 0:
        if code == -4:
            raise PSGDError("PSGD_E_CUDA: " + lib().psgd_training_cuda_error().decode())
        binding._check(code)


class _NoPlainCall:
    """In the place of _call.so: no call is a plain one, and all take the way through this package."""

    def __getattr__(self, name):
        return lambda *args: None


_call = None


def _plain():
    """The module behind _call.so: the plain call of an operator, or None where it is not one.  Every call works without it, with more time on the host: where it is missing, or
    compiled against another torch, a warning says so once."""
    global _call
    if _call is None:
        from . import build

        lib()
        why, module = "it is missing or compiled against another torch", None
        if build.call_fits():
            try:
                from . import _call as module
            except ImportError as e:
                why = str(e)
        if module is None:
            warnings.warn(f"_call.so cannot be used ({why}), small calls take 10 to 20 us longer: build it with `python -m paper_2509_11254_b200.build`", RuntimeWarning, stacklevel=4)
            module = _NoPlainCall()
        _call = module
    return _call


# ---- arguments ----------------------------------------------------------------------------------------------------
def _name(dtype):
    return str(dtype).replace("torch.", "")


def _matrix(t, name, dtypes=(_BF16,), shape=None, device=None):
    """Refuses what is not a CUDA matrix with unit column stride; returns (rows, columns, row stride in elements)."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise PSGDError(f"{name} must be a CUDA tensor")
    if t.dtype not in dtypes:
        raise PSGDError(f"{name} must be {' or '.join(map(_name, dtypes))}, not {_name(t.dtype)}")
    size = t.shape
    if len(size) != 2 or (shape is not None and size != shape):
        raise PSGDError(f"{name} must have shape {tuple(shape) if shape is not None else '(rows, columns)'}, not {tuple(size)}")
    rows, cols = size
    if cols < 1:
        raise PSGDError(f"{name} has no columns")
    ld, one = t.stride()
    if rows <= 1:
        ld = cols                                   # the stride of a single row is never used
    if one != 1 and cols > 1 or ld < cols:
        raise PSGDError(f"{name} must have unit column stride and rows that do not overlap")
    if device is not None and t.get_device() != device.index:
        raise PSGDError(f"{name} is on {t.device}, expected {device}")
    return rows, cols, ld


def _vector(t, name, dtype, n, device):
    """The address of a contiguous CUDA vector."""
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.shape != (n,) or not t.is_contiguous() or t.get_device() != device.index:
        raise PSGDError(f"{name} must be a contiguous {_name(dtype)} tensor of {n} elements on {device}")
    return t.data_ptr()


def _status(t, device):
    return _vector(t, "status", torch.int32, 1, device) if t is not None else None


def _stretch(t):
    """A matrix as the library's psgd_overlap takes it: address, rows, bytes per row, bytes from row to row."""
    rows, cols = t.shape
    return t.data_ptr(), rows, cols * t.element_size(), t.stride(0) * t.element_size()


def _operand(t, rows, cols, ld, stream, *outputs):
    """(tensor, row stride): `t` itself where the tensor cores' loads can read it in place (16-byte aligned rows), else a copy with padded rows.

    The library refuses outputs over the operands that it is given; over an operand that is copied they are refused here.
    """
    if t.data_ptr() % 16 == 0 and (rows <= 1 or ld % 8 == 0):
        return t, ld
    for out in outputs:
        if out is not None and lib().psgd_overlap(*_stretch(t), *_stretch(out)):
            raise PSGDError("an output overlaps an operand")
    pad = -(-cols // 8) * 8
    copy = _empty((rows, pad), dtype=t.dtype, device=t.device)
    _check(lib().psgd_copy_rows(t.data_ptr(), ld, rows, cols, copy.data_ptr(), pad, stream))
    return copy, pad


def _no_graph(name, inputs, instead, depth):
    """Warns, `depth` calls up, where autograd would lose the gradient of one of `inputs` without a word."""
    if torch.is_grad_enabled():
        for t in inputs:
            if t is not None and t.requires_grad:
                warnings.warn(f"{name}: the results have no autograd graph, no gradient will reach its inputs; {instead}, or call it under torch.no_grad()", stacklevel=depth)
                return


def _written(*tensors):
    """Tells autograd that a call has written into tensors of the caller's (None: none): whoever has saved one for its gradients then raises instead of using what it
    has become."""
    tensors = [t for t in tensors if t is not None]
    if tensors:
        torch.autograd.graph.increment_version(tensors)


# the handle of the current stream and the current device without the objects around them, where torch has it so
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _here(device, stream):
    """The current stream's handle where `device` is current and no other stream is asked for, else None."""
    return _raw_stream(device.index) if stream is None and device.index == _current_device() else None


@contextlib.contextmanager
def _there(device, stream, *inputs):
    """Makes `device` and `stream` current, so that what is allocated inside belongs to that stream; the call is then made again inside.

    The inputs may have been allocated on another stream: their memory is not given away before this stream has read them.
    """
    stream = stream if stream is not None else torch.cuda.current_stream(device)
    if stream.device != device:
        raise PSGDError(f"stream is on {stream.device}, the tensors are on {device}")
    with torch.cuda.device(device), torch.cuda.stream(stream):
        yield
        for t in inputs:
            if t is not None:
                t.record_stream(stream)


@lru_cache(maxsize=256)
def _workspace_bytes(call, *args):
    """What a workspace query of the library answers; `args` end with the device index (the answer depends on its multiprocessors)."""
    n = C.c_size_t()
    _check(getattr(lib(), call)(*args[:-1], C.byref(n)))
    return n.value


# ---- cross entropy and distillation -------------------------------------------------------------------------------
def _last_layer(grad, hidden, weight, target, token_weight, d_hidden, d_weight, status, stream):
    """target: (labels, ignore_index) or (teacher_logits, teacher_index, temperature)."""
    if len(target) == 3 and stream is None and d_hidden is None and d_weight is None and status is None:
        r = _plain().distill(grad, hidden, weight, *target, token_weight)
        if type(r) is tuple:
            return DistillationGrad(*r) if grad else Distillation(*r)
        if r is not None:
            _check(r)
    T, D, ldh = _matrix(hidden, "hidden")
    dev = hidden.device
    V, Dw, ldw = _matrix(weight, "weight", device=dev)
    if Dw != D or V < 1:
        raise PSGDError(f"weight must have shape (vocabulary, {D}), not {tuple(weight.shape)}")
    teacher = len(target) == 3
    if teacher:
        logits, index, temperature = target
        entries, K, ldl = _matrix(logits, "teacher_logits", _BOTH, device=dev)
        if not 1 <= K <= _MOST_ENTRIES or entries != T:
            raise PSGDError(f"teacher_logits must have shape ({T}, 1 to {_MOST_ENTRIES}), not {tuple(logits.shape)}")
        ldi = _matrix(index, "teacher_index", (torch.int64,), (T, K), dev)[2]
        if not 1e-3 <= temperature <= 1e3:
            raise PSGDError(f"temperature must lie within 0.001..1000, not {temperature}")
        inputs = (logits, index)
        at_target = logits.data_ptr(), ldl, _DTYPES[logits.dtype], index.data_ptr(), ldi, K, temperature
    else:
        labels, ignore_index = target
        inputs = (labels,)
        at_target = (_vector(labels, "labels", torch.int64, T, dev),)
    at_weight = _vector(token_weight, "token_weight", torch.float32, T, dev) if token_weight is not None else None
    lddh = _matrix(d_hidden, "d_hidden", shape=(T, D), device=dev)[2] if d_hidden is not None else D
    lddw = _matrix(d_weight, "d_weight", shape=(V, D), device=dev)[2] if d_weight is not None else D
    at_status = _status(status, dev)
    name = "linear_distillation" if teacher else "linear_cross_entropy"
    if not grad:
        _no_graph(name, (hidden, weight, token_weight, *inputs), f"{name}_grad returns the gradients of hidden and weight", 4)
    s = _here(dev, stream)
    if s is None:
        with _there(dev, stream, hidden, weight, *inputs, token_weight, d_hidden, d_weight, status), torch.no_grad():
            return _last_layer(grad, hidden, weight, target, token_weight, d_hidden, d_weight, status, None)
    call = "psgd_distill_" if teacher else "psgd_xent_"
    nbytes = _workspace_bytes(call + "workspace", T, V, D, *((K,) if teacher else ()), int(grad), dev.index)
    hidden, ldh = _operand(hidden, T, D, ldh, s, d_hidden, d_weight)
    weight, ldw = _operand(weight, V, D, ldw, s, d_hidden, d_weight)
    ws = _empty(nbytes, dtype=torch.uint8, device=dev)
    out = _empty(2 * T + 1, dtype=torch.float32, device=dev)
    at = out.data_ptr()                             # token_loss, lse, loss side by side
    args = hidden.data_ptr(), ldh, weight.data_ptr(), ldw, *at_target, at_weight, *(() if teacher else (ignore_index,)), T, V, D, at + 8 * T, at, at + 4 * T
    given = d_hidden, d_weight
    if grad:
        if d_hidden is None:
            d_hidden = _empty((T, D), dtype=_BF16, device=dev)
        if d_weight is None:
            d_weight = _empty((V, D), dtype=_BF16, device=dev)
        args += d_hidden.data_ptr(), lddh, d_weight.data_ptr(), lddw
    _check(getattr(lib(), call + ("grad" if grad else "loss"))(*args, at_status, ws.data_ptr(), nbytes, s))
    _written(*given)
    token_loss, lse, loss = out.split_with_sizes((T, T, 1))
    loss = loss.view(())
    if grad:
        return (DistillationGrad if teacher else CrossEntropyGrad)(loss, token_loss, lse, d_hidden, d_weight)
    return (Distillation if teacher else CrossEntropy)(loss, token_loss, lse)


def linear_cross_entropy(hidden, weight, labels, token_weight=None, ignore_index=-100, status=None, stream=None):
    """Softmax cross entropy of logits hidden @ weight.T, which are never stored.

    hidden [T, D] and weight [V, D] bfloat16, labels [T] int64, token_weight [T] float32 or None.  Returns (loss, token_loss, lse):
    the weighted mean over the rows whose label is not `ignore_index` (0 if there is none), the loss of every row (0 where
    ignored) and every row's log-sum-exp, float32.  A label outside 0..V-1 gives NaN and sets PSGD_W_LABEL.
    """
    return _last_layer(False, hidden, weight, (labels, ignore_index), token_weight, None, None, status, stream)


def linear_cross_entropy_grad(hidden, weight, labels, token_weight=None, ignore_index=-100, d_hidden=None, d_weight=None, status=None, stream=None):
    """The same with the gradients of the loss: returns (loss, token_loss, lse, d_hidden [T, D], d_weight [V, D]), the gradients bfloat16.

    The gradients of the logits, too, are rounded to bfloat16 before the two products that make these from them, whose sums are float32.
    d_hidden, d_weight: where to write them (bfloat16 matrices with unit column stride), for instance a slot of a bfloat16 gradient stack; they may not overlap
    `hidden`, `weight`, `labels`, `token_weight` or each other.
    """
    return _last_layer(True, hidden, weight, (labels, ignore_index), token_weight, d_hidden, d_weight, status, stream)


def linear_distillation(hidden, weight, teacher_logits, teacher_index, temperature=1.0, token_weight=None, status=None, stream=None):
    """How far the last layer's probabilities are from a teacher's of whom a few logits per token are known; logits hidden @ weight.T are never stored.

    hidden [T, D] and weight [V, D] bfloat16; teacher_logits [T, K] bfloat16 or float32, K up to 1024, of the columns teacher_index [T, K] int64; token_weight [T] float32 or
    None.  With p = softmax(logits / temperature) over the vocabulary and q = softmax(teacher_logits / temperature) over a token's entries, token_loss is
    temperature^2 sum q (log q - log p).  An entry with a negative index or the logit -inf is none, and a token without an entry does not count (as padding).
    Returns (loss, token_loss, lse): the weighted mean over the tokens that count (0 if there is none), every token's loss and log-sum-exp of logits / temperature, float32.
    An index beyond the vocabulary gives NaN and sets PSGD_W_LABEL.
    """
    return _last_layer(False, hidden, weight, (teacher_logits, teacher_index, temperature), token_weight, None, None, status, stream)


def linear_distillation_grad(hidden, weight, teacher_logits, teacher_index, temperature=1.0, token_weight=None, d_hidden=None, d_weight=None, status=None, stream=None):
    """The same with the gradients of the loss: returns (loss, token_loss, lse, d_hidden [T, D], d_weight [V, D]), the gradients bfloat16 (and those of the logits on the way).

    d_hidden, d_weight: where to write them, as for linear_cross_entropy_grad; they may not overlap the teacher's lists either.
    """
    return _last_layer(True, hidden, weight, (teacher_logits, teacher_index, temperature), token_weight, d_hidden, d_weight, status, stream)


# ---- 8-bit activations --------------------------------------------------------------------------------------------
class ActivationCheckpoint:
    """A matrix [T, F] kept in 8 bits: `q` [T, 32 G] int8 and one power-of-two scale byte per row and group of 32 values, `scales` [T, G]."""

    __slots__ = ("shape", "device", "groups", "_buf", "_at", "_q", "_s")

    def __init__(self, T, F, device, buf=None, at=0):
        """`buf`, `at`: bytes to live in and where they start (a multiple of 32), for several checkpoints in one allocation."""
        G = -(-F // GROUP)
        self.shape, self.groups, self.device, self._at = (T, F), G, device, at
        self._buf = buf if buf is not None else _empty(T * G * (GROUP + 1), dtype=torch.uint8, device=device)     # q, then scales
        self._q = self._buf.data_ptr() + at
        self._s = self._q + T * G * GROUP

    @property
    def q(self):
        T, G = self.shape[0], self.groups
        return self._buf[self._at:self._at + T * G * GROUP].view(torch.int8).view(T, G * GROUP)

    @property
    def scales(self):
        T, G = self.shape[0], self.groups
        at = self._at + T * G * GROUP
        return self._buf[at:at + T * G].view(T, G)

    @property
    def nbytes(self):
        return self.shape[0] * self.groups * (GROUP + 1)

    def unpack(self, dtype=_BF16, out=None, stream=None):
        """The values that the checkpoint stands for (exact in either type), [T, F]."""
        T, F = self.shape
        ld = F
        if out is not None:
            ld = _matrix(out, "out", _BOTH, self.shape, self.device)[2]
        elif dtype not in _DTYPES:
            raise PSGDError("dtype must be float32 or bfloat16")
        s = _here(self.device, stream)
        if s is None:
            with _there(self.device, stream, self._buf, out):
                return self.unpack(dtype, out)
        given = out
        if out is None:
            out = _empty((T, F), dtype=dtype, device=self.device)
        _check(lib().psgd_act_unpack(self._q, self._s, T, F, out.data_ptr(), ld, _DTYPES[out.dtype], s))
        _written(given)
        return out


def pack_activation(x, stream=None):
    """x [T, F] (bfloat16 or float32) in 8 bits: an ActivationCheckpoint."""
    T, F, ld = _matrix(x, "x", _BOTH)
    s = _here(x.device, stream)
    if s is None:
        with _there(x.device, stream, x):
            return pack_activation(x)
    kept = ActivationCheckpoint(T, F, x.device)
    _check(lib().psgd_act_pack(x.data_ptr(), ld, _DTYPES[x.dtype], T, F, kept._q, kept._s, s))
    return kept


def _kept(c, name, device, shape=None):
    if not isinstance(c, ActivationCheckpoint):
        raise PSGDError(f"{name} must be an ActivationCheckpoint")
    if c.device != device or (shape is not None and c.shape != shape):
        raise PSGDError(f"{name} does not match the other arguments' shape or device")


def weight_gradient(dy, kept, dtype=torch.float32, out=None, status=None, stream=None):
    """dy.T @ x for dy [T, O] bfloat16 and the checkpoint of x [T, F]: the weight gradient [O, F] of y = x W.T.

    float32 sums of exact products, written as `dtype` (float32 or bfloat16) or into `out` (for instance a slot of a gradient stack), which may not overlap dy.
    """
    T, O, ldy = _matrix(dy, "dy")
    dev = dy.device
    _kept(kept, "kept", dev)
    if kept.shape[0] != T:
        raise PSGDError(f"dy has {T} rows, the checkpoint {kept.shape[0]}")
    F = ldo = kept.shape[1]
    if out is not None:
        ldo = _matrix(out, "out", _BOTH, (O, F), dev)[2]
    elif dtype not in _DTYPES:
        raise PSGDError("dtype must be float32 or bfloat16")
    at_status = _status(status, dev)
    s = _here(dev, stream)
    if s is None:
        with _there(dev, stream, dy, kept._buf, out, status):
            return weight_gradient(dy, kept, dtype, out, status)
    nbytes = _workspace_bytes("psgd_act_wgrad_workspace", T, O, F, dev.index)
    dy, ldy = _operand(dy, T, O, ldy, s, out)
    ws = _empty(nbytes, dtype=torch.uint8, device=dev)
    given = out
    if out is None:
        out = _empty((O, F), dtype=dtype, device=dev)
    _check(lib().psgd_act_wgrad(dy.data_ptr(), ldy, kept._q, kept._s, T, O, F, out.data_ptr(), ldo, _DTYPES[out.dtype], at_status, ws.data_ptr(), nbytes, s))
    _written(given)
    return out


def swiglu_forward(gate, up, stream=None):
    """h = silu(gate) * up, [T, F] bfloat16.  Returns (h, checkpoint of gate, checkpoint of up), made in one pass."""
    T, F, ldg = _matrix(gate, "gate")
    dev = gate.device
    ldu = _matrix(up, "up", shape=(T, F), device=dev)[2]
    _no_graph("swiglu_forward", (gate, up), "swiglu_backward makes the gradients", 3)
    s = _here(dev, stream)
    if s is None:
        with _there(dev, stream, gate, up), torch.no_grad():
            return swiglu_forward(gate, up)
    h = _empty((T, F), dtype=_BF16, device=dev)
    size = -(-T * -(-F // GROUP) * (GROUP + 1) // 256) * 256
    kg = ActivationCheckpoint(T, F, dev, _empty(2 * size, dtype=torch.uint8, device=dev))      # they are kept and used together
    ku = ActivationCheckpoint(T, F, dev, kg._buf, size)
    _check(lib().psgd_swiglu_forward(gate.data_ptr(), ldg, up.data_ptr(), ldu, T, F, h.data_ptr(), F, kg._q, kg._s, ku._q, ku._s, s))
    return h, kg, ku


def swiglu_backward(dh, gate, up, recompute=False, stream=None):
    """Gradients (d_gate, d_up) of h = silu(gate) * up from dh [T, F] bfloat16 and the two checkpoints; with `recompute` also h again."""
    T, F, ld = _matrix(dh, "dh")
    dev = dh.device
    _kept(gate, "gate", dev, (T, F))
    _kept(up, "up", dev, (T, F))
    s = _here(dev, stream)
    if s is None:
        with _there(dev, stream, dh, gate._buf, up._buf):
            return swiglu_backward(dh, gate, up, recompute)
    d_gate = _empty((T, F), dtype=_BF16, device=dev)
    d_up = torch.empty_like(d_gate)
    h = torch.empty_like(d_gate) if recompute else None
    _check(lib().psgd_swiglu_backward(dh.data_ptr(), ld, gate._q, gate._s, up._q, up._s, T, F, d_gate.data_ptr(), F, d_up.data_ptr(), F,
                                      h.data_ptr() if recompute else None, F, s))
    return (d_gate, d_up, h) if recompute else (d_gate, d_up)
