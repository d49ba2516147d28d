"""Worker-batched layers on torch tensors: the operators declared in
include/cpdp_layers.h, which make the gradients that ``CPDPState`` steps with.

- ``add_rmsnorm`` / ``add_rmsnorm_backward``: residual addition and
  root-mean-square norm, its output optionally held in 8 bits
- ``checkpoint`` / ``restore`` / ``weight_gradient``: activations held in 8 bits
  for the backward pass, and the weight gradient that reads them
- ``gated_recurrence`` / ``gated_recurrence_backward`` /
  ``gated_recurrence_step``: h_t = a_t h_(t-1) + (1 - a_t) v_t, a = sigmoid(gate)
- ``linear_cross_entropy`` / ``linear_cross_entropy_backward``: softmax cross
  entropy over a vocabulary, from the activations and the head's weight
- ``causal_conv`` / ``causal_conv_backward`` / ``causal_conv_step``: a short
  convolution over time for each channel, and its silu
- ``selective_scan`` / ``selective_scan_backward`` / ``selective_scan_step``: a
  state space with some states per channel, whose step size, input and output
  weights depend on the token
- ``clip_gradients``: the norms of the workers' gradient rows, and the rows
  scaled down to a largest norm

Activations are (W, M, D): W workers, M tokens each, D features, contiguous
along D, float32 or bfloat16. One model's (M, D) is taken too, with a weight
(D,). Weights are float32 and may be slices of ``CPDPState.params`` (the head's,
which the loss takes, has the activations' type instead: a bfloat16 model casts
its slice), and weight gradients are written into slices of the [W][N] gradient
buffer::

    weight = st.params[:, a:a + D]                          # (W, D)
    y, s, saved = layers.add_rmsnorm(x, weight, residual, checkpoint=True)
    ...
    layers.weight_gradient(dy, saved, out=grads[:, b:b + O * D].view(W, O, D))
    dx, _ = layers.add_rmsnorm_backward(dy, s, weight, ds, dweight=grads[:, a:a + D])

Calls run on the current stream of their tensors' device (or on ``stream``) and
return without waiting. Outputs are allocated by torch; nothing is kept between
calls. There is no autograd (tensors that require a gradient are refused where
gradients are recorded; inside an autograd.Function they are not) and no CPU
implementation. A tensor that a call cannot take is refused with ValueError or
TypeError, anything that the library refuses with ``CPDPError``.
"""
from __future__ import annotations

import ctypes
import math
import struct
from dataclasses import dataclass

import torch

from . import cpdp as _c
from .state import _raw_stream

BLOCK = 32  # features that share an exponent
MAX_SIZE = 1 << 30  # of every axis
CARRY_STEPS = 16  # CPDP_CARRY_STEPS
CONV_MAX_TAPS = 4  # CPDP_CONV_MAX_TAPS
SCAN_MAX_STATES = 32  # CPDP_SCAN_MAX_STATES
NORM_MAX_FEATURES = 16384  # CPDP_NORM_MAX_FEATURES

_P, _I, _L, _F, _Z = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
# Every entry point declared in include/cpdp_layers.h: (result, arguments).
SIGNATURES = {
    "cpdp_add_rmsnorm": (_I, [_P, _L, _L, _P, _L, _L, _P, _L, _I, _I, _L, _I, _F, _P, _P, _P, _P, _P]),
    "cpdp_add_rmsnorm_backward_workspace": (_Z, [_I, _L, _I]),
    "cpdp_add_rmsnorm_backward": (_I, [_P, _L, _L, _P, _L, _L, _P, _L, _L, _P, _L, _I, _I, _L, _I, _F, _P, _P, _L, _I, _P,
                                       _Z, _P]),
    "cpdp_checkpoint": (_I, [_P, _L, _L, _I, _I, _L, _I, _P, _P, _P, _P]),
    "cpdp_restore": (_I, [_P, _P, _I, _L, _I, _P, _P]),
    "cpdp_weight_gradient_workspace": (_Z, [_P, _L, _L, _I, _I, _L, _I, _I]),
    "cpdp_weight_gradient": (_I, [_P, _L, _L, _I, _P, _P, _I, _L, _I, _I, _P, _L, _I, _P, _Z, _P]),
    "cpdp_gated_recurrence_workspace": (_Z, [_I, _L, _I]),
    "cpdp_gated_recurrence": (_I, [_P, _L, _L, _P, _L, _L, _I, _I, _L, _I, _P, _P, _P, _P, _P, _P, _Z, _P]),
    "cpdp_gated_recurrence_backward": (_I, [_P, _L, _L, _P, _L, _L, _P, _L, _L, _I, _I, _L, _I, _P, _P, _P, _P, _P, _L, _L,
                                            _P, _P, _Z, _P]),
    "cpdp_gated_recurrence_step": (_I, [_P, _L, _P, _L, _I, _I, _I, _P, _P, _P]),
    "cpdp_linear_cross_entropy_workspace": (_Z, [_P, _L, _L, _P, _L, _L, _I, _I, _L, _I, _I]),
    "cpdp_linear_cross_entropy": (_I, [_P, _L, _L, _P, _L, _L, _P, _I, _I, _L, _I, _I, _P, _P, _P, _Z, _P]),
    "cpdp_linear_cross_entropy_backward_workspace": (_Z, [_P, _L, _L, _P, _L, _L, _I, _I, _L, _I, _I]),
    "cpdp_linear_cross_entropy_backward": (_I, [_P, _P, _L, _L, _P, _L, _L, _P, _P, _I, _I, _L, _I, _I, _P, _P, _L, _I, _P, _Z, _P]),
    "cpdp_clip_gradients_workspace": (_Z, [_I, _L]),
    "cpdp_clip_gradients": (_I, [_P, _L, _I, _I, _L, _F, _P, _P, _L, _P, _Z, _P]),
    "cpdp_causal_conv": (_I, [_P, _L, _L, _P, _L, _P, _L, _P, _P, _I, _I, _I, _L, _I, _I, _P, _P, _P]),
    "cpdp_causal_conv_backward_workspace": (_Z, [_I, _I, _L, _I, _I]),
    "cpdp_causal_conv_backward": (_I, [_P, _L, _L, _P, _L, _L, _P, _L, _P, _L, _P, _P, _P, _I, _I, _I, _L, _I, _I, _P, _P, _P, _L, _P,
                                       _L, _I, _P, _Z, _P]),
    "cpdp_causal_conv_step": (_I, [_P, _L, _P, _L, _P, _L, _I, _I, _I, _I, _I, _P, _P, _P]),
    "cpdp_selective_scan_workspace": (_Z, [_I, _L, _I, _I]),
    "cpdp_selective_scan": (_I, [_P, _I, _I, _I, _L, _I, _I, _P, _P, _P, _P, _P, _Z, _P]),
    "cpdp_selective_scan_backward_workspace": (_Z, [_I, _L, _I, _I]),
    "cpdp_selective_scan_backward": (_I, [_P, _L, _L, _P, _I, _I, _I, _L, _I, _I, _P, _P, _P, _P, _P, _P, _P, _P, _P, _L, _P, _L, _P,
                                          _L, _I, _P, _Z, _P]),
    "cpdp_selective_scan_step": (_I, [_P, _I, _I, _I, _I, _I, _P, _P, _P]),
    "cpdp_layer_timeouts": (_I, [ctypes.POINTER(_L)]),
}

_loaded: dict = {}


def lib() -> ctypes.CDLL:
    """libcpdp with the layers' entry points declared."""
    L = _c.lib()
    if not _loaded:
        for name, (result, arguments) in SIGNATURES.items():
            f = getattr(L, name)
            f.restype, f.argtypes = result, arguments
            _loaded[name] = f
    return L


def _entry(name: str):
    """An entry point by name. A small call's cost is what Python does around
    it, so this and the checks below keep to one look at each property."""
    if not _loaded:
        lib()
    return _loaded[name]


_CODES = {torch.float32: _c.CPDP_F32, torch.bfloat16: _c.CPDP_BF16}
_F32, _BF16 = torch.float32, torch.bfloat16
# The current device's index without the checks of the public function, where torch has it.
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _dtype(t: torch.Tensor, name: str) -> int:
    code = _CODES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be float32 or bfloat16, got {t.dtype}")
    return code


def _check(status: int) -> None:
    if status:
        _c._check(status)


def _stream(index: int) -> int:
    if _raw_stream is not None:
        return _raw_stream(index)
    return torch.cuda.current_stream(index).cuda_stream


def _no_autograd(**tensors) -> None:
    """Refuses tensors whose gradient would be lost without a word."""
    for name, t in tensors.items():
        if t is not None and t.requires_grad and torch.is_grad_enabled():
            raise ValueError(f"{name} requires a gradient, which these calls do not record: detach it, or call under torch.no_grad()")


def _elsewhere(device: torch.device, stream) -> bool:
    """Whether a call runs on another device or stream than the current one."""
    return stream is not None or device.index != _current_device()


def _there(device: torch.device, stream):
    """The context in which such a call's outputs are allocated and its kernels
    launched."""
    if stream is None:
        return torch.cuda.device(device)
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device)
    elif stream.device != device:
        raise ValueError(f"the stream is one of {stream.device}, the tensors are on {device}")
    return torch.cuda.stream(stream)


def _input(t: torch.Tensor, name: str, shape: tuple, dtype: torch.dtype, device: torch.device) -> tuple:
    """The strides of an input of this shape and type, contiguous along its last axis."""
    strides = t.stride()
    if t.shape == shape and t.dtype is dtype and t.device == device and (strides[-1] == 1 or shape[-1] <= 1):
        return strides
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, not on {device}")
    raise ValueError(f"{name} must be contiguous along its last axis")


def _cuda(t: torch.Tensor, name: str) -> torch.device:
    if not t.is_cuda:
        raise ValueError(f"{name} is on {t.device}; the layers run on a CUDA device")
    return t.device


def _whole(t: torch.Tensor | None, name: str, shape: tuple, dtype: torch.dtype, device: torch.device) -> int | None:
    """The address of a contiguous array, or None where there is none."""
    if t is None:
        return None
    _input(t, name, shape, dtype, device)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _workspace(nbytes: int, device: torch.device) -> torch.Tensor | None:
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


def _ptr(t: torch.Tensor | None) -> int | None:
    return None if t is None else t.data_ptr()


@dataclass(slots=True)
class Checkpoint:
    """Activations held in 8 bits: ``codes`` int8 (W, M, 32 * ceil(D / 32)),
    ``exponents`` uint8 (W, M, ceil(D / 32)), and the number D of features.
    A value is code * 2^(exponent - 127), exact in bfloat16."""
    codes: torch.Tensor
    exponents: torch.Tensor
    features: int

    @property
    def nbytes(self) -> int:
        return self.codes.numel() + self.exponents.numel()


def _new_checkpoint(W: int, M: int, D: int, device: torch.device) -> Checkpoint:
    blocks = -(-D // BLOCK)
    return Checkpoint(torch.empty((W, M, blocks * BLOCK), dtype=torch.int8, device=device),
                      torch.empty((W, M, blocks), dtype=torch.uint8, device=device), D)


def _sized(t: torch.Tensor, name: str) -> tuple:
    """The shape of an array whose sizes the library's arguments can hold."""
    if max(t.shape) > MAX_SIZE:
        raise ValueError(f"{name} has an axis of more than {MAX_SIZE}: {tuple(t.shape)}")
    return t.shape


def _three(t: torch.Tensor, name: str) -> tuple:
    if t.dim() != 3:
        raise ValueError(f"{name} must be (W, M, D), or (M, D) of one model; got {tuple(t.shape)}")
    return _sized(t, name)


def add_rmsnorm(x, weight, residual=None, *, eps: float = 1e-6, checkpoint: bool = False, stream=None):
    """s = x + residual (rounded to x's type), y = weight * s / sqrt(mean(s^2) + eps).

    Returns (y, s, saved). Without a residual s is x itself. With ``checkpoint``
    y is held in 8 bits, ``saved`` is that Checkpoint and y is bfloat16, the
    values that it stands for: the product that follows and its weight gradient
    then see the same numbers. Else y has x's type and ``saved`` is None."""
    if x.dim() == 2 and weight.dim() == 1:
        y, s, saved = add_rmsnorm(x[None], weight[None], None if residual is None else residual[None], eps=eps,
                                  checkpoint=checkpoint, stream=stream)
        return y[0], x if residual is None else s[0], saved
    shape, dtype, device = x.shape, x.dtype, x.device
    xs, ws, code = x.stride(), weight.stride(), _CODES.get(dtype)
    # one test where all is well: a decoding step costs what Python does around it
    if not (stream is None and code is not None and x.is_cuda and device.index == _current_device() and len(shape) == 3 and max(shape) <= MAX_SIZE
            and weight.shape == (shape[0], shape[2]) and weight.dtype is _F32 and weight.device == device
            and xs[-1] == 1 == ws[-1] and not (x.requires_grad or weight.requires_grad or residual is not None and residual.requires_grad)):
        _no_autograd(x=x, weight=weight, residual=residual)
        if _elsewhere(_cuda(x, "x"), stream):
            with _there(device, stream):
                return add_rmsnorm(x, weight, residual, eps=eps, checkpoint=checkpoint)
        code = _dtype(x, "x")
        _input(x, "x", _three(x, "x"), dtype, device)
        _input(weight, "weight", (shape[0], shape[2]), _F32, device)
    W, M, D = shape
    rs = (0, 0)
    s, s_at, r_at = x, None, None
    if residual is not None:
        rs, r_at = _input(residual, "residual", shape, dtype, device), residual.data_ptr()
        s = torch.empty(shape, dtype=dtype, device=device)
        s_at = s.data_ptr()
    if checkpoint:
        saved = _new_checkpoint(W, M, D, device)
        y = torch.empty(shape, dtype=_BF16, device=device)
        codes, exponents = saved.codes.data_ptr(), saved.exponents.data_ptr()
    else:
        y = torch.empty(shape, dtype=dtype, device=device)
        saved = codes = exponents = None
    _check(_entry("cpdp_add_rmsnorm")(x.data_ptr(), xs[0], xs[1], r_at, rs[0], rs[1], weight.data_ptr(), ws[0], code, W, M, D, eps,
                                      y.data_ptr(), s_at, codes, exponents, _stream(device.index)))
    return y, s, saved


def _gradient_out(out, name: str, shape: tuple, dtype: torch.dtype, device: torch.device) -> torch.Tensor:
    """The caller's slice of the gradient rows (each worker's part contiguous), or a new tensor."""
    if out is None:
        if dtype not in _CODES:
            raise TypeError(f"{name} must be float32 or bfloat16, got {dtype}")
        return torch.empty(shape, dtype=dtype, device=device)
    _dtype(out, name)
    if tuple(out.shape) != shape or out.device != device:
        raise ValueError(f"{name} must have shape {shape} on {device}, got {tuple(out.shape)} on {out.device}")
    if not out.is_contiguous() and not out[0].is_contiguous():
        raise ValueError(f"each worker's part of {name} must be contiguous")
    if shape[0] > 1 and out.stride(0) < math.prod(shape[1:]):
        raise ValueError(f"the workers' parts of {name} overlap: worker stride {out.stride(0)}")
    return out


def _rows_apart(t: torch.Tensor, name: str) -> None:
    """Refuses an output (A, B, D) some of whose rows share memory: all of one axis's rows lie between two of the other's."""
    (A, B, D), (a, b, _) = t.shape, t.stride()
    if A > 1 and B > 1:
        (n, inner), outer = ((B, b), a) if a >= b else ((A, a), b)
        apart = inner >= D and outer >= (n - 1) * inner + D
    else:
        apart = (A <= 1 or a >= D) and (B <= 1 or b >= D)
    if not apart and t.numel():
        raise ValueError(f"rows of {name} overlap: shape {tuple(t.shape)}, strides {t.stride()}")


def add_rmsnorm_backward(dy, s, weight, ds=None, *, eps: float = 1e-6, dweight=None, dtype=torch.float32, stream=None):
    """Gradients of ``add_rmsnorm``: (dx, dweight). dy is the gradient of y and
    s what the forward pass returned as s; ds, where given, is the gradient that
    reaches s by other ways (the residual stream's) and is added to dx. dx is
    the gradient of x and of the residual. dweight is written into the tensor
    given, (W, D) float32 or bfloat16, or into a new one of ``dtype``."""
    if s.dim() == 2 and weight.dim() == 1:
        dx, dw = add_rmsnorm_backward(dy[None], s[None], weight[None], None if ds is None else ds[None], eps=eps,
                                      dweight=None if dweight is None else dweight[None], dtype=dtype, stream=stream)
        return dx[0], dw[0]
    _no_autograd(dy=dy, s=s, weight=weight, ds=ds, dweight=dweight)
    device = _cuda(s, "s")
    if _elsewhere(device, stream):
        with _there(device, stream):
            return add_rmsnorm_backward(dy, s, weight, ds, eps=eps, dweight=dweight, dtype=dtype)
    W, M, D = shape = _three(s, "s")
    kind, code = s.dtype, _dtype(s, "s")
    ss, gs = _input(s, "s", shape, kind, device), _input(dy, "dy", shape, kind, device)
    ws, ts, t_at = _input(weight, "weight", (W, D), _F32, device), (0, 0), None
    if ds is not None:
        ts, t_at = _input(ds, "ds", shape, kind, device), ds.data_ptr()
    dweight = _gradient_out(dweight, "dweight", (W, D), dtype, device)
    dx = torch.empty(shape, dtype=kind, device=device)
    needed = _entry("cpdp_add_rmsnorm_backward_workspace")(W, M, D)
    work = _workspace(needed, device)
    _check(_entry("cpdp_add_rmsnorm_backward")(
        dy.data_ptr(), gs[0], gs[1], s.data_ptr(), ss[0], ss[1], t_at, ts[0], ts[1], weight.data_ptr(), ws[0], code, W, M, D, eps,
        dx.data_ptr(), dweight.data_ptr(), dweight.stride(0), _CODES[dweight.dtype], _ptr(work), needed, _stream(device.index)))
    return dx, dweight


def checkpoint(x, *, values: bool = True, stream=None):
    """x (W, M, D) held in 8 bits: (Checkpoint, the bfloat16 values that it
    stands for). values=False: None in their place."""
    if x.dim() == 2:
        saved, held = checkpoint(x[None], values=values, stream=stream)
        return saved, held[0] if values else None
    _no_autograd(x=x)
    device = _cuda(x, "x")
    if _elsewhere(device, stream):
        with _there(device, stream):
            return checkpoint(x, values=values)
    W, M, D = shape = _three(x, "x")
    code = _dtype(x, "x")
    xs = _input(x, "x", shape, x.dtype, device)
    saved = _new_checkpoint(W, M, D, device)
    held = torch.empty(shape, dtype=_BF16, device=device) if values else None
    _check(_entry("cpdp_checkpoint")(x.data_ptr(), xs[0], xs[1], code, W, M, D, saved.codes.data_ptr(), saved.exponents.data_ptr(),
                                     _ptr(held), _stream(device.index)))
    return saved, held


def _saved(saved: Checkpoint) -> tuple[int, int, int]:
    """(W, M, D) of a Checkpoint that the library can read."""
    codes, exponents, D = saved.codes, saved.exponents, saved.features
    blocks = -(-D // BLOCK)
    device, shape = _cuda(codes, "codes"), codes.shape
    if len(shape) != 3:
        raise ValueError(f"codes must be (W, M, {blocks * BLOCK}), got {tuple(shape)}")
    W, M, P = shape
    _sized(codes, "codes")
    if not (P == blocks * BLOCK and codes.dtype is torch.int8 and exponents.dtype is torch.uint8 and exponents.shape == (W, M, blocks)
            and exponents.device == device and codes.is_contiguous() and exponents.is_contiguous()):
        _whole(codes, "codes", (W, M, blocks * BLOCK), torch.int8, device)
        _whole(exponents, "exponents", (W, M, blocks), torch.uint8, device)
    return W, M, D


def restore(saved: Checkpoint, *, stream=None):
    """The bfloat16 values (W, M, D) that a Checkpoint stands for."""
    W, M, D = _saved(saved)
    device = saved.codes.device
    if _elsewhere(device, stream):
        with _there(device, stream):
            return restore(saved)
    held = torch.empty((W, M, D), dtype=_BF16, device=device)
    _check(_entry("cpdp_restore")(saved.codes.data_ptr(), saved.exponents.data_ptr(), W, M, D, held.data_ptr(), _stream(device.index)))
    return held


def weight_gradient(dy, saved: Checkpoint, *, out=None, dtype=torch.float32, stream=None):
    """dW[w] = dy[w]^T x^[w] of a linear layer whose input the Checkpoint holds:
    dy (W, M, O), x^ (W, M, I), dW (W, O, I), written into ``out`` (float32 or
    bfloat16, e.g. a view of the gradient rows) or a new tensor of ``dtype``.
    float32 dy is rounded to bfloat16, the type of the product's operands; the
    sums are float32."""
    if dy.dim() == 2:
        return weight_gradient(dy[None], saved, out=None if out is None else out[None], dtype=dtype, stream=stream)[0]
    _no_autograd(dy=dy, out=out)
    W, M, D = _saved(saved)
    device = saved.codes.device
    if _elsewhere(device, stream):
        with _there(device, stream):
            return weight_gradient(dy, saved, out=out, dtype=dtype)
    code = _dtype(dy, "dy")
    O = _three(dy, "dy")[2]
    gs = _input(dy, "dy", (W, M, O), dy.dtype, device)
    out = _gradient_out(out, "out", (W, O, D), dtype, device)
    dy_at = dy.data_ptr()
    needed = _entry("cpdp_weight_gradient_workspace")(dy_at, gs[0], gs[1], code, W, M, O, D)
    work = _workspace(needed, device)
    _check(_entry("cpdp_weight_gradient")(
        dy_at, gs[0], gs[1], code, saved.codes.data_ptr(), saved.exponents.data_ptr(), W, M, O, D, out.data_ptr(), out.stride(0),
        _CODES[out.dtype], _ptr(work), needed, _stream(device.index)))
    return out


def _sequences(gate) -> tuple:
    if gate.dim() != 3:
        raise ValueError(f"gate must be (B, T, D), got {tuple(gate.shape)}")
    _dtype(gate, "gate")
    return _sized(gate, "gate")


def gated_recurrence(gate, value, h0=None, lengths=None, *, carry: bool = True, stream=None):
    """h_t = a_t h_(t-1) + (1 - a_t) v_t with a = sigmoid(gate), for B sequences.

    gate, value (B, T, D) float32 or bfloat16 (two halves of one product's
    output, say); h0 float32 (B, D) or None for zeros; lengths int32 (B,) or
    None: beyond its length a sequence keeps its state and h is 0. Returns
    (h, h_last, carry): h (B, T, D) of gate's type, h_last float32 (B, D), and
    the states at every CARRY_STEPS steps, float32, which the backward pass
    starts from (carry=False: None)."""
    _no_autograd(gate=gate, value=value, h0=h0)
    device = _cuda(gate, "gate")
    if _elsewhere(device, stream):
        with _there(device, stream):
            return gated_recurrence(gate, value, h0, lengths, carry=carry)
    B, T, D = shape = _sequences(gate)
    dtype = gate.dtype
    gs, vs = _input(gate, "gate", shape, dtype, device), _input(value, "value", shape, dtype, device)
    h0_at, n_at = _whole(h0, "h0", (B, D), _F32, device), _whole(lengths, "lengths", (B,), torch.int32, device)
    h = torch.empty(shape, dtype=dtype, device=device)
    last = torch.empty((B, D), dtype=_F32, device=device)
    carries = torch.empty((B, -(-T // CARRY_STEPS), D), dtype=_F32, device=device) if carry else None
    needed = _entry("cpdp_gated_recurrence_workspace")(B, T, D)
    work = _workspace(needed, device)
    _check(_entry("cpdp_gated_recurrence")(
        gate.data_ptr(), gs[0], gs[1], value.data_ptr(), vs[0], vs[1], _CODES[dtype], B, T, D, h0_at, n_at, h.data_ptr(),
        last.data_ptr(), _ptr(carries), _ptr(work), needed, _stream(device.index)))
    return h, last, carries


def gated_recurrence_backward(dh, gate, value, carry, dh_last=None, lengths=None, *, out=None, stream=None):
    """Gradients of ``gated_recurrence``: (dgate, dvalue, dh0) from dh (B, T, D)
    and dh_last float32 (B, D) or None. dgate and dvalue are the halves of one
    (B, T, 2 D) tensor, ``out`` where given (contiguous along its last axis):
    the gradient of one product that made gate and value."""
    _no_autograd(dh=dh, gate=gate, value=value, carry=carry, dh_last=dh_last, out=out)
    device = _cuda(gate, "gate")
    if _elsewhere(device, stream):
        with _there(device, stream):
            return gated_recurrence_backward(dh, gate, value, carry, dh_last, lengths, out=out)
    B, T, D = shape = _sequences(gate)
    dtype = gate.dtype
    gs, vs = _input(gate, "gate", shape, dtype, device), _input(value, "value", shape, dtype, device)
    os = _input(dh, "dh", shape, dtype, device)
    carry_at = _whole(carry, "carry", (B, -(-T // CARRY_STEPS), D), _F32, device)
    last_at, n_at = _whole(dh_last, "dh_last", (B, D), _F32, device), _whole(lengths, "lengths", (B,), torch.int32, device)
    if out is None:
        out = torch.empty((B, T, 2 * D), dtype=dtype, device=device)
    ps = _input(out, "out", (B, T, 2 * D), dtype, device)
    _rows_apart(out, "out")
    dgate, dvalue = out.chunk(2, 2)
    dh0 = torch.empty((B, D), dtype=_F32, device=device)
    needed = _entry("cpdp_gated_recurrence_workspace")(B, T, D)
    work = _workspace(needed, device)
    _check(_entry("cpdp_gated_recurrence_backward")(
        dh.data_ptr(), os[0], os[1], gate.data_ptr(), gs[0], gs[1], value.data_ptr(), vs[0], vs[1], _CODES[dtype], B, T, D, carry_at,
        last_at, n_at, dgate.data_ptr(), dvalue.data_ptr(), ps[0], ps[1], dh0.data_ptr(), _ptr(work), needed, _stream(device.index)))
    return dgate, dvalue, dh0


def gated_recurrence_step(gate, value, state, *, stream=None):
    """One token for each of B sequences: ``state`` (float32, (B, D)) is replaced
    by the next state, which is returned rounded to gate's type. gate, value (B, D)."""
    shape, dtype, device, state_strides = gate.shape, gate.dtype, gate.device, state.stride()
    gs, vs, code = gate.stride(), value.stride(), _CODES.get(dtype)
    # one test where all is well: a decoding step costs what Python does around it
    if not (stream is None and code is not None and gate.is_cuda and device.index == _current_device() and len(shape) == 2
            and value.shape == shape == state.shape and max(shape) <= MAX_SIZE and value.dtype is dtype and state.dtype is _F32
            and value.device == device == state.device and gs[-1] == 1 == vs[-1] and state_strides == (shape[1], 1)
            and not (gate.requires_grad or value.requires_grad or state.requires_grad)):
        _no_autograd(gate=gate, value=value, state=state)
        if _elsewhere(_cuda(gate, "gate"), stream):
            with _there(device, stream):
                return gated_recurrence_step(gate, value, state)
        code = _dtype(gate, "gate")
        if len(shape) != 2:
            raise ValueError(f"gate must be (B, D), got {tuple(shape)}")
        _sized(gate, "gate")
        gs, vs = _input(gate, "gate", shape, dtype, device), _input(value, "value", shape, dtype, device)
        _whole(state, "state", shape, _F32, device)
    B, D = shape
    h = torch.empty(shape, dtype=dtype, device=device)
    _check(_entry("cpdp_gated_recurrence_step")(gate.data_ptr(), gs[0], value.data_ptr(), vs[0], code, B, D,
                                                state.data_ptr(), h.data_ptr(), _stream(device.index)))
    return h


def _head(x, weight, targets) -> tuple:
    """What the calls of the loss share: W, M, V, D and the arguments of x and weight."""
    shape, dtype, device, ws, xs = x.shape, x.dtype, x.device, weight.shape, x.stride()
    at, code = weight.stride(), _CODES.get(dtype)
    # one test where all is well: few tokens cost what Python does around them
    if not (code is not None and len(shape) == 3 and len(ws) == 3 and max(shape) <= MAX_SIZE and max(ws) <= MAX_SIZE
            and ws[0] == shape[0] and ws[2] == shape[2] and weight.dtype is dtype and weight.device == device and xs[2] == 1 == at[2]
            and targets.shape == shape[:2] and targets.dtype is torch.int64 and targets.device == device and targets.is_contiguous()):
        W, M, D = _three(x, "x")
        code = _dtype(x, "x")
        xs = _input(x, "x", shape, dtype, device)
        if weight.dim() != 3:
            raise ValueError(f"weight must be (W, V, D), or (V, D) of one model; got {tuple(ws)}")
        _sized(weight, "weight")
        at = _input(weight, "weight", (W, ws[1], D), dtype, device)
        _whole(targets, "targets", (W, M), torch.int64, device)
    W, M, D = shape
    return (W, M, ws[1], D), (x.data_ptr(), xs[0], xs[1], weight.data_ptr(), at[0], at[1]), targets.data_ptr(), code


def linear_cross_entropy(x, weight, targets, *, stream=None):
    """Cross entropy of each token's target under softmax(weight x): (loss, lse).

    x (W, M, D) and weight (W, V, D) of one type, float32 or bfloat16; targets
    int64 (W, M), negative where a token is ignored: its loss is 0. loss and
    lse = log(sum(exp(logits))), which the backward pass takes, are float32
    (W, M). A target of V or more has the loss NaN. The logits are not kept."""
    if x.dim() == 2 and weight.dim() == 2:
        loss, lse = linear_cross_entropy(x[None], weight[None], targets[None], stream=stream)
        return loss[0], lse[0]
    if x.requires_grad or weight.requires_grad:
        _no_autograd(x=x, weight=weight)
    device = _cuda(x, "x")
    if _elsewhere(device, stream):
        with _there(device, stream):
            return linear_cross_entropy(x, weight, targets)
    (W, M, V, D), operands, targets_at, code = _head(x, weight, targets)
    loss, lse = torch.empty((W, M), dtype=_F32, device=device), torch.empty((W, M), dtype=_F32, device=device)
    needed = _entry("cpdp_linear_cross_entropy_workspace")(*operands, code, W, M, V, D)
    work = _workspace(needed, device)
    _check(_entry("cpdp_linear_cross_entropy")(*operands, targets_at, code, W, M, V, D, loss.data_ptr(), lse.data_ptr(), _ptr(work), needed,
                                               _stream(device.index)))
    return loss, lse


def linear_cross_entropy_backward(dloss, x, weight, targets, lse, *, dweight=None, dtype=torch.float32, stream=None):
    """Gradients of ``linear_cross_entropy``: (dx, dweight) from dloss float32
    (W, M), the gradient of each token's loss (1 / M each for a mean). dx has x's
    type and is 0 in ignored tokens' rows. dweight (W, V, D) is written into the
    tensor given, float32 or bfloat16 (a view of the gradient rows, say), or into
    a new one of ``dtype``."""
    if x.dim() == 2 and weight.dim() == 2:
        dx, dw = linear_cross_entropy_backward(dloss[None], x[None], weight[None], targets[None], lse[None],
                                               dweight=None if dweight is None else dweight[None], dtype=dtype, stream=stream)
        return dx[0], dw[0]
    _no_autograd(dloss=dloss, x=x, weight=weight, lse=lse, dweight=dweight)
    device = _cuda(x, "x")
    if _elsewhere(device, stream):
        with _there(device, stream):
            return linear_cross_entropy_backward(dloss, x, weight, targets, lse, dweight=dweight, dtype=dtype)
    (W, M, V, D), operands, targets_at, code = _head(x, weight, targets)
    dloss_at, lse_at = _whole(dloss, "dloss", (W, M), _F32, device), _whole(lse, "lse", (W, M), _F32, device)
    dweight = _gradient_out(dweight, "dweight", (W, V, D), dtype, device)
    dx = torch.empty((W, M, D), dtype=x.dtype, device=device)
    needed = _entry("cpdp_linear_cross_entropy_backward_workspace")(*operands, code, W, M, V, D)
    work = _workspace(needed, device)
    _check(_entry("cpdp_linear_cross_entropy_backward")(
        dloss_at, *operands, targets_at, lse_at, code, W, M, V, D, dx.data_ptr(), dweight.data_ptr(), dweight.stride(0),
        _CODES[dweight.dtype], _ptr(work), needed, _stream(device.index)))
    return dx, dweight


def _workers_part(t, name: str, tail: tuple, W: int, device) -> int:
    """The worker stride of float32 weights (W, *tail) whose parts are contiguous each."""
    shape = (W, *tail)
    if t.shape != shape or t.dtype is not _F32 or t.device != device:
        if tuple(t.shape) != shape:
            raise ValueError(f"{name} must have shape {shape}, got {tuple(t.shape)}")
        if t.dtype != _F32:
            raise TypeError(f"{name} must be float32, got {t.dtype}")
        raise ValueError(f"{name} is on {t.device}, not on {device}")
    if not t.is_contiguous() and not t[0].is_contiguous():
        raise ValueError(f"each worker's part of {name} must be contiguous")
    return t.stride(0)


def _per_worker(B: int, weight, name: str, dims: int) -> int:
    """The number of workers whose weights these are; their sequences are neighbours."""
    if weight.dim() != dims:
        raise ValueError(f"{name} must have {dims} axes, the workers' first; got {tuple(weight.shape)}")
    W = _sized(weight, name)[0]
    if W < 1 or B % W:
        raise ValueError(f"{B} sequences are not as many for each of {W} workers")
    return W


def _sequence_shape(t, name: str) -> tuple:
    if t.dim() != 3:
        raise ValueError(f"{name} must be (B, T, D), got {tuple(t.shape)}")
    _dtype(t, name)
    return _sized(t, name)


def causal_conv(x, weight, bias, state=None, lengths=None, *, stream=None):
    """y_t = silu(bias + sum_k weight[k] x_(t-K+1+k)), for B sequences: (y, last).

    x (B, T, D) float32 or bfloat16; weight float32 (W, D, K) with K from 2 to
    CONV_MAX_TAPS and bias (W, D): those of worker w are for the w-th of W equal
    groups of sequences (one model's (D, K) and (D,) are taken too). state
    (B, K - 1, D) of x's type holds the inputs before the first step (None:
    zeros), last the ones before the next. lengths int32 (B,) or None: beyond its
    length a sequence is not read and y is 0."""
    if weight.dim() == 2 and bias.dim() == 1:
        weight, bias = weight[None], bias[None]
    _no_autograd(x=x, weight=weight, bias=bias, state=state)
    device = _cuda(x, "x")
    if _elsewhere(device, stream):
        with _there(device, stream):
            return causal_conv(x, weight, bias, state, lengths)
    B, T, D = shape = _sequence_shape(x, "x")
    dtype = x.dtype
    W, K = _per_worker(B, weight, "weight", 3), weight.shape[2]
    xs = _input(x, "x", shape, dtype, device)
    ws, bs = _workers_part(weight, "weight", (D, K), W, device), _workers_part(bias, "bias", (D,), W, device)
    state_at, n_at = _whole(state, "state", (B, K - 1, D), dtype, device), _whole(lengths, "lengths", (B,), torch.int32, device)
    y = torch.empty(shape, dtype=dtype, device=device)
    last = torch.empty((B, max(K - 1, 0), D), dtype=dtype, device=device)
    _check(_entry("cpdp_causal_conv")(x.data_ptr(), xs[0], xs[1], weight.data_ptr(), ws, bias.data_ptr(), bs, state_at, n_at, _CODES[dtype],
                                      W, B, T, D, K, y.data_ptr(), last.data_ptr(), _stream(device.index)))
    return y, last


def causal_conv_backward(dy, x, weight, bias, state=None, lengths=None, dlast=None, *, dweight=None, dbias=None, dstate=None,
                         dtype=torch.float32, stream=None):
    """Gradients of ``causal_conv``: (dx, dweight, dbias) from dy (B, T, D) and
    dlast (B, K - 1, D) or None. dweight (W, D, K) and dbias (W, D) are written
    into the tensors given, float32 or bfloat16 both (views of the gradient rows,
    say), or into new ones of ``dtype``. Where dstate, (B, K - 1, D) of x's type,
    is given, the gradient of state is written there."""
    if weight.dim() == 2 and bias.dim() == 1:
        dx, dw, db = causal_conv_backward(dy, x, weight[None], bias[None], state, lengths, dlast, dweight=None if dweight is None else dweight[None],
                                          dbias=None if dbias is None else dbias[None], dstate=dstate, dtype=dtype, stream=stream)
        return dx, dw[0], db[0]
    _no_autograd(dy=dy, x=x, weight=weight, bias=bias, state=state, dlast=dlast, dweight=dweight, dbias=dbias, dstate=dstate)
    device = _cuda(x, "x")
    if _elsewhere(device, stream):
        with _there(device, stream):
            return causal_conv_backward(dy, x, weight, bias, state, lengths, dlast, dweight=dweight, dbias=dbias, dstate=dstate, dtype=dtype)
    B, T, D = shape = _sequence_shape(x, "x")
    kind = x.dtype
    W, K = _per_worker(B, weight, "weight", 3), weight.shape[2]
    xs, gs = _input(x, "x", shape, kind, device), _input(dy, "dy", shape, kind, device)
    ws, bs = _workers_part(weight, "weight", (D, K), W, device), _workers_part(bias, "bias", (D,), W, device)
    few = (B, K - 1, D)
    state_at, n_at = _whole(state, "state", few, kind, device), _whole(lengths, "lengths", (B,), torch.int32, device)
    dlast_at, dstate_at = _whole(dlast, "dlast", few, kind, device), _whole(dstate, "dstate", few, kind, device)
    if dweight is not None:
        dtype = dweight.dtype
    elif dbias is not None:
        dtype = dbias.dtype
    dweight, dbias = _gradient_out(dweight, "dweight", (W, D, K), dtype, device), _gradient_out(dbias, "dbias", (W, D), dtype, device)
    if dbias.dtype != dtype:
        raise TypeError(f"dweight and dbias must have one type, got {dtype} and {dbias.dtype}")
    dx = torch.empty(shape, dtype=kind, device=device)
    needed = _entry("cpdp_causal_conv_backward_workspace")(W, B, T, D, K)
    work = _workspace(needed, device)
    _check(_entry("cpdp_causal_conv_backward")(
        dy.data_ptr(), gs[0], gs[1], x.data_ptr(), xs[0], xs[1], weight.data_ptr(), ws, bias.data_ptr(), bs, state_at, dlast_at, n_at,
        _CODES[kind], W, B, T, D, K, dx.data_ptr(), dstate_at, dweight.data_ptr(), dweight.stride(0), dbias.data_ptr(), dbias.stride(0),
        _CODES[dtype], _ptr(work), needed, _stream(device.index)))
    return dx, dweight, dbias


def causal_conv_step(x, weight, bias, state, *, stream=None):
    """One token for each of B sequences: x (B, D) gives y (B, D), and ``state``
    (B, K - 1, D), the inputs before it, is moved on by x."""
    if weight.dim() == 2 and bias.dim() == 1:
        weight, bias = weight[None], bias[None]
    shape, dtype, device, wshape = x.shape, x.dtype, x.device, weight.shape
    xs, ws, bs, code = x.stride(), weight.stride(), bias.stride(), _CODES.get(dtype)
    # one test where all is well: a decoding step costs what Python does around it
    if not (stream is None and code is not None and x.is_cuda and device.index == _current_device() and len(shape) == 2 and len(wshape) == 3
            and wshape[0] > 0 and shape[0] % wshape[0] == 0 and max(shape) <= MAX_SIZE >= wshape[2] and shape[1] == wshape[1] and xs[-1] == 1
            and weight.dtype is _F32 is bias.dtype and ws[1:] == (wshape[2], 1) and bias.shape == wshape[:2] and bs[1] == 1
            and state.dtype is dtype and state.shape == (shape[0], wshape[2] - 1, shape[1]) and state.is_contiguous()
            and weight.device == device == bias.device == state.device
            and not (x.requires_grad or weight.requires_grad or bias.requires_grad or state.requires_grad)):
        _no_autograd(x=x, weight=weight, bias=bias, state=state)
        if _elsewhere(_cuda(x, "x"), stream):
            with _there(device, stream):
                return causal_conv_step(x, weight, bias, state)
        code = _dtype(x, "x")
        if len(shape) != 2:
            raise ValueError(f"x must be (B, D), got {tuple(shape)}")
        B, D = _sized(x, "x")
        W = _per_worker(B, weight, "weight", 3)
        _input(x, "x", shape, dtype, device)
        _workers_part(weight, "weight", (D, wshape[2]), W, device)
        _workers_part(bias, "bias", (D,), W, device)
        _whole(state, "state", (B, wshape[2] - 1, D), dtype, device)
    B, D = shape
    y = torch.empty(shape, dtype=dtype, device=device)
    _check(_entry("cpdp_causal_conv_step")(x.data_ptr(), xs[0], weight.data_ptr(), ws[0], bias.data_ptr(), bs[0], code, wshape[0], B, D, wshape[2],
                                           state.data_ptr(), y.data_ptr(), _stream(device.index)))
    return y


# cpdp_scan_inputs: a pointer and two strides each of u, delta, z, b and c; a pointer and a stride each of a_log, skip and
# bias; lengths. All fields are of 8 bytes.
_pack_scan = struct.Struct("=22q").pack


def _scan_inputs(u, delta, a_log, b, c, skip, bias, z, lengths, device) -> tuple:
    """(W, the sizes, the inputs) of a scan; u is (B, T, D), or (B, D) of a single step."""
    shape, dtype = u.shape, u.dtype
    _dtype(u, "u")
    _sized(u, "u")
    B, D = shape[0], shape[-1]
    W, N = _per_worker(B, a_log, "a_log", 3), a_log.shape[2]
    few = (*shape[:-1], N)
    step = len(shape) == 2

    def at(t, name, shape):
        s = _input(t, name, shape, dtype, device)
        return t.data_ptr(), s[0], 0 if step else s[1]

    inputs = _pack_scan(*at(u, "u", shape), *at(delta, "delta", shape), *((0, 0, 0) if z is None else at(z, "z", shape)),
                        *at(b, "b", few), *at(c, "c", few), a_log.data_ptr(), _workers_part(a_log, "a_log", (D, N), W, device),
                        skip.data_ptr(), _workers_part(skip, "skip", (D,), W, device), bias.data_ptr(),
                        _workers_part(bias, "bias", (D,), W, device), _whole(lengths, "lengths", (B,), torch.int32, device) or 0)
    return W, N, inputs


def _of_one_model(a_log, skip, bias) -> tuple:
    """The weights with an axis of workers."""
    return (a_log[None], skip[None], bias[None]) if a_log.dim() == 2 and skip.dim() == bias.dim() == 1 else (a_log, skip, bias)


def selective_scan(u, delta, a_log, b, c, skip, bias, z=None, h0=None, lengths=None, *, carry: bool = True, stream=None):
    """With dt = softplus(delta + bias), h_t = exp(-dt exp(a_log)) h_(t-1) + dt u_t b_t
    for N states per channel and y_t = (sum_n c_t h_t + skip u_t) silu(z_t), for B
    sequences: (y, last, carry).

    u, delta, z (B, T, D) float32 or bfloat16 (z None: no gate); b, c (B, T, N) of
    the same type; a_log float32 (W, D, N) with N up to SCAN_MAX_STATES, skip and
    bias (W, D): those of worker w are for the w-th of W equal groups of
    sequences (one model's, without the axis W, are taken too); h0 float32
    (B, D, N) or None for zeros; lengths int32 (B,) or None: beyond its length a
    sequence keeps its state and y is 0. last float32 (B, D, N); carry, the states
    at every CARRY_STEPS steps, is what the backward pass starts from
    (carry=False: None)."""
    a_log, skip, bias = _of_one_model(a_log, skip, bias)
    _no_autograd(u=u, delta=delta, a_log=a_log, b=b, c=c, skip=skip, bias=bias, z=z, h0=h0)
    device = _cuda(u, "u")
    if _elsewhere(device, stream):
        with _there(device, stream):
            return selective_scan(u, delta, a_log, b, c, skip, bias, z, h0, lengths, carry=carry)
    B, T, D = shape = _sequence_shape(u, "u")
    W, N, inputs = _scan_inputs(u, delta, a_log, b, c, skip, bias, z, lengths, device)
    h0_at = _whole(h0, "h0", (B, D, N), _F32, device)
    y, last = torch.empty(shape, dtype=u.dtype, device=device), torch.empty((B, D, N), dtype=_F32, device=device)
    carries = torch.empty((B, -(-T // CARRY_STEPS), D, N), dtype=_F32, device=device) if carry else None
    needed = _entry("cpdp_selective_scan_workspace")(B, T, D, N)
    work = _workspace(needed, device)
    _check(_entry("cpdp_selective_scan")(inputs, _CODES[u.dtype], W, B, T, D, N, h0_at, y.data_ptr(), last.data_ptr(), _ptr(carries),
                                         _ptr(work), needed, _stream(device.index)))
    return y, last, carries


def selective_scan_backward(dy, u, delta, a_log, b, c, skip, bias, carry, z=None, dlast=None, lengths=None, *, da_log=None, dskip=None,
                            dbias=None, dtype=torch.float32, stream=None):
    """Gradients of ``selective_scan`` from dy (B, T, D) and dlast float32
    (B, D, N) or None: (du, ddelta, da_log, db, dc, dskip, dbias, dz, dh0), dz None
    where there is no z. The weights' are written into the tensors given, float32
    or bfloat16 all (views of the gradient rows, say), or into new ones of
    ``dtype``."""
    if a_log.dim() == 2 and skip.dim() == bias.dim() == 1:
        da_log, dskip, dbias = (None if t is None else t[None] for t in (da_log, dskip, dbias))
        out = selective_scan_backward(dy, u, delta, a_log[None], b, c, skip[None], bias[None], carry, z, dlast, lengths, da_log=da_log,
                                      dskip=dskip, dbias=dbias, dtype=dtype, stream=stream)
        return tuple(t[0] if i in (2, 5, 6) else t for i, t in enumerate(out))
    _no_autograd(dy=dy, u=u, delta=delta, a_log=a_log, b=b, c=c, skip=skip, bias=bias, carry=carry, z=z, dlast=dlast, da_log=da_log,
                 dskip=dskip, dbias=dbias)
    device = _cuda(u, "u")
    if _elsewhere(device, stream):
        with _there(device, stream):
            return selective_scan_backward(dy, u, delta, a_log, b, c, skip, bias, carry, z, dlast, lengths, da_log=da_log, dskip=dskip,
                                           dbias=dbias, dtype=dtype)
    B, T, D = shape = _sequence_shape(u, "u")
    kind = u.dtype
    W, N, inputs = _scan_inputs(u, delta, a_log, b, c, skip, bias, z, lengths, device)
    gs = _input(dy, "dy", shape, kind, device)
    carry_at = _whole(carry, "carry", (B, -(-T // CARRY_STEPS), D, N), _F32, device)
    dlast_at = _whole(dlast, "dlast", (B, D, N), _F32, device)
    given = [t for t in (da_log, dskip, dbias) if t is not None]
    dtype = given[0].dtype if given else dtype
    da_log = _gradient_out(da_log, "da_log", (W, D, N), dtype, device)
    dskip, dbias = _gradient_out(dskip, "dskip", (W, D), dtype, device), _gradient_out(dbias, "dbias", (W, D), dtype, device)
    if not da_log.dtype == dskip.dtype == dbias.dtype:
        raise TypeError(f"da_log, dskip and dbias must have one type, got {da_log.dtype}, {dskip.dtype} and {dbias.dtype}")
    du, ddelta = torch.empty(shape, dtype=kind, device=device), torch.empty(shape, dtype=kind, device=device)
    dz = None if z is None else torch.empty(shape, dtype=kind, device=device)
    db, dc = (torch.empty((B, T, N), dtype=kind, device=device) for _ in range(2))
    dh0 = torch.empty((B, D, N), dtype=_F32, device=device)
    needed = _entry("cpdp_selective_scan_backward_workspace")(B, T, D, N)
    work = _workspace(needed, device)
    _check(_entry("cpdp_selective_scan_backward")(
        dy.data_ptr(), gs[0], gs[1], inputs, _CODES[kind], W, B, T, D, N, carry_at, dlast_at, du.data_ptr(), ddelta.data_ptr(),
        _ptr(dz), db.data_ptr(), dc.data_ptr(), dh0.data_ptr(), da_log.data_ptr(), da_log.stride(0), dskip.data_ptr(), dskip.stride(0),
        dbias.data_ptr(), dbias.stride(0), _CODES[dtype], _ptr(work), needed, _stream(device.index)))
    return du, ddelta, da_log, db, dc, dskip, dbias, dz, dh0


def selective_scan_step(u, delta, a_log, b, c, skip, bias, state, z=None, *, stream=None):
    """One token for each of B sequences: ``state`` (float32, (B, D, N)) is
    replaced by the next state, and y (B, D) is returned. u, delta, z (B, D); b, c
    (B, N); the weights as those of ``selective_scan``."""
    if a_log.dim() == 2:
        a_log, skip, bias = _of_one_model(a_log, skip, bias)
    shape, dtype, device, few, weights = u.shape, u.dtype, u.device, b.shape, a_log.shape
    us, ds, bs, cs, ws, ks, os = u.stride(), delta.stride(), b.stride(), c.stride(), a_log.stride(), skip.stride(), bias.stride()
    zs, z_at = ((0, 1), 0) if z is None else (z.stride(), z.data_ptr())
    # one test where all is well: a decoding step costs what Python does around it
    if not (stream is None and dtype in _CODES and u.is_cuda and device.index == _current_device() and len(shape) == 2 and len(weights) == 3
            and delta.shape == shape and (z is None or z.shape == shape and z.dtype is dtype and z.device == device and not z.requires_grad)
            and weights[0] > 0 and shape[0] % weights[0] == 0 and max(shape) <= MAX_SIZE >= weights[2] and shape[1] == weights[1]
            and skip.shape == weights[:2] == bias.shape and few == (shape[0], weights[2]) == c.shape and state.shape == (*shape, weights[2])
            and delta.dtype is dtype and b.dtype is dtype and c.dtype is dtype and state.dtype is _F32 and a_log.dtype is _F32
            and skip.dtype is _F32 and bias.dtype is _F32 and ws[1:] == (weights[2], 1) and us[1] == ds[1] == zs[1] == bs[1] == cs[1] == ks[1] == os[1] == 1
            and state.is_contiguous() and delta.device == device == b.device == c.device == state.device
            and a_log.device == device == skip.device == bias.device
            and not (u.requires_grad or delta.requires_grad or b.requires_grad or c.requires_grad or state.requires_grad
                     or a_log.requires_grad or skip.requires_grad or bias.requires_grad)):
        _no_autograd(u=u, delta=delta, a_log=a_log, b=b, c=c, skip=skip, bias=bias, state=state, z=z)
        if _elsewhere(_cuda(u, "u"), stream):
            with _there(device, stream):
                return selective_scan_step(u, delta, a_log, b, c, skip, bias, state, z)
        if len(shape) != 2:
            raise ValueError(f"u must be (B, D), got {tuple(shape)}")
        N = _scan_inputs(u, delta, a_log, b, c, skip, bias, z, None, device)[1]
        _whole(state, "state", (*shape, N), _F32, device)
    B, D = shape
    inputs = _pack_scan(u.data_ptr(), us[0], 0, delta.data_ptr(), ds[0], 0, z_at, zs[0], 0, b.data_ptr(), bs[0], 0, c.data_ptr(), cs[0], 0,
                        a_log.data_ptr(), ws[0], skip.data_ptr(), ks[0], bias.data_ptr(), os[0], 0)
    y = torch.empty(shape, dtype=dtype, device=device)
    _check(_entry("cpdp_selective_scan_step")(inputs, _CODES[dtype], weights[0], B, D, weights[2], state.data_ptr(), y.data_ptr(),
                                              _stream(device.index)))
    return y


def clip_gradients(grads, max_norm: float, *, out=None, stream=None):
    """The norm of each worker's row of grads (W, N), float32 (W,), and the rows
    times min(1, max_norm / norm): written into ``out``, of grads' shape and type,
    or over grads where none is given (rows that are within max_norm are left as
    they are then). An infinite max_norm leaves every row as it is. grads float32 or bfloat16; its rows may be slices of longer
    ones. One model's (N,) is taken too."""
    if grads.dim() == 1:
        return clip_gradients(grads[None], max_norm, out=None if out is None else out[None], stream=stream)[0]
    if out is None:
        out = grads
    shape, dtype, device, gs, os = grads.shape, grads.dtype, grads.device, grads.stride(), out.stride()
    code = _CODES.get(dtype)
    # one test where all is well: a small model's rows cost what Python does around them
    if not (stream is None and code is not None and grads.is_cuda and device.index == _current_device() and len(shape) == 2 and shape[0] <= MAX_SIZE
            and out.shape == shape and out.dtype is dtype and out.device == device and gs[1] == 1 == os[1]
            and not (grads.requires_grad or out.requires_grad)):
        _no_autograd(grads=grads, out=out)
        if _elsewhere(_cuda(grads, "grads"), stream):
            with _there(device, stream):
                return clip_gradients(grads, max_norm, out=out)
        if grads.dim() != 2:
            raise ValueError(f"grads must be (W, N), or (N,) of one model; got {tuple(shape)}")
        if shape[0] > MAX_SIZE:
            raise ValueError(f"grads has an axis of more than {MAX_SIZE} workers: {tuple(shape)}")
        code = _dtype(grads, "grads")
        gs, os = _input(grads, "grads", shape, dtype, device), _input(out, "out", shape, dtype, device)
    W, N = shape
    norms = torch.empty((W,), dtype=_F32, device=device)
    if W == 0:
        return norms
    needed = _entry("cpdp_clip_gradients_workspace")(W, N)
    work = _workspace(needed, device)
    _check(_entry("cpdp_clip_gradients")(grads.data_ptr(), gs[0], code, W, N, max_norm, norms.data_ptr(), out.data_ptr(), os[0], _ptr(work),
                                         needed, _stream(device.index)))
    return norms


def wait_timeouts() -> int:
    """Bounded waits of the kernels of ``weight_gradient`` and of the loss that
    ran out since the last call (0 expected; the tiles concerned are NaN). Waits
    for the current device."""
    count = _L()
    _check(_entry("cpdp_layer_timeouts")(ctypes.byref(count)))
    return count.value
