"""Python names for include/ginex_train.h, the operators of the training step on gathered rows: rows
sorted by expert and back, activations kept in 8 bits, and their use in the backward pass.

Tensors in, tensors out, nothing computed here.  Rows are f32, bf16 or f16 tensors of two dimensions whose
last one is dense; any stride from row to row will do.  Every call enqueues on the current stream and
returns at once.

dispatch, combine and activate keep autograd's graph where it is recorded; their gradients are the calls that are made for
them.  Results of those, and codes, are constants to autograd.  Tensors that carry a tangent of forward mode are refused
everywhere, and so are such gradients in a backward pass.
"""
from __future__ import annotations

import ctypes as C
import functools
from dataclasses import dataclass, field

import torch
from torch.autograd import forward_ad

from . import _lib
from ._lib import CodesDesc, RoutingDesc, RowsDesc
from .api import GinexError, _check, _workspace

CODE_BLOCK = 32                 # channels that share a scale
ACTIVATIONS = {"relu": 1, "silu": 2, "gelu": 3}
_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


# The current stream's handle without a stream object around it (2.6 us of a call's 11).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(device=None):
    """Of the current GPU, whose number a caller may have already."""
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device() if device is None else device)


def _no_tangent(t, what):
    """The kernels read a tensor's values, and what they give would count as a constant to forward mode (which no_grad leaves
    on, and which is off inside of an autograd function)."""
    if forward_ad._current_level >= 0 and torch._C._is_fwd_grad_enabled() and isinstance(t, torch.Tensor) \
            and forward_ad.unpack_dual(t).tangent is not None:
        raise RuntimeError(f"{what}: no tangent of forward mode goes through this call")


def _here(t, what, dtype=None):
    """A tensor in the memory of the current GPU."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{what}: expected a tensor in GPU memory")
    if t.get_device() != torch.cuda.current_device():
        raise ValueError(f"{what}: on {t.device}, which is not the current GPU")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{what}: expected dtype {dtype}, got {t.dtype}")
    if t.is_neg():
        raise ValueError(f"{what}: in memory with the other sign (see Tensor.resolve_neg)")
    _no_tangent(t, what)
    return t


def _dense(t, what, shape, dtype):
    _here(t, what, dtype)
    if t.shape != shape:
        raise ValueError(f"{what}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{what}: expected a contiguous tensor")
    return t


def _space(workspace, need, like):
    """The caller's workspace, or one for this call where there is none or it is too small."""
    if workspace is None or workspace.numel() < need:
        return _workspace(need, like.device)
    _here(workspace, "workspace", torch.uint8)
    if not workspace.is_contiguous():
        raise ValueError("workspace: expected a contiguous tensor")
    return workspace


def _with(made, what, t):
    """A route or compressed rows in the memory that ``t`` is in, too."""
    if made._device != t.get_device():
        raise ValueError(f"{what}: on GPU {made._device}, the rows on {t.device}")
    return made


def _rows(t, what):
    """The descriptor of a matrix of rows."""
    _here(t, what)
    kind = _TYPES.get(t.dtype)
    if kind is None:
        raise ValueError(f"{what}: expected float32, bfloat16 or float16, got {t.dtype}")
    if t.dim() != 2:
        raise ValueError(f"{what}: expected two dimensions, got {t.dim()}")
    n, width = t.shape
    stride, step = t.stride()
    if step != 1 and width > 1:
        raise ValueError(f"{what}: the elements of a row must be dense")
    if n <= 1:
        stride = width          # (a single row may have any)
    return RowsDesc(t.data_ptr(), n, width, stride, kind)


def _overwritten(t):
    """autograd hears of it, which may have kept the tensor."""
    if not t.is_inference():
        torch.autograd.graph.increment_version(t)


def _out(out, what, shape, dtype, like):
    """A tensor for the result and its descriptor."""
    if out is None:
        out = like.new_empty(shape, dtype=dtype)
        return out, RowsDesc(out.data_ptr(), shape[0], shape[1], shape[1], _TYPES[dtype])
    _here(out, what, dtype)
    if tuple(out.shape) != shape:
        raise ValueError(f"{what}: expected shape {shape}, got {tuple(out.shape)}")
    desc = _rows(out, what)
    _overwritten(out)
    return out, desc


def _first_derivative(backward):
    """For the backward of an autograd function: what the kernels give is no graph, and in a gradient that is to be
    differentiated it would count as a constant.  (autograd's own once_differentiable notices only where the incoming
    gradient requires one.)"""
    @functools.wraps(backward)
    def checked(ctx, *grads):
        if torch.is_grad_enabled():
            raise RuntimeError(f"{type(ctx).__name__}: there is no second derivative (create_graph=True asks for one)")
        for grad in grads:
            _no_tangent(grad, type(ctx).__name__)
        return backward(ctx, *grads)
    return checked


def _activation(name):
    if name not in ACTIVATIONS:
        raise ValueError(f"unknown activation {name!r}: one of {sorted(ACTIVATIONS)}")
    return ACTIVATIONS[name]


@dataclass(frozen=True)
class Route:
    """Where the rows go: pair (r, j) is in slot ``slot[r, j]`` or in none (-1), the slots of expert e are
    ``offsets[e]`` .. ``offsets[e + 1] - 1``, and slot s holds row ``source[s]`` (-1 behind the last one)."""
    offsets: torch.Tensor       # int64 [experts + 1]
    slot: torch.Tensor          # int32 [rows, top]
    source: torch.Tensor        # int32 [rows * top]
    _desc: RoutingDesc = field(init=False, repr=False, compare=False)
    _device: int = field(init=False, repr=False, compare=False)

    def __post_init__(self):
        _here(self.slot, "slot", torch.int32)
        if self.slot.dim() != 2 or self.offsets.dim() != 1 or self.offsets.numel() < 2:
            raise ValueError("expected offsets [experts + 1] and slot [rows, top]")
        rows, top = self.slot.shape
        _dense(self.offsets, "offsets", (self.offsets.numel(),), torch.int64)
        _dense(self.slot, "slot", (rows, top), torch.int32)
        _dense(self.source, "source", (rows * top,), torch.int32)
        self.__dict__["_desc"] = RoutingDesc(rows, top, self.experts, self.offsets.data_ptr(),
                                             self.slot.data_ptr(), self.source.data_ptr())
        self.__dict__["_device"] = self.slot.get_device()

    @classmethod
    def _made(cls, offsets, slot, source):
        """Of tensors that are known to be right."""
        made = object.__new__(cls)
        rows, top = slot.shape
        made.__dict__.update(offsets=offsets, slot=slot, source=source, _device=slot.get_device(), _desc=RoutingDesc(
            rows, top, offsets.numel() - 1, offsets.data_ptr(), slot.data_ptr(), source.data_ptr()))
        return made

    def _tensors(self):
        return self.offsets, self.slot, self.source

    @property
    def rows(self) -> int:
        return self.slot.shape[0]

    @property
    def top(self) -> int:
        return self.slot.shape[1]

    @property
    def experts(self) -> int:
        return self.offsets.numel() - 1


def route(chosen, experts, capacity=None, workspace=None) -> Route:
    """ginex_route: sorts the pairs (row, choice) of ``chosen`` [rows, top] (int32 or int64) by expert.  A
    value outside 0 .. experts - 1 means no expert; an expert gets ``capacity`` slots at most."""
    lib = _lib.load()
    _here(chosen, "chosen")
    if chosen.dtype not in (torch.int32, torch.int64):
        raise ValueError(f"chosen: expected int32 or int64, got {chosen.dtype}")
    if chosen.dim() != 2 or not chosen.is_contiguous():
        raise ValueError("chosen: expected a contiguous tensor [rows, top]")
    if capacity is not None and capacity < 0:
        raise ValueError(f"capacity={capacity}")
    rows, top = chosen.shape
    need = lib.ginex_route_workspace_bytes(rows, top, experts)
    if need == 0:
        raise GinexError(-1, lib.ginex_last_error().decode())
    ws = _space(workspace, need, chosen)
    made = Route._made(chosen.new_empty(experts + 1, dtype=torch.int64),
                       chosen.new_empty((rows, top), dtype=torch.int32),
                       chosen.new_empty(rows * top, dtype=torch.int32))
    _check(lib.ginex_route(chosen.data_ptr(), int(chosen.dtype == torch.int64),
                           -1 if capacity is None else min(capacity, (1 << 31) - 1), C.byref(made._desc),
                           ws.data_ptr(), ws.numel(), _stream()))
    return made


def _recorded(out):
    """A call that autograd records makes its result."""
    if out is not None:
        raise ValueError("out: autograd records this call, whose result has to be a new tensor")


class Dispatch(torch.autograd.Function):
    """Rows to their slots."""

    @staticmethod
    def forward(ctx, x, r):
        ctx.save_for_backward(*r._tensors())
        return dispatch(x, r)

    @staticmethod
    @_first_derivative
    def backward(ctx, grad):
        return dispatch_backward(grad.contiguous(), Route(*ctx.saved_tensors)), None


class Combine(torch.autograd.Function):
    """The slots' rows back to their rows, weighted."""

    @staticmethod
    def forward(ctx, z, weights, r):
        ctx.save_for_backward(z, weights, *r._tensors())
        return combine(z, r, weights)

    @staticmethod
    @_first_derivative
    def backward(ctx, grad):
        z, weights, *route = ctx.saved_tensors
        dz, dweights = combine_backward(grad.contiguous(), z, Route(*route), weights)
        return dz, dweights, None


class Activation(torch.autograd.Function):
    """An activation whose input is kept in 8 bits for its gradient; the codes are put into the list ``made``."""

    @staticmethod
    def forward(ctx, x, name, made=None):
        y, kept = activate(x, name)
        ctx.save_for_backward(kept.codes, kept.scales)
        ctx.width, ctx.name = kept.width, name
        if made is not None:
            made.append(kept)
        return y

    @staticmethod
    @_first_derivative
    def backward(ctx, grad):
        kept = Compressed(*ctx.saved_tensors, ctx.width)
        return activate_backward(kept, grad.contiguous(), ctx.name), None, None


def dispatch(x, route: Route, out=None):
    """ginex_dispatch: the rows of ``x`` in their slots, [rows * top, width]; slots without a row are 0."""
    desc = _rows(x, "x")
    if x.requires_grad and torch.is_grad_enabled():
        _recorded(out)
        return Dispatch.apply(x, route)
    out, to = _out(out, "out", (route.source.numel(), desc.width), x.dtype, x)
    _check(_lib.load().ginex_dispatch(C.byref(_with(route, "route", x)._desc), C.byref(desc), C.byref(to),
                                      _stream()))
    return out


def _combine(z, route, weights, out):
    desc = _rows(z, "z")
    out, to = _out(out, "out", (route.rows, desc.width), z.dtype, z)
    _check(_lib.load().ginex_combine(C.byref(_with(route, "route", z)._desc), C.byref(desc),
                                     None if weights is None else weights.data_ptr(), C.byref(to),
                                     _stream()))
    return out


def combine(z, route: Route, weights, out=None):
    """ginex_combine: y[r] = sum_j weights[r, j] z[slot[r, j]]; ``weights`` f32 [rows, top]."""
    _dense(weights, "weights", (route.rows, route.top), torch.float32)
    if (weights.requires_grad or getattr(z, "requires_grad", False)) and torch.is_grad_enabled():
        _recorded(out)
        return Combine.apply(z, weights, route)
    return _combine(z, route, weights, out)


def dispatch_backward(grad, route: Route, out=None):
    """The gradient of dispatch: the sum of a row's slots."""
    return _combine(grad, route, None, out)


def combine_backward(grad, z, route: Route, weights):
    """ginex_combine_backward: the gradients of ``z`` and of ``weights``."""
    _dense(weights, "weights", (route.rows, route.top), torch.float32)
    desc, zdesc = _rows(grad, "grad"), _rows(z, "z")
    dz, to = _out(None, "dz", (zdesc.rows, zdesc.width), z.dtype, z)
    dweights = torch.empty_like(weights)
    _check(_lib.load().ginex_combine_backward(C.byref(_with(route, "route", z)._desc), C.byref(desc),
                                              C.byref(zdesc),
                                              weights.data_ptr(), C.byref(to), dweights.data_ptr(),
                                              _stream()))
    return dz, dweights


@dataclass(frozen=True)
class Compressed:
    """Rows in 8 bits: blocks of 32 channels share a power of two, code q of a block with scale byte b
    stands for q * 2^(b - 133), b = 255 for NaN."""
    codes: torch.Tensor         # int8 [rows, 32 * blocks]
    scales: torch.Tensor        # uint8 [rows, blocks]
    width: int
    _desc: CodesDesc = field(init=False, repr=False, compare=False)
    _device: int = field(init=False, repr=False, compare=False)

    def __post_init__(self):
        _here(self.codes, "codes", torch.int8)
        if self.codes.dim() != 2:
            raise ValueError("codes: expected two dimensions")
        rows, blocks = self.codes.shape[0], -(-self.width // CODE_BLOCK)
        _dense(self.codes, "codes", (rows, blocks * CODE_BLOCK), torch.int8)
        _dense(self.scales, "scales", (rows, blocks), torch.uint8)
        self.__dict__["_desc"] = CodesDesc(rows, self.width, self.codes.data_ptr(), self.scales.data_ptr())
        self.__dict__["_device"] = self.codes.get_device()

    @classmethod
    def _made(cls, codes, scales, width):
        """Of tensors that are known to be right."""
        made = object.__new__(cls)
        made.__dict__.update(codes=codes, scales=scales, width=width, _device=codes.get_device(), _desc=CodesDesc(
            codes.shape[0], width, codes.data_ptr(), scales.data_ptr()))
        return made

    @property
    def rows(self) -> int:
        return self.codes.shape[0]


def _compress(x, desc, activation, to):
    n, width = desc.rows, desc.width
    blocks = -(-width // CODE_BLOCK)
    kept = Compressed._made(x.new_empty((n, blocks * CODE_BLOCK), dtype=torch.int8),
                            x.new_empty((n, blocks), dtype=torch.uint8), width)
    _check(_lib.load().ginex_compress(C.byref(desc), activation, None if to is None else C.byref(to),
                                      C.byref(kept._desc), _stream()))
    return kept


def compress(x) -> Compressed:
    """ginex_compress: ``x`` kept in 8.25 bits a value."""
    return _compress(x, _rows(x, "x"), 0, None)


def activate(x, activation, out=None):
    """ginex_compress with an activation ("relu", "silu", "gelu"): its values, and ``x`` compressed for the
    backward pass.  ``out`` may be ``x``."""
    kind = _activation(activation)
    desc = _rows(x, "x")
    if x.requires_grad and torch.is_grad_enabled():
        _recorded(out)
        made = []
        return Activation.apply(x, activation, made), made[0]
    out, to = _out(out, "out", (desc.rows, desc.width), x.dtype, x)
    return out, _compress(x, desc, kind, to)


def restore(kept: Compressed, dtype=torch.float32, out=None):
    """ginex_restore: the values that the codes stand for."""
    if dtype not in _TYPES:
        raise ValueError(f"expected float32, bfloat16 or float16, got {dtype}")
    current = torch.cuda.current_device() if kept._device >= 0 else None
    if kept._device != current:
        raise ValueError(f"kept: on {kept.codes.device}, which is not the current GPU")
    out, to = _out(out, "out", (kept.rows, kept.width), dtype, kept.codes)
    _check(_lib.load().ginex_restore(C.byref(kept._desc), C.byref(to), _stream(current)))
    return out


def activate_backward(kept: Compressed, grad, activation, out=None):
    """ginex_activate_backward: ``grad`` times the activation's derivative at the kept values.  ``out`` may
    be ``grad``."""
    kind = _activation(activation)
    desc = _rows(grad, "grad")
    out, to = _out(out, "out", (desc.rows, desc.width), grad.dtype, grad)
    _check(_lib.load().ginex_activate_backward(C.byref(_with(kept, "kept", grad)._desc), kind,
                                               C.byref(desc), C.byref(to), _stream()))
    return out


def weight_gradient(kept: Compressed, grad, route: Route = None, out=None, workspace=None):
    """ginex_weight_gradient: per expert the sum over its slots of (kept row)^T (row of ``grad``), f32
    [experts, width, grad width]; without a route one layer's, [width, grad width]."""
    lib = _lib.load()
    desc = _rows(grad, "grad")
    shape = (kept.width, grad.shape[1])
    if route is not None:
        shape = (route.experts, *shape)
    if out is not None:
        _overwritten(_dense(out, "out", shape, torch.float32))
    else:
        out = torch.empty(shape, dtype=torch.float32, device=grad.device)
    need = lib.ginex_weight_gradient_workspace_bytes(grad.shape[0], shape[0] if route is not None else 1,
                                                     kept.width, grad.shape[1])
    if need == 0:
        raise GinexError(-1, lib.ginex_last_error().decode())
    ws = _space(workspace, need, grad)
    _check(lib.ginex_weight_gradient(C.byref(_with(kept, "kept", grad)._desc),
                                     None if route is None else C.byref(_with(route, "route", grad)._desc),
                                     C.byref(desc), out.data_ptr(), ws.data_ptr(), ws.numel(), _stream()))
    return out
