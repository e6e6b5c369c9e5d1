"""Python names for include/ginex_layers.h, layers of a model on gathered rows: linear layers with bias, activation and
residual (one for all rows, or one per expert of a route) and the gradients of their rows and biases, a whole layer of experts
for a few rows, layer norm and the lookup of learned rows with their gradients.

Tensors in, tensors out, nothing computed here.  Rows are as in training.py; weights are [width, out] or [experts, width, out]
with either of the last two dimensions dense (``module.weight.t()`` as it is), biases and other vectors of the rows' type.
Every call enqueues on the current stream and returns at once.

linear, layer_norm and lookup keep autograd's graph where it is recorded.  linear keeps its rows and what its activation is
applied to in 8 bits; layer_norm keeps its rows as they are.  expert_layer has no gradient and refuses to be recorded.
What the calls for gradients give is a constant to autograd.  Tensors that carry a tangent of forward mode are refused everywhere.
A graph may capture a step with its backward pass: ask for the gradients by torch.autograd.grad, and let no graph of autograd that
was recorded outside of the capture hold the same leaves meanwhile (autograd would wait for the stream that it was recorded on).
"""
from __future__ import annotations

import contextlib
import ctypes as C

import torch

from . import _lib
from ._lib import WeightsDesc
from .api import GinexError, _check
from .training import (_TYPES, ACTIVATIONS, Compressed, Route, _activation, _dense, _first_derivative, _here, _out, _overwritten,
                       _raw_stream, _recorded, _rows, _space, _stream, _with, activate_backward, compress, dispatch_backward, weight_gradient)

FEW_ROWS, FEW_TOP = 64, 16      # of expert_layer

# The plain case of a call without the interpreter's part: False until it has been looked for, None where there is none.
_quick = False
_NO_ROUTE = (None, None, None)
_AS_IT_IS = contextlib.nullcontext()


def _quick_for(x):
    """(the compiled calls, current GPU, its stream) for a call on ``x``, or None."""
    global _quick
    if _quick is False:
        _lib.load()
        _quick = _lib.quick() if _raw_stream is not None else None
    if _quick is None or not getattr(x, "is_cuda", False):
        return None
    device = torch._C._cuda_getDevice()
    return _quick, device, _raw_stream(device)


def _layer_weights(weight, like, experts):
    """The descriptor of the weights of one layer, or of one per expert."""
    _here(weight, "weight", like.dtype)
    if weight.dim() != (2 if experts is None else 3):
        raise ValueError(f"weight: expected {'[width, out]' if experts is None else '[experts, width, out]'}, got "
                         f"{tuple(weight.shape)}")
    *count, width, out = weight.shape
    of, along, across = weight.stride() if count else (0, *weight.stride())
    if across == 1 or out == 1:
        turned, stride = 0, (out if width == 1 else along)
    elif along == 1 or width == 1:
        turned, stride = 1, across
    else:
        raise ValueError("weight: one of its last two dimensions must be dense")
    count = count[0] if count else 1
    return WeightsDesc(weight.data_ptr(), count, turned, width, out, stride, of if count > 1 else 0, _TYPES[like.dtype])


def _vector(t, what, shape, dtype):
    return None if t is None else _dense(t, what, shape, dtype).data_ptr()


def _any_grad(*tensors):
    return torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors)


def _codes_for(rows, width, like):
    blocks = -(-width // 32)
    return Compressed._made(like.new_empty((rows, blocks * 32), dtype=torch.int8),
                            like.new_empty((rows, blocks), dtype=torch.uint8), width)


class Linear(torch.autograd.Function):
    """A linear layer whose rows and pre-activations are kept in 8 bits; those are put into the list ``made``."""

    @staticmethod
    def forward(ctx, x, weight, bias, residual, activation, route, slots, made):
        kept = None
        if activation is not None or made is not None:
            y, kept = linear(x, weight, bias, activation, residual, route, slots, keep=True)
        else:
            y = linear(x, weight, bias, None, residual, route, slots)
        if made is not None:
            made.append(kept)
        rows = compress(x) if ctx.needs_input_grad[1] else None
        saved = [weight]
        for k in (rows, None if activation is None else kept):
            saved += [None, None] if k is None else [k.codes, k.scales]
        ctx.save_for_backward(*saved, *(() if route is None else route._tensors()))
        ctx.widths, ctx.activation, ctx.slots = (x.shape[1], y.shape[1]), activation, slots
        ctx.bias_type = None if bias is None else bias.dtype
        return y

    @staticmethod
    @_first_derivative
    def backward(ctx, grad):
        weight, rows, row_scales, kept, kept_scales, *route = ctx.saved_tensors
        r = Route(*route) if route else None
        grad = grad.contiguous()
        dz = grad
        if ctx.activation is not None:
            dz = activate_backward(Compressed(kept, kept_scales, ctx.widths[1]), grad, ctx.activation)
        dx = dw = db = dres = None
        if ctx.needs_input_grad[0]:
            dx = linear_backward(dz, weight, r)
            if r is not None and not ctx.slots:
                dx = dispatch_backward(dx, r)
        if ctx.needs_input_grad[1]:
            by = r
            if r is not None and ctx.slots:     # slot s has row s
                own = torch.arange(dz.shape[0], dtype=torch.int32, device=dz.device)
                by = Route(r.offsets, own[:, None], own)
            dw = weight_gradient(Compressed(rows, row_scales, ctx.widths[0]), dz, by).to(weight.dtype)
        if ctx.needs_input_grad[2]:
            db = bias_gradient(dz, r).to(ctx.bias_type)
        if ctx.needs_input_grad[3]:
            dres = grad
            if r is not None:                   # (slots without a row are cleared, whatever the residual)
                taken = torch.arange(grad.shape[0], device=grad.device) < r.offsets[-1]
                dres = torch.where(taken[:, None], grad, torch.zeros((), dtype=grad.dtype, device=grad.device))
        return dx, dw, db, dres, None, None, None, None


def linear(x, weight, bias=None, activation=None, residual=None, route: Route = None, slots=False, keep=False, out=None):
    """ginex_linear: activation(x weight + bias) + residual, the sums in f32, rounded once.  With a route the rows are the
    slots', [rows * top, out]: those of ``x`` [rows, width] by the route, or (``slots``) of ``x`` [rows * top, width] as they
    are; weights and biases are the experts', and slots without a row are 0.  ``keep``: (result, what the activation is applied
    to in 8 bits, for activate_backward).  ``out`` may be ``residual``."""
    if out is None and not keep and (activation is None or activation in ACTIVATIONS):
        at = _quick_for(x)
        got = at and at[0].linear(at[1], at[2], x, weight, bias, 0 if activation is None else ACTIVATIONS[activation], residual,
                                  *(_NO_ROUTE if route is None else route._tensors()), bool(slots))
        if got:
            _check(got[0])
            return got[1]
    desc = _rows(x, "x")
    experts = None if route is None else route.experts
    if _any_grad(x, weight, bias, residual):
        _recorded(out)
        made = [] if keep else None
        y = Linear.apply(x, weight, bias, residual, activation, route, slots, made)
        return (y, made[0]) if keep else y
    w = _layer_weights(weight, x, experts)
    if slots and route is None:
        raise ValueError("slots: there is no route")
    n = desc.rows if route is None else _with(route, "route", x).source.numel()
    kind = 0 if activation is None else _activation(activation)
    b = _vector(bias, "bias", (w.out,) if route is None else (w.experts, w.out), x.dtype)
    res = None
    if residual is not None:
        _here(residual, "residual", x.dtype)
        if tuple(residual.shape) != (n, w.out):
            raise ValueError(f"residual: expected shape {(n, w.out)}, got {tuple(residual.shape)}")
        res = C.byref(_rows(residual, "residual"))
    y, to = _out(out, "out", (n, w.out), x.dtype, x)
    kept = _codes_for(n, w.out, x) if keep else None
    _check(_lib.load().ginex_linear(C.byref(desc), C.byref(w), b, kind, res, None if route is None else C.byref(route._desc),
                                    int(slots), C.byref(to), None if kept is None else C.byref(kept._desc), _stream()))
    return (y, kept) if keep else y


def linear_backward(grad, weight, route: Route = None, out=None):
    """The gradient of linear's rows: ``grad`` times the weights turned over.  ``grad`` is that of activation's argument (see
    activate_backward); with a route it is the slots' and so is the result, which dispatch_backward adds up by rows."""
    if not isinstance(weight, torch.Tensor) or weight.dim() < 2:
        raise ValueError("weight: expected a tensor [width, out] or [experts, width, out]")
    recorded = torch.is_grad_enabled() and (weight.requires_grad or getattr(grad, "requires_grad", False))
    with torch.no_grad() if recorded else _AS_IT_IS:
        return linear(grad, weight.mT, route=route, slots=route is not None, out=out)


def bias_gradient(grad, route: Route = None, out=None, workspace=None):
    """ginex_bias_gradient: the sum of ``grad``'s rows, f32 [width]; with a route the sums of the experts' slots, [experts,
    width]."""
    if out is None and workspace is None:
        at = _quick_for(grad)
        got = at and at[0].bias_gradient(at[1], at[2], grad, *(_NO_ROUTE if route is None else route._tensors()))
        if got:
            _check(got[0])
            return got[1]
    lib = _lib.load()
    desc = _rows(grad, "grad")
    experts = 1 if route is None else route.experts
    shape = (desc.width,) if route is None else (experts, desc.width)
    if out is not None:
        _overwritten(_dense(out, "out", shape, torch.float32))
    else:
        out = grad.new_empty(shape, dtype=torch.float32)
    need = lib.ginex_bias_gradient_workspace_bytes(desc.rows, experts, desc.width)
    if need == 0:
        raise GinexError(-1, lib.ginex_last_error().decode())
    ws = _space(workspace, need, grad)
    _check(lib.ginex_bias_gradient(C.byref(desc), None if route is None else C.byref(_with(route, "route", grad)._desc),
                                   out.data_ptr(), ws.data_ptr(), ws.numel(), _stream()))
    return out


def expert_layer(x, router, weight, top, activation=None, bias=None, out=None, workspace=None):
    """ginex_expert_layer: a whole layer of experts for up to 64 rows: the ``top`` experts of the largest scores
    ``x router^T`` (``router`` [experts, width]), and the sum of their answers activation(x weight + bias) by the softmax of
    those scores.  It has no gradient."""
    if out is None and workspace is None and (activation is None or activation in ACTIVATIONS):
        at = _quick_for(x)
        got = at and at[0].expert_layer(at[1], at[2], x, router, weight, bias, top,
                                        0 if activation is None else ACTIVATIONS[activation])
        if got:
            _check(got[0])
            return got[1]
    lib = _lib.load()
    desc, rdesc = _rows(x, "x"), _rows(router, "router")
    if _any_grad(x, router, weight, bias):
        raise ValueError("expert_layer has no gradient: call it without autograd, or use route, linear and combine")
    if router.dtype != x.dtype:
        raise ValueError(f"router: expected dtype {x.dtype}, got {router.dtype}")
    w = _layer_weights(weight, x, rdesc.rows)
    kind = 0 if activation is None else _activation(activation)
    b = _vector(bias, "bias", (w.experts, w.out), x.dtype)
    y, to = _out(out, "out", (desc.rows, w.out), x.dtype, x)
    need = lib.ginex_expert_layer_workspace_bytes(desc.rows, top, w.experts, w.width, w.out)
    if need == 0:
        raise GinexError(-1, lib.ginex_last_error().decode())
    ws = _space(workspace, need, x)
    _check(lib.ginex_expert_layer(C.byref(desc), C.byref(rdesc), C.byref(w), b, top, kind, C.byref(to), ws.data_ptr(),
                                  ws.numel(), _stream()))
    return y


class LayerNorm(torch.autograd.Function):
    """Layer norm; its statistics are put into the list ``made``."""

    @staticmethod
    def forward(ctx, x, weight, bias, eps, made):
        y, stats = layer_norm(x, weight, bias, eps, stats=True)
        made.append(stats)
        ctx.save_for_backward(x, stats, weight)
        ctx.bias_type = None if bias is None else bias.dtype
        return y

    @staticmethod
    @_first_derivative
    def backward(ctx, grad):
        x, stats, weight = ctx.saved_tensors
        vectors = ctx.needs_input_grad[1] or ctx.needs_input_grad[2]
        dx, dw, db = layer_norm_backward(grad.contiguous(), x, stats, weight, vectors=vectors)
        return (dx, dw.to(weight.dtype) if ctx.needs_input_grad[1] else None,
                db.to(ctx.bias_type) if ctx.needs_input_grad[2] else None, None, None)


def layer_norm(x, weight=None, bias=None, eps=1e-5, stats=False, out=None):
    """ginex_layer_norm over the rows of ``x``; with ``stats`` also f32 [rows, 2], mean and 1 / sqrt(variance + eps) of every
    row, for layer_norm_backward.  ``out`` may be ``x``."""
    if out is None:
        at = _quick_for(x)
        got = at and at[0].layer_norm(at[1], at[2], x, weight, bias, eps, bool(stats))
        if got:
            _check(got[0])
            return got[1:] if stats else got[1]
    desc = _rows(x, "x")
    if _any_grad(x, weight, bias):
        _recorded(out)
        made = []
        y = LayerNorm.apply(x, weight, bias, eps, made)
        return (y, made[0]) if stats else y
    w, b = _vector(weight, "weight", (desc.width,), x.dtype), _vector(bias, "bias", (desc.width,), x.dtype)
    y, to = _out(out, "out", (desc.rows, desc.width), x.dtype, x)
    kept = x.new_empty((desc.rows, 2), dtype=torch.float32) if stats else None
    _check(_lib.load().ginex_layer_norm(C.byref(desc), w, b, eps, C.byref(to), None if kept is None else kept.data_ptr(),
                                        _stream()))
    return (y, kept) if stats else y


def layer_norm_backward(grad, x, stats, weight=None, vectors=True, out=None, workspace=None):
    """ginex_layer_norm_backward: the gradients of ``x``, of the weight and of the bias (f32 [width]; None with ``vectors``
    False).  ``out`` may be ``grad``."""
    if out is None and workspace is None and vectors:
        at = _quick_for(grad)
        got = at and at[0].layer_norm_backward(at[1], at[2], grad, x, stats, weight)
        if got:
            _check(got[0])
            return got[1:]
    lib = _lib.load()
    desc, xdesc = _rows(grad, "grad"), _rows(x, "x")
    _dense(stats, "stats", (xdesc.rows, 2), torch.float32)
    w = _vector(weight, "weight", (xdesc.width,), x.dtype)
    dx, to = _out(out, "out", (xdesc.rows, xdesc.width), x.dtype, x)
    dweight = dbias = ws = None
    if vectors:
        dweight = x.new_empty(xdesc.width, dtype=torch.float32)
        dbias = torch.empty_like(dweight)
        need = lib.ginex_layer_norm_backward_workspace_bytes(xdesc.rows, xdesc.width)
        if need == 0:
            raise GinexError(-1, lib.ginex_last_error().decode())
        ws = _space(workspace, need, x)
    _check(lib.ginex_layer_norm_backward(C.byref(desc), C.byref(xdesc), stats.data_ptr(), w, C.byref(to),
                                         None if dweight is None else dweight.data_ptr(),
                                         None if dbias is None else dbias.data_ptr(), None if ws is None else ws.data_ptr(),
                                         0 if ws is None else ws.numel(), _stream()))
    return dx, dweight, dbias


def _ids(ids):
    _here(ids, "ids")
    if ids.dtype not in (torch.int32, torch.int64):
        raise ValueError(f"ids: expected int32 or int64, got {ids.dtype}")
    if ids.dim() != 1 or not ids.is_contiguous():
        raise ValueError("ids: expected a contiguous tensor of one dimension")
    return int(ids.dtype == torch.int64)


class Lookup(torch.autograd.Function):
    """Rows of a table."""

    @staticmethod
    def forward(ctx, table, ids, scale):
        ctx.save_for_backward(ids)
        ctx.rows, ctx.scale = table.shape[0], scale
        return lookup(table, ids, scale)

    @staticmethod
    @_first_derivative
    def backward(ctx, grad):
        ids, = ctx.saved_tensors
        return lookup_backward(grad.contiguous(), ids, ctx.rows, ctx.scale), None, None


def lookup(table, ids, scale=1.0, out=None):
    """ginex_lookup: ``scale`` times the rows ``ids`` (int32 or int64) of ``table``; 0 for an id outside of it."""
    if out is None:
        at = _quick_for(table)
        got = at and at[0].lookup(at[1], at[2], table, ids, scale)
        if got:
            _check(got[0])
            return got[1]
    desc = _rows(table, "table")
    wide = _ids(ids)
    if _any_grad(table):
        _recorded(out)
        return Lookup.apply(table, ids, scale)
    out, to = _out(out, "out", (ids.numel(), desc.width), table.dtype, table)
    _check(_lib.load().ginex_lookup(C.byref(desc), ids.data_ptr(), wide, scale, C.byref(to), _stream()))
    return out


def lookup_backward(grad, ids, rows, scale=1.0, out=None, workspace=None):
    """ginex_lookup_backward: the gradient of a table of ``rows`` rows, of ``grad``'s type."""
    if out is None and workspace is None:
        at = _quick_for(grad)
        got = at and at[0].lookup_backward(at[1], at[2], grad, ids, rows, scale)
        if got:
            _check(got[0])
            return got[1]
    lib = _lib.load()
    desc = _rows(grad, "grad")
    wide = _ids(ids)
    if ids.numel() != desc.rows:
        raise ValueError(f"ids: expected {desc.rows}, got {ids.numel()}")
    need = lib.ginex_lookup_backward_workspace_bytes(desc.rows, rows, desc.width)
    if need == 0:
        raise GinexError(-1, lib.ginex_last_error().decode())
    dtable, to = _out(out, "out", (rows, desc.width), grad.dtype, grad)
    ws = _space(workspace, need, grad)
    _check(lib.ginex_lookup_backward(C.byref(desc), ids.data_ptr(), wide, scale, C.byref(to), ws.data_ptr(), ws.numel(),
                                     _stream()))
    return dtable
