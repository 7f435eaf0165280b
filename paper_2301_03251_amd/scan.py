"""Gated linear recurrence over the steps of sequences, on the library's HIP
kernels (``ql_gated_scan_*``): what carries a sequence's past to the step whose
features a quantum layer encodes.

    h_t = a_t h_{t-1} + (1 - a_t) x_t,  a_t = sigmoid(gate_t)
"""

from __future__ import annotations

import ctypes
import functools

from .norm import has_tangent, on_device, type_of
from .qlayer import _check, _ptr, _stream, _torch, load

BLOCK = 16  # QL_SCAN_BLOCK


@functools.lru_cache(maxsize=1024)
def _workspace_bytes(type_, batch, steps, features):
    out = ctypes.c_size_t()
    _check(load().ql_gated_scan_workspace_bytes(type_, batch, steps, features, ctypes.byref(out)))
    return out.value


def _wide(x):
    torch = _torch()
    return x.dtype if x.dtype == torch.float64 else torch.float32


def _same(t, x, what):
    if t.shape != x.shape or t.dtype != x.dtype or t.get_device() != x.get_device():
        raise ValueError(f"{what} must have x's shape, dtype and device")


def _check_x(x, dims):
    device = x.get_device()
    if device < 0 or x.dim() != dims or x.shape[-1] < 1:
        raise ValueError("x must be a CUDA tensor " + ("[batch, steps, features]" if dims == 3 else "[batch, features]"))
    return device, type_of(x, "x")


def _check_state(s, x, what):
    want = (x.shape[0], x.shape[-1])
    if tuple(s.shape) != want or s.dtype != _wide(x) or s.get_device() != x.get_device():
        raise ValueError(f"{what} must be a {_wide(x)} tensor {want} on x's device")


def _check_starts(starts, x):
    torch = _torch()
    if starts.shape != x.shape[:-1] or starts.dtype != torch.bool or starts.get_device() != x.get_device():
        raise ValueError(f"starts must be a bool tensor {tuple(x.shape[:-1])} on x's device")


def _strided(t):
    """(tensor, its address and strides but the last): a copy where features do not lie side by side."""
    if t.is_neg():
        t = t.resolve_neg()
    if t.stride(-1) != 1 and t.shape[-1] > 1:
        t = t.contiguous()
    return t, (t.data_ptr(), *t.stride()[:-1])


def gated_scan_forward(x, gate, initial=None, starts=None, states=True):
    """(h, last, states) of x and gate [batch, steps, features]: h in x's dtype, and
    in float32 (float64 for float64 x) the last state [batch, features] and, what
    ``gated_scan_backward`` takes, the state before every ``BLOCK`` steps (None
    without ``states``). ``initial`` [batch, features], of last's dtype, is
    the state before the first step (default 0). ``starts`` (bool [batch, steps]) is
    true where a sequence begins: the state before it is 0, whatever came. Autograd
    does not see the call: ``gated_scan`` is the differentiable one."""
    torch = _torch()
    device, t = _check_x(x, 3)
    _same(gate, x, "gate")
    if initial is not None:
        _check_state(initial, x, "initial")
    if starts is not None:
        _check_starts(starts, x)
    there = on_device(device)
    if there is not None:
        with there:
            return gated_scan_forward(x, gate, initial, starts, states)
    batch, steps, features = x.shape
    x, xs = _strided(x)
    gate, zs = _strided(gate)
    if initial is not None:
        initial = initial.contiguous().resolve_neg()
    if starts is not None:
        starts = starts.contiguous()
    wide = _wide(x)
    h = x.new_empty((batch, steps, features))
    last = x.new_empty((batch, features), dtype=wide)
    kept = x.new_empty((batch, (steps + BLOCK - 1) // BLOCK, features), dtype=wide) if states else None
    ws, ws_bytes = None, _workspace_bytes(t, batch, steps, features)
    if ws_bytes:
        ws = x.new_empty(ws_bytes, dtype=torch.uint8)
    _check(load().ql_gated_scan_forward(t, batch, steps, features, *xs, *zs, _ptr(starts), _ptr(initial), _ptr(h), _ptr(last),
                                        _ptr(kept), _ptr(ws), ws_bytes, _stream(x.device)))
    return h, last, kept


def gated_scan_backward(grad_h, x, gate, states, starts=None, grad_last=None, want_initial=True):
    """(grad_x, grad_gate, grad_initial) from the forward's x, gate, starts and
    states; grad_last is what reaches the last state, grad_initial (None if it is
    not wanted) what goes to the first. Autograd does not see the call."""
    torch = _torch()
    device, t = _check_x(x, 3)
    _same(gate, x, "gate")
    _same(grad_h, x, "grad_h")
    batch, steps, features = x.shape
    wide, blocks = _wide(x), (steps + BLOCK - 1) // BLOCK
    if (tuple(states.shape) != (batch, blocks, features) or states.dtype != wide or states.get_device() != device
            or not states.is_contiguous() or states.is_neg()):
        raise ValueError(f"states must be a contiguous {wide} tensor {(batch, blocks, features)} on x's device")
    if starts is not None:
        _check_starts(starts, x)
    if grad_last is not None:
        _check_state(grad_last, x, "grad_last")
    there = on_device(device)
    if there is not None:
        with there:
            return gated_scan_backward(grad_h, x, gate, states, starts, grad_last, want_initial)
    x, xs = _strided(x)
    gate, zs = _strided(gate)
    grad_h, gs = _strided(grad_h)
    if grad_last is not None:
        grad_last = grad_last.contiguous().resolve_neg()
    if starts is not None:
        starts = starts.contiguous()
    gx, gz = x.new_empty((batch, steps, features)), x.new_empty((batch, steps, features))
    gi = x.new_empty((batch, features), dtype=wide) if want_initial else None
    ws, ws_bytes = None, _workspace_bytes(t, batch, steps, features)
    if ws_bytes:
        ws = x.new_empty(ws_bytes, dtype=torch.uint8)
    _check(load().ql_gated_scan_backward(t, batch, steps, features, *gs, *xs, *zs, _ptr(states), _ptr(starts),
                                         _ptr(grad_last), _ptr(gx), _ptr(gz), _ptr(gi), _ptr(ws), ws_bytes,
                                         _stream(x.device)))
    return gx, gz, gi


def gated_scan_step(x, gate, state, starts=None):
    """One step of batch sequences: h [batch, features] of x's dtype from x and gate
    [batch, features]; state [batch, features] (float32, float64 for float64 x;
    contiguous) changes in place. ``starts`` (bool [batch]) takes the state
    before as 0. Not differentiable: refused where autograd would follow it."""
    torch = _torch()
    device, t = _check_x(x, 2)
    _same(gate, x, "gate")
    _check_state(state, x, "state")
    if not state.is_contiguous() or state.is_neg():
        raise ValueError("state must be contiguous, and no view of negatives")
    if starts is not None:
        _check_starts(starts, x)
    if (torch.is_grad_enabled() and any(v.requires_grad for v in (x, gate, state))) or has_tangent(x, gate, state):
        raise ValueError("gated_scan_step is not differentiable: detach its tensors or call it under torch.no_grad()")
    there = on_device(device)
    if there is not None:
        with there:
            return gated_scan_step(x, gate, state, starts)
    batch, features = x.shape
    x, xs = _strided(x)
    gate, zs = _strided(gate)
    if starts is not None:
        starts = starts.contiguous()
    h = x.new_empty((batch, features))
    _check(load().ql_gated_scan_step(t, batch, features, *xs, *zs, _ptr(starts), _ptr(state), _ptr(h), _stream(x.device)))
    if not state.is_inference():
        torch.autograd.graph.increment_version([state])
    return h


@functools.lru_cache(maxsize=None)
def _function():
    torch = _torch()

    class GatedScanFn(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, gate, initial, starts):
            h, last, states = gated_scan_forward(x, gate, initial, starts)
            ctx.set_materialize_grads(False)
            ctx.save_for_backward(x, gate, states, starts)
            return h, last

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, grad_h, grad_last):
            x, gate, states, starts = ctx.saved_tensors
            if grad_h is None:
                if grad_last is None:
                    return None, None, None, None
                grad_h = torch.zeros_like(x)
            return (*gated_scan_backward(grad_h, x, gate, states, starts, grad_last, ctx.needs_input_grad[2]), None)

    return GatedScanFn


def gated_scan(x, gate, initial=None, starts=None):
    """(h, last): ``gated_scan_forward`` of x and gate (CUDA tensors [batch, steps,
    features] of float32, float64, bfloat16 or float16), differentiable once in x,
    gate and initial, in reverse mode (forward mode raises). With last as the next
    call's initial a long sequence goes in parts."""
    torch = _torch()
    ts = [t for t in (x, gate, initial) if t is not None]
    if (torch.is_grad_enabled() and any(t.requires_grad for t in ts)) or has_tangent(*ts):
        return _function().apply(x, gate, initial, starts)
    return gated_scan_forward(x, gate, initial, starts, states=False)[:2]
