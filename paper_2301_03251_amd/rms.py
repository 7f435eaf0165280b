"""Root-mean-square norm of feature rows with the residual's addition, on the
library's HIP kernels (``ql_rms_norm_*``).

In a network of residual blocks in front of a quantum layer, one pass adds a
block's output to the residual and norms the sum for the next block; for a
product in 8 bits it writes the normed rows as e4m3 with one scale each.
"""

from __future__ import annotations

import ctypes
import functools

from .norm import _check_rows, _parameter, _rows, has_tangent, on_device, types
from .qlayer import _check, _ptr, _stream, _torch, load


@functools.lru_cache(maxsize=1024)
def _workspace_bytes(type_, rows, features, backward):
    out = ctypes.c_size_t()
    _check(load().ql_rms_norm_workspace_bytes(type_, rows, features, backward, ctypes.byref(out)))
    return out.value


def _like_x(t, x, what):
    if t.shape != x.shape or t.dtype != x.dtype or t.get_device() != x.get_device():
        raise ValueError(f"{what} must have x's shape, dtype and device")


def _forward(x, weight, residual, eps, stats, quantized):
    """(y, summed, rstd, scale)."""
    torch = _torch()
    device, shape, xt = _check_rows(x)
    n = shape[-1]
    wt = xt if weight is None else _parameter(weight, device, n, "weight")
    if residual is not None:
        _like_x(residual, x, "residual")
    there = on_device(device)
    if there is not None:
        with there:
            return _forward(x, weight, residual, eps, stats, quantized)
    xr, rows, xs = _rows(x, shape)
    summed, rr, rs = x, None, 0
    if residual is not None:
        rr, _, rs = _rows(residual, shape)
        summed = x.new_empty(shape)
    y = x.new_empty(shape, dtype=torch.float8_e4m3fn if quantized else None)
    wide = x.dtype if xt < 2 else torch.float32
    rstd = x.new_empty(shape[:-1], dtype=wide) if stats else None
    scale = x.new_empty(shape[:-1], dtype=torch.float32) if quantized else None
    ws, ws_bytes = None, _workspace_bytes(xt, rows, n, 0)
    if ws_bytes:
        ws = x.new_empty(ws_bytes, dtype=torch.uint8)
    _check(load().ql_rms_norm_forward(xt, wt, rows, n, xr.data_ptr(), xs, _ptr(rr), rs, _ptr(weight), eps,
                                      _ptr(summed) if residual is not None else None, y.data_ptr(), _ptr(rstd),
                                      _ptr(scale), _ptr(ws), ws_bytes, _stream(x.device)))
    return y, summed, rstd, scale


def rms_norm_forward(x, weight=None, residual=None, eps=1e-6, stats=True):
    """(y, summed, rstd): the norm of the rows of summed = x + residual (x itself
    without a residual) along their last axis; rstd, which with summed is what
    ``rms_norm_backward`` takes, is None without ``stats``. Autograd does not see
    the call: ``rms_norm`` is the differentiable one."""
    return _forward(x, weight, residual, eps, stats, False)[:3]


def rms_norm_quantized(x, weight=None, residual=None, eps=1e-6):
    """(q, scale, summed): ``rms_norm_forward`` with y in 8 bits, for rows of
    float32, bfloat16 or float16. q is float8_e4m3fn and scale float32 [...], the
    row's largest |y| / 448: y = q * scale, rounded to nearest, halves to even. A row
    of zeros has scale 0, one that holds an infinity or NaN has NaN. Not differentiable: refused where autograd would follow it."""
    torch = _torch()
    ts = [t for t in (x, weight, residual) if t is not None]
    if (torch.is_grad_enabled() and any(t.requires_grad for t in ts)) or has_tangent(*ts):
        raise ValueError("rms_norm_quantized is not differentiable: detach its tensors or call it under torch.no_grad()")
    q, summed, _, scale = _forward(x, weight, residual, eps, False, True)
    return q, scale, summed


def rms_norm_backward(grad_y, summed, rstd, weight=None, grad_summed=None, want_x=True, want_weight=True,
                      weight_dtype=None):
    """(grad_x, grad_weight) from the forward's summed and rstd; None for each
    that is not wanted. grad_summed is what reaches summed from elsewhere; grad_x
    is the residual's gradient too. grad_weight has weight's dtype
    (``weight_dtype``, default summed's, without a weight). Autograd does not see
    the call."""
    device, shape, xt = _check_rows(summed)
    n = shape[-1]
    if weight is not None:
        wt, wd = _parameter(weight, device, n, "weight"), weight.dtype
    else:
        wd = summed.dtype if weight_dtype is None else weight_dtype
        wt = types().get(wd, -1)
    _like_x(grad_y, summed, "grad_y")
    if grad_summed is not None:
        _like_x(grad_summed, summed, "grad_summed")
    sd = summed.dtype if xt < 2 else _torch().float32
    if (rstd.shape != shape[:-1] or rstd.dtype != sd or rstd.get_device() != device or not rstd.is_contiguous()
            or rstd.is_neg()):
        raise ValueError(f"rstd must be a contiguous {sd} tensor {tuple(shape[:-1])} on x's device")
    there = on_device(device)
    if there is not None:
        with there:
            return rms_norm_backward(grad_y, summed, rstd, weight, grad_summed, want_x, want_weight, weight_dtype)
    xr, rows, xs = _rows(summed, shape)
    gr, _, gs = _rows(grad_y, shape)
    hr, hs = None, 0
    if grad_summed is not None:
        hr, _, hs = _rows(grad_summed, shape)
    gx = summed.new_empty(shape) if want_x else None
    gw = summed.new_empty(n, dtype=wd) if want_weight else None
    ws_bytes = _workspace_bytes(xt, rows, n, 1)
    ws = summed.new_empty(ws_bytes, dtype=_torch().uint8)
    _check(load().ql_rms_norm_backward(xt, wt, rows, n, gr.data_ptr(), gs, _ptr(hr), hs, xr.data_ptr(), xs,
                                       rstd.data_ptr(), _ptr(weight), _ptr(gx), _ptr(gw), ws.data_ptr(), ws_bytes,
                                       _stream(summed.device)))
    return gx, gw


@functools.lru_cache(maxsize=None)
def _function():
    torch = _torch()

    class RmsNormFn(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, weight, residual, eps):
            y, summed, rstd = rms_norm_forward(x, weight, residual, eps)
            ctx.set_materialize_grads(False)
            ctx.save_for_backward(summed, rstd, weight)
            return y if residual is None else (y, summed)

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, grad_y, grad_summed=None):
            summed, rstd, weight = ctx.saved_tensors
            want_x = ctx.needs_input_grad[0] or ctx.needs_input_grad[2]
            if grad_y is None:
                gx, gw = grad_summed, None
            else:
                gx, gw = rms_norm_backward(grad_y, summed, rstd, weight, grad_summed, want_x, ctx.needs_input_grad[1])
            return gx, gw, gx if ctx.needs_input_grad[2] else None, None

    return RmsNormFn


def rms_norm(x, weight=None, residual=None, eps=1e-6):
    """Root-mean-square norm over the last axis of x (CUDA tensor [...,
    features] of float32, float64, bfloat16 or float16): y = s / sqrt(mean(s^2) +
    eps) * weight, s = x + residual. Returns y, with a residual (y, s): s is
    the next residual. Differentiable once in x, weight and residual, in
    reverse mode (forward mode raises). weight has x's dtype, or is float32
    beside 16-bit rows; residual has x's shape and dtype."""
    torch = _torch()
    ts = [t for t in (x, weight, residual) if t is not None]
    if (torch.is_grad_enabled() and any(t.requires_grad for t in ts)) or has_tangent(*ts):
        return _function().apply(x, weight, residual, eps)
    y, summed, _ = rms_norm_forward(x, weight, residual, eps, stats=False)
    return y if residual is None else (y, summed)


@functools.lru_cache(maxsize=None)
def _module_class():
    torch = _torch()

    class RMSNormModule(torch.nn.Module):
        def __init__(self, features, eps, dtype, device):
            super().__init__()
            self.features, self.eps = int(features), float(eps)
            self.weight = torch.nn.Parameter(torch.ones(self.features, dtype=dtype, device=device))

        def forward(self, x, residual=None):
            return rms_norm(x, self.weight, residual, self.eps)

        def extra_repr(self):
            return f"{self.features}, eps={self.eps}"

    return RMSNormModule


def RMSNorm(features, eps=1e-6, dtype=None, device="cuda"):
    """``rms_norm`` as a ``torch.nn.Module`` with a weight of ones: called with x,
    or with x and a residual. dtype None is torch's default."""
    return _module_class()(features, eps, dtype, device)
