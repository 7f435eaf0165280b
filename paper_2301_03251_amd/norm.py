"""Layer norm of feature rows on the library's HIP kernels (``ql_layer_norm_*``).

In front of a quantum layer it brings a network's features to the range of the
encoding's angles (``weight`` and ``bias`` set scale and offset), and its
backward takes the layer's input gradients on to the layers before it.
"""

from __future__ import annotations

import ctypes
import functools

from .qlayer import _check, _ptr, _stream, _torch, load


_TYPES = {}


def types():
    """torch dtype -> ql_type."""
    if not _TYPES:
        torch = _torch()
        _TYPES.update({torch.float32: 0, torch.float64: 1, torch.bfloat16: 2, torch.float16: 3})
    return _TYPES


def type_of(t, what):
    try:
        return (_TYPES or types())[t.dtype]
    except KeyError:
        raise ValueError(f"{what} must be float32, float64, bfloat16 or float16, got {t.dtype}") from None


def on_device(index):
    """A context in which the device is current (None: it is already)."""
    torch = _torch()
    return None if index == torch.cuda.current_device() else torch.cuda.device(index)


def has_tangent(*tensors):
    """Whether forward mode carries a derivative of one of them (None: no)."""
    fwd = _torch().autograd.forward_ad
    return fwd._current_level >= 0 and any(t is not None and fwd.unpack_dual(t).tangent is not None for t in tensors)


@functools.lru_cache(maxsize=1024)
def _workspace_bytes(type_, rows, features, backward):
    out = ctypes.c_size_t()
    _check(load().ql_layer_norm_workspace_bytes(type_, rows, features, backward, ctypes.byref(out)))
    return out.value


def _rows(t, shape):
    """(tensor, rows, stride between rows) of t's rows along its last axis; a
    copy where they do not lie a fixed stride apart."""
    n = shape[-1]
    if t.is_neg():
        t = t.resolve_neg()
    if len(shape) == 2:
        stride, unit = t.stride()
        if unit == 1 or n == 1:
            return t, shape[0], stride
    elif not t.is_contiguous() and (n == 1 or t.stride(-1) == 1):
        try:
            t = t.view(-1, n)
            return t, t.shape[0], t.stride(0)
        except RuntimeError:
            pass
    t = t.contiguous()
    return t, t.numel() // n, n


def _parameter(p, device, n, what):
    if p.dim() != 1 or p.shape[0] != n or p.get_device() != device or not p.is_contiguous() or p.is_neg():
        raise ValueError(f"{what} must be a contiguous tensor [{n}] on x's device")
    return type_of(p, what)


def _check_rows(x):
    device, shape = x.get_device(), x.shape
    if device < 0 or not shape or shape[-1] < 1:
        raise ValueError("x must be a CUDA tensor [..., features]")
    return device, shape, type_of(x, "x")


def layer_norm_forward(x, weight=None, bias=None, eps=1e-5, stats=True):
    """(y, mean, rstd) of the rows along x's last axis; mean and rstd (what
    ``layer_norm_backward`` takes) are None without ``stats``. Autograd does not
    see the call: ``layer_norm`` is the differentiable one."""
    device, shape, xt = _check_rows(x)
    n, wt = shape[-1], xt
    if weight is not None:
        wt = _parameter(weight, device, n, "weight")
        if bias is not None and _parameter(bias, device, n, "bias") != wt:
            raise ValueError("weight and bias must have the same dtype")
    elif bias is not None:
        wt = _parameter(bias, device, n, "bias")
    there = on_device(device)
    if there is not None:
        with there:
            return layer_norm_forward(x, weight, bias, eps, stats)
    xr, rows, stride = _rows(x, shape)
    y = x.new_empty(shape)
    mean = rstd = None
    if stats:
        mean, rstd = x.new_empty((2, *shape[:-1]), dtype=None if xt < 2 else _torch().float32).unbind(0)
    ws, ws_bytes = None, _workspace_bytes(xt, rows, n, 0)
    if ws_bytes:
        ws = x.new_empty(ws_bytes, dtype=_torch().uint8)
    _check(load().ql_layer_norm_forward(xt, wt, rows, n, xr.data_ptr(), stride, _ptr(weight), _ptr(bias), eps,
                                        y.data_ptr(), _ptr(mean), _ptr(rstd), _ptr(ws), ws_bytes, _stream(x.device)))
    return y, mean, rstd


def layer_norm_backward(grad_y, x, mean, rstd, weight=None, want_x=True, want_weight=True, want_bias=True,
                        weight_dtype=None):
    """(grad_x, grad_weight, grad_bias) from the forward's x, mean and rstd;
    None for each that is not wanted. The gradients of weight and bias have
    weight's dtype (``weight_dtype``, default x's, without a weight). Autograd
    does not see the call."""
    device, shape, xt = _check_rows(x)
    n = shape[-1]
    if weight is not None:
        wt, wd = _parameter(weight, device, n, "weight"), weight.dtype
    else:
        wd = x.dtype if weight_dtype is None else weight_dtype
        wt = types().get(wd, -1)
    if grad_y.shape != shape or grad_y.dtype != x.dtype or grad_y.get_device() != device:
        raise ValueError("grad_y must have x's shape, dtype and device")
    sd = x.dtype if xt < 2 else _torch().float32
    for s in (mean, rstd):
        if s.shape != shape[:-1] or s.dtype != sd or s.get_device() != device or not s.is_contiguous() or s.is_neg():
            raise ValueError(f"mean and rstd must be contiguous {sd} tensors {tuple(shape[:-1])} on x's device")
    there = on_device(device)
    if there is not None:
        with there:
            return layer_norm_backward(grad_y, x, mean, rstd, weight, want_x, want_weight, want_bias, weight_dtype)
    xr, rows, xs = _rows(x, shape)
    gr, _, gs = _rows(grad_y, shape)
    gx = x.new_empty(shape) if want_x else None
    gw = x.new_empty(n, dtype=wd) if want_weight else None
    gb = x.new_empty(n, dtype=wd) if want_bias else None
    ws_bytes = _workspace_bytes(xt, rows, n, 1)
    ws = x.new_empty(ws_bytes, dtype=_torch().uint8)
    _check(load().ql_layer_norm_backward(xt, wt, rows, n, gr.data_ptr(), gs, xr.data_ptr(), xs, mean.data_ptr(),
                                         rstd.data_ptr(), _ptr(weight), _ptr(gx), _ptr(gw), _ptr(gb), ws.data_ptr(),
                                         ws_bytes, _stream(x.device)))
    return gx, gw, gb


@functools.lru_cache(maxsize=None)
def _function():
    torch = _torch()

    class LayerNormFn(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, weight, bias, eps):
            y, mean, rstd = layer_norm_forward(x, weight, bias, eps)
            ctx.weight_dtype = bias.dtype if bias is not None else None
            ctx.save_for_backward(x, weight, mean, rstd)
            return y

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, grad_y):
            x, weight, mean, rstd = ctx.saved_tensors
            want = ctx.needs_input_grad
            return (*layer_norm_backward(grad_y, x, mean, rstd, weight, want[0], want[1], want[2], ctx.weight_dtype),
                    None)

    return LayerNormFn


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """Layer norm over x's last axis (CUDA tensor [..., features] of float32,
    float64, bfloat16 or float16), differentiable once in x, weight and bias, in
    reverse mode (forward mode raises). weight and bias have x's dtype, or are
    float32 beside 16-bit rows."""
    torch = _torch()
    if (torch.is_grad_enabled() and (x.requires_grad or (weight is not None and weight.requires_grad)
                                     or (bias is not None and bias.requires_grad))) or has_tangent(x, weight, bias):
        return _function().apply(x, weight, bias, eps)
    return layer_norm_forward(x, weight, bias, eps, stats=False)[0]


@functools.lru_cache(maxsize=None)
def _module_class():
    torch = _torch()

    class LayerNormModule(torch.nn.Module):
        def __init__(self, features, eps, bias, dtype, device):
            super().__init__()
            self.features, self.eps = int(features), float(eps)
            self.weight = torch.nn.Parameter(torch.ones(self.features, dtype=dtype, device=device))
            self.bias = torch.nn.Parameter(torch.zeros(self.features, dtype=dtype, device=device)) if bias else None

        def forward(self, x):
            return layer_norm(x, self.weight, self.bias, self.eps)

        def extra_repr(self):
            return f"{self.features}, eps={self.eps}, bias={self.bias is not None}"

    return LayerNormModule


def LayerNorm(features, eps=1e-5, bias=True, dtype=None, device="cuda"):
    """``layer_norm`` as a ``torch.nn.Module`` with a weight of ones and a bias
    of zeros. dtype None is torch's default."""
    return _module_class()(features, eps, bias, dtype, device)
