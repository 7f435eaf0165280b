"""Layer norm of feature rows on the library's HIP kernels (``ql_layer_norm_*``).

In front of a quantum layer it brings a network's features to the range of the
encoding's angles (``weight`` and ``bias`` set scale and offset), and its
backward takes the layer's input gradients on to the layers before it.
"""

from __future__ import annotations

import ctypes
import functools

from .qlayer import _check, _ptr, _stream, _torch, load


@functools.lru_cache(maxsize=None)
def types():
    """torch dtype -> ql_type."""
    torch = _torch()
    return {torch.float32: 0, torch.float64: 1, torch.bfloat16: 2, torch.float16: 3}


def type_of(t, what):
    try:
        return types()[t.dtype]
    except KeyError:
        raise ValueError(f"{what} must be float32, float64, bfloat16 or float16, got {t.dtype}") from None


@functools.lru_cache(maxsize=1024)
def _workspace_bytes(type_, rows, features, backward):
    out = ctypes.c_size_t()
    _check(load().ql_layer_norm_workspace_bytes(type_, rows, features, backward, ctypes.byref(out)))
    return out.value


def _rows(t):
    """(tensor, rows, stride between rows) of t's rows along its last axis; a
    copy where they do not lie a fixed stride apart."""
    if t.dim() == 2 and (t.stride(1) == 1 or t.shape[1] == 1):
        rows, stride = t.shape[0], t.stride(0)
        if stride >= 0:
            return t, rows, stride
    if not t.is_contiguous():
        try:
            return _rows(t.view(-1, t.shape[-1]))
        except RuntimeError:
            t = t.contiguous()
    n = t.shape[-1]
    return t, t.numel() // n if n else 0, n


def _parameter(p, x, n, what):
    if p.dim() != 1 or p.shape[0] != n or p.device != x.device or not p.is_contiguous():
        raise ValueError(f"{what} must be a contiguous tensor [{n}] on {x.device}")
    return type_of(p, what)


def _check_rows(x):
    if not x.is_cuda or x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError("x must be a CUDA tensor [..., features]")
    return type_of(x, "x")


def _weight_type(x, xt, weight, bias):
    wt = None
    for p, what in ((weight, "weight"), (bias, "bias")):
        if p is not None:
            t = _parameter(p, x, x.shape[-1], what)
            if wt is not None and t != wt:
                raise ValueError("weight and bias must have the same dtype")
            wt = t
    return xt if wt is None else wt


def _stats_dtype(x):
    torch = _torch()
    return torch.float64 if x.dtype == torch.float64 else torch.float32


def layer_norm_forward(x, weight=None, bias=None, eps=1e-5, stats=True):
    """(y, mean, rstd) of the rows along x's last axis; mean and rstd (what
    ``layer_norm_backward`` takes) are None without ``stats``."""
    torch = _torch()
    xt = _check_rows(x)
    wt = _weight_type(x, xt, weight, bias)
    with torch.cuda.device_of(x):
        xr, rows, stride = _rows(x)
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        mean = rstd = None
        if stats:
            mean, rstd = torch.empty((2, *x.shape[:-1]), dtype=_stats_dtype(x), device=x.device).unbind(0)
        ws_bytes = _workspace_bytes(xt, rows, x.shape[-1], 0)
        ws = torch.empty(ws_bytes, dtype=torch.uint8, device=x.device) if ws_bytes else None
        _check(load().ql_layer_norm_forward(xt, wt, rows, x.shape[-1], xr.data_ptr(), stride, _ptr(weight), _ptr(bias),
                                            eps, y.data_ptr(), _ptr(mean), _ptr(rstd), _ptr(ws), ws_bytes,
                                            _stream(x.device)))
    return y, mean, rstd


def layer_norm_backward(grad_y, x, mean, rstd, weight=None, want_x=True, want_weight=True, want_bias=True,
                        weight_dtype=None):
    """(grad_x, grad_weight, grad_bias) from the forward's x, mean and rstd;
    None for each that is not wanted. The gradients of weight and bias have
    weight's dtype (``weight_dtype``, default x's, without a weight)."""
    torch = _torch()
    xt = _check_rows(x)
    n = x.shape[-1]
    if weight is not None:
        wt, wd = _parameter(weight, x, n, "weight"), weight.dtype
    else:
        wd = x.dtype if weight_dtype is None else weight_dtype
        wt = types().get(wd, -1)
    if grad_y.shape != x.shape or grad_y.dtype != x.dtype or grad_y.device != x.device:
        raise ValueError("grad_y must have x's shape, dtype and device")
    sd = _stats_dtype(x)
    for s in (mean, rstd):
        if s.shape != x.shape[:-1] or s.dtype != sd or s.device != x.device or not s.is_contiguous():
            raise ValueError(f"mean and rstd must be contiguous {sd} tensors {tuple(x.shape[:-1])}")
    with torch.cuda.device_of(x):
        xr, rows, xs = _rows(x)
        gr, _, gs = _rows(grad_y)
        gx = torch.empty(x.shape, dtype=x.dtype, device=x.device) if want_x else None
        gw = torch.empty(n, dtype=wd, device=x.device) if want_weight else None
        gb = torch.empty(n, dtype=wd, device=x.device) if want_bias else None
        ws_bytes = _workspace_bytes(xt, rows, n, 1)
        ws = torch.empty(ws_bytes, dtype=torch.uint8, device=x.device)
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
    float64, bfloat16 or float16), differentiable in x, weight and bias.
    weight and bias have x's dtype, or are float32 beside 16-bit rows."""
    torch = _torch()
    if torch.is_grad_enabled() and (x.requires_grad or (weight is not None and weight.requires_grad)
                                    or (bias is not None and bias.requires_grad)):
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
