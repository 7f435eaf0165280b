"""Embedding lookup and its gradient by sorted tokens, on the library's HIP
kernels (``ql_embedding_*``): the features that a network's tokens begin with.
"""

from __future__ import annotations

import ctypes
import functools

from .norm import _rows, has_tangent, on_device, type_of
from .qlayer import _check, _stream, _torch, load


@functools.lru_cache(maxsize=1024)
def _workspace_bytes(type_, tokens, rows, features):
    out = ctypes.c_size_t()
    _check(load().ql_embedding_workspace_bytes(type_, tokens, rows, features, ctypes.byref(out)))
    return out.value


def _check_tokens(tokens, device):
    """1 for int64 tokens, 0 for int32."""
    torch = _torch()
    if tokens.dtype not in (torch.int64, torch.int32) or tokens.get_device() != device or device < 0:
        raise ValueError("tokens must be an int64 or int32 CUDA tensor on the other tensors' device")
    return int(tokens.dtype == torch.int64)


def _padding(padding):
    """(whether there is one, it) as the C entries take them."""
    if padding is None:
        return 0, 0
    padding = int(padding)
    if not -(1 << 63) <= padding < 1 << 63:
        raise ValueError("padding must be a 64-bit integer")
    return 1, padding


def embedding_forward(tokens, weight, scale=1.0, padding=None):
    """Rows of weight [rows, features] for tokens [...], times ``scale``: [...,
    features]. Tokens equal to ``padding`` (any integer) give zeros; others
    outside [0, rows) give NaN, as nothing on the host reads them. Autograd does not
    see the call: ``embedding`` is the differentiable one."""
    if weight.dim() != 2:
        raise ValueError("weight must be a CUDA tensor [rows, features]")
    device, t = weight.get_device(), type_of(weight, "weight")
    wide = _check_tokens(tokens, device)
    there = on_device(device)
    if there is not None:
        with there:
            return embedding_forward(tokens, weight, scale, padding)
    rows, features = weight.shape
    if features and not weight.is_contiguous():
        weight, _, stride = _rows(weight, weight.shape)
    else:
        weight, stride = weight.resolve_neg(), features
    tokens = tokens.contiguous().resolve_neg()
    y = weight.new_empty((*tokens.shape, features))
    _check(load().ql_embedding_forward(t, wide, tokens.numel(), rows, features, tokens.data_ptr(), weight.data_ptr(),
                                       stride, scale, *_padding(padding), y.data_ptr(), _stream(weight.device)))
    return y


def embedding_backward(grad, tokens, rows, scale=1.0, padding=None):
    """The gradient [rows, features] of the table from grad [..., features] and the
    forward's tokens [...]: sums in an order that the call's tokens fix, the same bits
    every time; zeros for rows without tokens. Autograd does not see the call."""
    torch = _torch()
    device, t = grad.get_device(), type_of(grad, "grad")
    wide = _check_tokens(tokens, device)
    if grad.dim() < 1 or grad.shape[:-1] != tokens.shape:
        raise ValueError("grad must be a CUDA tensor [..., features] of tokens [...]")
    there = on_device(device)
    if there is not None:
        with there:
            return embedding_backward(grad, tokens, rows, scale, padding)
    rows, features, n = int(rows), grad.shape[-1], tokens.numel()
    ws_bytes = _workspace_bytes(t, n, rows, features)
    grad, _, stride = _rows(grad, grad.shape)
    tokens = tokens.contiguous().resolve_neg()
    out = grad.new_empty((rows, features))
    ws = grad.new_empty(ws_bytes, dtype=torch.uint8)
    _check(load().ql_embedding_backward(t, wide, n, rows, features, tokens.data_ptr(), grad.data_ptr(), stride, scale,
                                        *_padding(padding), out.data_ptr(), ws.data_ptr(), ws_bytes,
                                        _stream(grad.device)))
    return out


@functools.lru_cache(maxsize=None)
def _function():
    torch = _torch()

    class EmbeddingFn(torch.autograd.Function):
        @staticmethod
        def forward(ctx, tokens, weight, scale, padding):
            ctx.rows, ctx.scale, ctx.padding = weight.shape[0], scale, padding
            ctx.save_for_backward(tokens)
            return embedding_forward(tokens, weight, scale, padding)

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, grad):
            return None, embedding_backward(grad, ctx.saved_tensors[0], ctx.rows, ctx.scale, ctx.padding), None, None

    return EmbeddingFn


def embedding(tokens, weight, scale=1.0, padding=None):
    """``embedding_forward`` of tokens (CUDA tensor [...] of int64 or int32) in
    weight [rows, features] (float32, float64, bfloat16 or float16),
    differentiable once in weight, in reverse mode (forward mode raises). The
    gradient is dense."""
    if (_torch().is_grad_enabled() and weight.requires_grad) or has_tangent(weight):
        return _function().apply(tokens, weight, scale, padding)
    return embedding_forward(tokens, weight, scale, padding)


@functools.lru_cache(maxsize=None)
def _module_class():
    torch = _torch()

    class EmbeddingModule(torch.nn.Module):
        def __init__(self, rows, features, scale, padding, dtype, device):
            super().__init__()
            self.scale, self.padding = float(scale), padding
            self.weight = torch.nn.Parameter(torch.randn(int(rows), int(features), dtype=dtype, device=device))

        def forward(self, tokens):
            return embedding(tokens, self.weight, self.scale, self.padding)

        def extra_repr(self):
            return f"{self.weight.shape[0]}, {self.weight.shape[1]}, scale={self.scale}, padding={self.padding}"

    return EmbeddingModule


def Embedding(rows, features, scale=1.0, padding=None, dtype=None, device="cuda"):
    """``embedding`` as a ``torch.nn.Module`` with a normally distributed table.
    dtype None is torch's default."""
    return _module_class()(rows, features, scale, padding, dtype, device)
