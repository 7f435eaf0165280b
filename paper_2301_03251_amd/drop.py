"""Dropout on the library's HIP kernel (``ql_dropout``): the mask comes from a
counter-based generator and is drawn again where the gradient needs it, so none
is stored, and a captured graph draws a new one at every replay.
"""

from __future__ import annotations

import copy
import functools

from .norm import _check_rows, _rows, has_tangent, on_device
from .qlayer import _check, _stream, _torch, load


def _numbers(key):
    """(seed, offset, device address) of a key."""
    torch = _torch()
    if isinstance(key, torch.Tensor):
        return 0, 0, key.data_ptr()
    seed, offset = (int(k) for k in key)
    if not (0 <= seed < 1 << 64 and 0 <= offset < 1 << 64):
        raise ValueError("seed and offset must be in [0, 2^64)")
    return seed, offset, None


def dropout_forward(x, p, key):
    """y = x / (1 - p) for elements that a generator keeps with probability 1 - p,
    0 for the others (NaN and infinities among them). The mask depends on the
    key and each element's place in x's row-major order alone, so the same
    call takes a gradient back. Autograd does not see the call.

    ``key`` is (seed, offset), each in [0, 2^64), or an int64 CUDA tensor of the
    two, which is read when the kernel runs. Element i is kept where word i mod 4
    of Philox 4x32-10 of the counter (i // 4, offset) under the key seed is at
    least p * 2^32."""
    torch = _torch()
    device, shape, xt = _check_rows(x)
    if isinstance(key, torch.Tensor) and (key.dtype != torch.int64 or key.shape != (2,) or key.get_device() != device
                                          or not key.is_contiguous() or key.is_neg()):
        raise ValueError("key must be (seed, offset) or a contiguous int64 tensor of the two on x's device")
    seed, offset, address = _numbers(key)
    there = on_device(device)
    if there is not None:
        with there:
            return dropout_forward(x, p, key)
    xr, rows, stride = _rows(x, shape)
    y = x.new_empty(shape)
    _check(load().ql_dropout(xt, rows, shape[-1], xr.data_ptr(), stride, p, seed, offset, address, y.data_ptr(),
                             _stream(x.device)))
    return y


@functools.lru_cache(maxsize=None)
def _function():
    torch = _torch()

    class DropoutFn(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, p, key):
            ctx.p = p
            if isinstance(key, torch.Tensor):
                ctx.key = None
                ctx.save_for_backward(key)
            else:
                ctx.key = key = tuple(key)  # the caller's list may change before the backward pass
            return dropout_forward(x, p, key)

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, grad_y):
            return dropout_forward(grad_y, ctx.p, ctx.saved_tensors[0] if ctx.key is None else ctx.key), None, None

    return DropoutFn


def dropout(x, p, key):
    """``dropout_forward`` of x (CUDA tensor [..., features] of float32, float64,
    bfloat16 or float16), differentiable once, in reverse mode (forward mode
    raises). A key tensor must not change before the backward pass."""
    if (_torch().is_grad_enabled() and x.requires_grad) or has_tangent(x):
        return _function().apply(x, p, key)
    return dropout_forward(x, p, key)


@functools.lru_cache(maxsize=None)
def _module_class():
    torch = _torch()

    def new_seed():
        return int(torch.randint((1 << 63) - 1, ()))

    class DropoutModule(torch.nn.Module):
        def __init__(self, p, seed, device):
            super().__init__()
            self.p = float(p)
            if not 0 <= self.p <= 1:
                raise ValueError("p must be in [0, 1]")
            if seed is None:
                seed = new_seed()
            # the seed, and the number of calls so far. No buffer: DistributedDataParallel makes the
            # ranks' buffers alike, and with them their masks
            self.key = torch.tensor([int(seed), 0], dtype=torch.int64, device=device)

        def __deepcopy__(self, memo):
            twin = self.__class__.__new__(self.__class__)
            memo[id(self)] = twin
            twin.__setstate__(copy.deepcopy(self.__dict__, memo))
            twin.key.copy_(torch.tensor([new_seed(), 0], dtype=torch.int64))
            return twin

        def _apply(self, fn, recurse=True):
            super()._apply(fn, recurse)
            self.key = fn(self.key)
            return self

        def _save_to_state_dict(self, destination, prefix, keep_vars):
            super()._save_to_state_dict(destination, prefix, keep_vars)
            destination[prefix + "key"] = self.key if keep_vars else self.key.detach()

        def _load_from_state_dict(self, state, prefix, metadata, strict, missing, unexpected, errors):
            name = prefix + "key"
            key = state.get(name)
            super()._load_from_state_dict({k: v for k, v in state.items() if k != name}, prefix, metadata, strict, missing,
                                          unexpected, errors)
            if key is None:
                if strict:
                    missing.append(name)
            elif key.shape != self.key.shape:
                errors.append(f"size mismatch for {name}: {tuple(key.shape)} in the state, {tuple(self.key.shape)} here")
            elif metadata.get("assign_to_params_buffers"):
                self.key = key
            else:
                self.key.copy_(key)  # in place: a captured graph reads it where it is

        def draw(self):
            """The next call's key, which is counted."""
            key = self.key.clone()
            self.key[1].add_(1)
            return key

        def forward(self, x, key=None):
            if not self.training or self.p == 0:
                return x
            if key is None:
                # a call from inside a backward pass is a recomputation, which must not draw another mask
                if torch._C._current_graph_task_id() != -1:
                    raise RuntimeError("Dropout in a backward pass (recomputation by a checkpoint) needs the first "
                                       "call's key: draw it outside, key = layer.draw(), and call layer(x, key)")
                key = self.draw()
            return dropout(x, self.p, key)

        def extra_repr(self):
            return f"p={self.p}"

    return DropoutModule


def Dropout(p=0.1, seed=None, device="cuda"):
    """``dropout`` as a ``torch.nn.Module``; the identity in evaluation. Its tensor
    ``key`` holds the seed (in [0, 2^63); None draws one from torch's generator)
    and the number of calls so far, which is the offset: every call has a mask of
    its own, in replays of a captured graph too, and a loaded state goes on where
    the saved one was. Layers of a network and processes that train together have each
    its own seed, which ``DistributedDataParallel`` leaves alone; processes that load
    one state set ``key[0]`` anew. A copy (``copy.deepcopy``) draws a seed of its own, as
    None does, and starts at 0: blocks that are copies of one drop other places.

    Recomputation (``torch.utils.checkpoint``) runs a layer again in the backward
    pass, where it must draw the mask that it drew before: what is checkpointed takes
    the key as an argument, ``key = layer.draw()`` outside and ``layer(x, key)``
    inside. Without a key a call in a backward pass raises RuntimeError."""
    return _module_class()(p, seed, device)
