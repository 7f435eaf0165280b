"""Orthogonalised updates of matrix-shaped weights on the library's HIP kernels
(``ql_orthogonalize``, ``ql_muon_step``): the optimiser's step for the matrices
of a hybrid network, its quantum layers' angles as [layers, angles] among them.
"""

from __future__ import annotations

import array
import ctypes
import functools

from .norm import has_tangent, type_of
from .qlayer import _check, _stream, _torch, load

COEFFICIENTS = (3.4445, -4.7750, 2.0315)


class _Ortho(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("a", "b", "c", "eps")] + [("steps", ctypes.c_int32)]


class _Muon(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("lr", "momentum", "weight_decay")] + [("nesterov", ctypes.c_int32)]


@functools.lru_cache(maxsize=64)
def _options(steps, coefficients, eps):
    a, b, c = coefficients
    return _Ortho(a, b, c, eps, steps)


@functools.lru_cache(maxsize=1024)
def _workspace_bytes(type_, shapes):
    """``shapes``: (rows, cols, batch) of every entry."""
    words = array.array("q", [v for s in shapes for v in (*s, *(0,) * 12)])
    out = ctypes.c_size_t()
    _check(load().ql_orthogonalize_workspace_bytes(type_, words.buffer_info()[0], len(shapes), ctypes.byref(out)))
    return out.value


def _viewed(t):
    """t as [batch, rows, cols] without a copy; None where its leading axes do not collapse."""
    if t.dim() < 4:
        return t if t.dim() == 3 else t.unsqueeze(0)
    try:
        return t.view(-1, *t.shape[-2:])
    except RuntimeError:
        return None


def _readable(t):
    """t, or a copy of it whose leading axes collapse and whose memory holds its values."""
    t = t.resolve_neg()
    return t.contiguous() if t.dim() > 3 and _viewed(t) is None else t


def _writable(t, what):
    if t.is_neg():
        raise ValueError(f"{what} must not be a view of negatives")


def _batches(*tensors):
    """The tensors' matrices as views [batch, rows, cols] in step: one of all of
    them, or one for each index of the first axis where they do not collapse."""
    views = [_viewed(t) for t in tensors]
    if all(v is not None for v in views):
        yield views
    else:
        for parts in zip(*tensors):
            yield from _batches(*parts)


def _written(tensors):
    """Tells autograd of writes to the tensors, as torch's own in-place operations do."""
    _torch().autograd.graph.increment_version([t for t in tensors if not t.is_inference()])


def _run(call, type_, words, shapes, device, *options):
    torch = _torch()
    need = _workspace_bytes(type_, tuple(shapes))
    ws = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    _check(call(type_, words.buffer_info()[0], len(shapes), *map(ctypes.byref, options),
                None if ws is None else ws.data_ptr(), need, _stream(device)))


def orthogonalize(g, steps=5, coefficients=COEFFICIENTS, eps=1e-7, out=None):
    """The orthogonalised update of g [..., rows, cols] (CUDA tensor of float32,
    float64, bfloat16 or float16, any strides): g / (|g|_F + eps) with its
    singular values taken towards 1 by ``steps`` Newton-Schulz steps. ``out``
    may be g. Not differentiable: refused where autograd would follow it."""
    torch = _torch()
    t, given = type_of(g, "g"), out
    if not g.is_cuda or g.dim() < 2:
        raise ValueError("g must be a CUDA tensor [..., rows, cols]")
    if (torch.is_grad_enabled() and (g.requires_grad or (out is not None and out.requires_grad))) or has_tangent(g, out):
        raise ValueError("orthogonalize is not differentiable: detach its tensors or call it under torch.no_grad()")
    if out is None:
        out = torch.empty(g.shape, dtype=g.dtype, device=g.device)
    elif out.shape != g.shape or out.dtype != g.dtype or out.device != g.device:
        raise ValueError("out must have g's shape, dtype and device")
    else:
        _writable(out, "out")
    if g.numel() == 0:
        return out
    with torch.cuda.device_of(g):
        g, words, shapes = _readable(g), array.array("q"), []
        for q, o in _batches(g, out):
            batch, rows, cols = q.shape
            shapes.append((rows, cols, batch))
            words.extend((rows, cols, batch, q.data_ptr(), *q.stride(), 0, 0, 0, 0, o.data_ptr(), *o.stride()))
        _run(load().ql_orthogonalize, t, words, shapes, g.device,
             _options(int(steps), tuple(coefficients), float(eps)))
    if given is not None:
        _written((given,))
    return out


def muon_step(params, grads, momenta, lr=0.02, momentum=0.95, nesterov=True, weight_decay=0.0, steps=5,
              coefficients=COEFFICIENTS, eps=1e-7):
    """One step of all matrices [..., rows, cols] of ``params`` (lists of CUDA
    tensors of one dtype on one device), in place:

        m = momentum * m + g,  u = g + momentum * m (nesterov; else m)
        p = (1 - lr * weight_decay) * p - lr * sqrt(max(1, rows / cols)) * orthogonalize(u)

    ``momenta`` are float32 (float64 for float64 weights). Autograd does not
    follow the step."""
    torch = _torch()
    if not len(params) == len(grads) == len(momenta):
        raise ValueError("params, grads and momenta must be lists of the same length")
    if not params:
        return
    first = params[0]
    t, device, dtype = type_of(first, "params"), first.device, first.dtype
    state = torch.float64 if dtype == torch.float64 else torch.float32
    words, shapes = [], []
    held = []  # copies of gradients, whose memory is theirs until the launch
    for p, g, m in zip(params, grads, momenta):
        if not p.is_cuda or p.dim() < 2 or p.dtype != dtype or p.device != device:
            raise ValueError("params must be CUDA tensors [..., rows, cols] of one dtype on one device")
        if g.shape != p.shape or g.dtype != dtype or g.device != device:
            raise ValueError("a gradient must have its parameter's shape, dtype and device")
        if m.shape != p.shape or m.dtype != state or m.device != device:
            raise ValueError(f"a momentum must be {state}, of its parameter's shape and device")
        _writable(p, "a parameter")
        _writable(m, "a momentum")
        if p.numel() == 0:
            continue
        g = _readable(g)
        held.append(g)
        if p.dim() == 2:
            rows, cols = p.shape
            shapes.append((rows, cols, 1))
            words += (rows, cols, 1, g.data_ptr(), 0, *g.stride(), m.data_ptr(), 0, *m.stride(), p.data_ptr(), 0,
                      *p.stride())
        else:
            for gb, mb, pb in _batches(g, m, p):
                batch, rows, cols = pb.shape
                shapes.append((rows, cols, batch))
                words += (rows, cols, batch, gb.data_ptr(), *gb.stride(), mb.data_ptr(), *mb.stride(), pb.data_ptr(),
                          *pb.stride())
    if not shapes:
        return
    with torch.cuda.device_of(first):
        _run(load().ql_muon_step, t, array.array("q", words), shapes, device,
             _Muon(lr, momentum, weight_decay, bool(nesterov)), _options(int(steps), tuple(coefficients), float(eps)))
    _written((*params, *momenta))


@functools.lru_cache(maxsize=None)
def _class():
    torch = _torch()

    def wide(p):
        return torch.float64 if p.dtype == torch.float64 else torch.float32

    class MuonOptimizer(torch.optim.Optimizer):
        def load_state_dict(self, state_dict):
            """As the base class, which gives state its parameter's dtype; a momentum keeps its own."""
            super().load_state_dict(state_dict)
            saved = [i for g in state_dict["param_groups"] for i in g["params"]]
            held = [p for g in self.param_groups for p in g["params"]]
            for i, p in zip(saved, held):
                if "momentum" in state_dict["state"].get(i, {}):
                    m = state_dict["state"][i]["momentum"]
                    self.state[p]["momentum"] = m.detach().to(device=p.device, dtype=wide(p), copy=True)

        @torch.no_grad()
        def step(self, closure=None):
            loss = None
            if closure is not None:
                with torch.enable_grad():
                    loss = closure()
            for group in self.param_groups:
                kinds = {}
                for p in group["params"]:
                    if p.grad is None:
                        continue
                    state = self.state[p]
                    if not state:
                        state["momentum"] = torch.zeros_like(p, dtype=wide(p))
                    kinds.setdefault((p.device, p.dtype), []).append((p, p.grad, state["momentum"]))
                for matrices in kinds.values():
                    lists = [[t if group["matrix"] is None else t.view(group["matrix"]) for t in ts]
                             for ts in zip(*matrices)]
                    muon_step(*lists, **{k: group[k] for k in ("lr", "momentum", "nesterov", "weight_decay", "steps",
                                                              "coefficients", "eps")})
            return loss

    return MuonOptimizer


def Muon(params, lr=0.02, momentum=0.95, nesterov=True, weight_decay=0.0, steps=5, coefficients=COEFFICIENTS, eps=1e-7):
    """``muon_step`` as a ``torch.optim.Optimizer`` over matrices. A group of flat
    weights, such as a quantum layer's, is taken as matrices with the group's
    ``matrix`` = (rows, cols); other vectors belong to another optimiser."""
    defaults = dict(lr=lr, momentum=momentum, nesterov=nesterov, weight_decay=weight_decay, steps=steps,
                    coefficients=tuple(coefficients), eps=eps, matrix=None)
    optimizer = _class()(params, defaults)
    for group in optimizer.param_groups:
        for p in group["params"]:
            if p.dim() < 2 and group["matrix"] is None:
                raise ValueError("Muon takes matrices: give flat weights a group with matrix=(rows, cols)")
    return optimizer
