"""Gated linear recurrence: refusals (CPU), and forward, backward and the single
step against the formulas in 80 bits (needs an MI355X).

Tolerances follow the kernels' rounding step by step, u the arithmetic's unit
roundoff. In float32 the gate's exponential is off by (2 |z| + 2) u of itself (the product in its
exponent and the instruction), so a and 1 - a by at most k = (2 |z| + 8) u of
themselves. With m the recurrence of magnitudes, a state's error obeys
d_t = a_t d_{t-1} + (k_t + 8 u) m_t: one step's rounding, once in its block's map and once
in the block itself, and the block's in the maps after it. What comes back in the
backward pass obeys the same recurrence from the end.
"""

from __future__ import annotations

import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")
import torch.autograd.forward_ad as fwd  # noqa: E402

import paper_2301_03251_amd as Q  # noqa: E402

F32, F64, BF16, F16 = 0, 1, 2, 3
TYPES = {"f32": torch.float32, "f64": torch.float64, "bf16": torch.bfloat16, "f16": torch.float16}
OUT_U = {"f32": 2.0 ** -24, "f64": 2.0 ** -53, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
gpu = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    return Q.load()


FAKE = ctypes.c_void_p(0x1000)
ODD = ctypes.c_void_p(0x1001)


def _fwd(lib, type_=F32, batch=2, steps=3, n=4, x=FAKE, xb=12, xs=4, z=FAKE, zb=12, zs=4, starts=None, initial=None, h=FAKE, last=None,
         states=None, ws=None, ws_bytes=0):
    return lib.ql_gated_scan_forward(type_, batch, steps, n, x, xb, xs, z, zb, zs, starts, initial, h, last, states, ws,
                                     ws_bytes, None)


BAD_SIZES = [dict(type_=4), dict(batch=-1), dict(n=0), dict(n=(1 << 22) + 1), dict(batch=(1 << 25) + 1), dict(xb=-1), dict(zb=-1)]


@pytest.mark.parametrize("kw,code", [(k, -1) for k in BAD_SIZES] + [
    (dict(steps=-1), -1), (dict(steps=(1 << 30) + 1), -1), (dict(batch=1 << 20, steps=1 << 30), -1), (dict(xs=-1), -1), (dict(zs=-1), -1),
    (dict(xs=1 << 46), -1), (dict(x=None), -1), (dict(z=None), -1), (dict(h=None), -1), (dict(x=ODD), -1), (dict(z=ODD), -1),
    (dict(h=ODD), -1), (dict(initial=ODD), -1), (dict(last=ODD), -1), (dict(states=ODD), -1), (dict(steps=5000), -1),
    (dict(steps=5000, ws=ctypes.c_void_p(0x1008), ws_bytes=1 << 20), -1), (dict(steps=5000, ws=FAKE, ws_bytes=8), -2),
])
def test_forward_refuses(lib, kw, code):
    assert _fwd(lib, **kw) == code
    assert lib.ql_last_error()


def _bwd(lib, type_=F32, batch=2, steps=3, n=4, g=FAKE, gb=12, gs=4, x=FAKE, xb=12, xs=4, z=FAKE, zb=12, zs=4, states=FAKE,
         starts=None, last=None, gx=FAKE, gz=FAKE, gi=None, ws=None, ws_bytes=0):
    return lib.ql_gated_scan_backward(type_, batch, steps, n, g, gb, gs, x, xb, xs, z, zb, zs, states, starts, last, gx, gz,
                                      gi, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [(k, -1) for k in BAD_SIZES] + [
    (dict(gb=-1), -1), (dict(gs=-1), -1), (dict(g=None), -1), (dict(x=None), -1), (dict(z=None), -1), (dict(states=None), -1),
    (dict(gx=None), -1), (dict(gz=None), -1), (dict(g=ODD), -1), (dict(states=ODD), -1), (dict(last=ODD), -1), (dict(gx=ODD), -1),
    (dict(gz=ODD), -1), (dict(gi=ODD), -1), (dict(steps=5000), -1), (dict(steps=5000, ws=FAKE, ws_bytes=8), -2),
])
def test_backward_refuses(lib, kw, code):
    assert _bwd(lib, **kw) == code
    assert lib.ql_last_error()


def _step(lib, type_=F32, batch=2, n=4, x=FAKE, xb=4, z=FAKE, zb=4, starts=None, state=FAKE, h=FAKE):
    return lib.ql_gated_scan_step(type_, batch, n, x, xb, z, zb, starts, state, h, None)


@pytest.mark.parametrize("kw", BAD_SIZES + [
    dict(x=None), dict(z=None), dict(state=None), dict(h=None), dict(x=ODD), dict(z=ODD), dict(h=ODD),
    dict(state=ctypes.c_void_p(0x1002), type_=BF16),
])
def test_step_refuses(lib, kw):
    assert _step(lib, **kw) == -1
    assert lib.ql_last_error()


def test_workspace_bytes(lib):
    out = ctypes.c_size_t()
    assert lib.ql_gated_scan_workspace_bytes(F32, 1, 8, 1, None) == -1
    assert lib.ql_gated_scan_workspace_bytes(F32, 1, -8, 1, ctypes.byref(out)) == -1
    for steps in (0, 1, 16, 128):
        assert lib.ql_gated_scan_workspace_bytes(F32, 3, steps, 100, ctypes.byref(out)) == 0 and out.value == 0
    assert lib.ql_gated_scan_workspace_bytes(F32, 1, 65536, 64, ctypes.byref(out)) == 0 and out.value > 0
    assert lib.ql_gated_scan_workspace_bytes(F32, 1, 1 << 30, 64, ctypes.byref(out)) == 0 and out.value <= 4096 * 2 * 64 * 4
    assert lib.ql_gated_scan_workspace_bytes(F32, 0, 65536, 64, ctypes.byref(out)) == 0 and out.value == 0


def test_no_sequences(lib):
    assert _fwd(lib, batch=0, x=None, z=None, h=None) == 0
    assert _bwd(lib, batch=0, g=None, x=None, z=None, states=None, gx=None, gz=None) == 0
    assert _step(lib, batch=0, x=None, z=None, state=None, h=None) == 0


def test_python_refuses_cpu_tensors():
    x = torch.zeros(2, 3, 4)
    for bad in (lambda: Q.gated_scan(x, x), lambda: Q.gated_scan_step(x[0], x[0], x[0]), lambda: Q.gated_scan(x.long(), x.long())):
        with pytest.raises(ValueError):
            bad()


# ---------------------------------------------------------------------------
# values

@pytest.fixture(scope="module")
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    Q.load()


def host(t):
    return t.detach().cpu().double().numpy()


class Reference:
    """The recurrence step by step in 80 bits, and the bounds of a kernel's error."""

    def __init__(self, name, x, z, initial=None, starts=None, g=None, g_last=None):
        big = np.longdouble
        x, z = host(x).astype(big), host(z).astype(big)
        batch, steps, n = x.shape
        u, out = (2.0 ** -53 if name == "f64" else 2.0 ** -24), 1.01 * OUT_U[name]
        tiny = 6e-8 * (name == "f16") + 1e-30
        e = np.exp(-np.abs(z))
        a = np.where(z >= 0, 1, e) / (1 + e)
        rest = np.where(z >= 0, e, 1) / (1 + e)
        k = (2 * np.minimum(np.abs(z), 100) + 8) * u
        starts = np.zeros((batch, steps), bool) if starts is None else starts.cpu().numpy()
        h, d, m, before, d_before = (np.empty_like(x) for _ in range(5))
        s = np.zeros((batch, n), big) if initial is None else host(initial).astype(big)
        ds, ms = np.zeros_like(s), np.abs(s)
        for t in range(steps):
            go = ~starts[:, t, None]
            s, ds, ms = np.where(go, s, 0), np.where(go, ds, 0), np.where(go, ms, 0)
            before[:, t], d_before[:, t] = s, ds
            s = a[:, t] * s + rest[:, t] * x[:, t]
            ms = a[:, t] * ms + rest[:, t] * np.abs(x[:, t])
            ds = a[:, t] * ds + (k[:, t] + 8 * u) * ms
            h[:, t], d[:, t], m[:, t] = s, ds, ms
        self.h, self.dh = h, d + out * np.abs(h) + tiny
        self.last, self.dlast = s, ds + tiny
        if g is None:
            return
        g = host(g).astype(big)
        G, dG = np.empty_like(x), np.empty_like(x)
        s = np.zeros((batch, n), big) if g_last is None else host(g_last).astype(big)
        ds, ms = np.zeros_like(s), np.abs(s)
        for t in range(steps - 1, -1, -1):
            G[:, t] = g[:, t] + s
            ms = ms + np.abs(g[:, t])
            ds = ds + 2 * u * ms
            dG[:, t] = ds
            go = ~starts[:, t, None]
            s = np.where(go, a[:, t] * G[:, t], 0)
            ds = np.where(go, a[:, t] * (ds + (k[:, t] + 8 * u) * ms), 0)
            ms = np.where(go, a[:, t] * ms, 0)
        self.ginitial, self.dginitial = s, ds + tiny
        self.gx = rest * G
        self.dgx = rest * dG + np.abs(self.gx) * (k + 2 * u + out) + tiny
        q = (before - x) * a * rest
        dq = a * rest * (d_before + u * (np.abs(before) + np.abs(x))) + np.abs(q) * (2 * k + 4 * u)
        self.gz = G * q
        self.dgz = np.abs(q) * dG + np.abs(G) * dq + np.abs(self.gz) * (2 * u + out) + tiny


def near(got, want, bound, what):
    got = host(got)
    assert got.shape == want.shape and np.isfinite(got).all(), what
    off = np.abs(got - want) - bound
    assert off.size == 0 or (off <= 0).all(), \
        f"{what}: {float(np.max(off)):.3e} over the bound at {np.unravel_index(np.argmax(off), off.shape)}"


def make(batch, steps, n, dtype, seed, initial=True, starts=True):
    r = np.random.default_rng(seed)
    t = lambda a, d=dtype: torch.from_numpy(np.asarray(a)).to("cuda", d)  # noqa: E731
    wide = torch.float64 if dtype == torch.float64 else torch.float32
    x, g = t(r.normal(size=(batch, steps, n))), t(r.normal(size=(batch, steps, n)))
    z = t(2 + 2 * r.normal(size=(batch, steps, n)))
    first = t(r.normal(size=(batch, n)), wide) if initial else None
    begin = t(r.random((batch, steps)) < 0.05, torch.bool) if starts else None
    return x, z, first, begin, g, t(r.normal(size=(batch, n)), wide)


def check_case(name, x, z, initial, starts, g, g_last):
    ref = Reference(name, x, z, initial, starts, g, g_last)
    h, last, states = Q.gated_scan_forward(x, z, initial, starts)
    near(h, ref.h, ref.dh, "h")
    near(last, ref.last, ref.dlast, "last")
    gx, gz, gi = Q.gated_scan_backward(g, x, z, states, starts, g_last)
    near(gx, ref.gx, ref.dgx, "grad_x")
    near(gz, ref.gz, ref.dgz, "grad_gate")
    near(gi, ref.ginitial, ref.dginitial, "grad_initial")
    return h, last, states


# one wavefront, four and eight; blocks and turns cut short; few columns in segments
SHAPES = [(1, 1, 1), (2, 1, 5), (3, 2, 7), (1, 15, 3), (2, 16, 64), (2, 17, 65), (1, 63, 10), (4, 64, 16), (2, 65, 33), (1, 255, 64),
          (1, 256, 64), (2, 257, 40), (3, 300, 130), (1, 1000, 64), (1, 4097, 5), (2, 5000, 9), (5, 700, 200), (300, 40, 70)]


@gpu
@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("initial,starts", [(False, False), (True, True)])
@pytest.mark.parametrize("batch,steps,n", SHAPES)
def test_values(need_gpu, batch, steps, n, initial, starts, name):
    check_case(name, *make(batch, steps, n, TYPES[name], seed=steps + n, initial=initial, starts=starts))


@gpu
@pytest.mark.parametrize("batch,steps,n,name", [(1, 66000, 3, "f32"), (1, 66000, 1, "bf16"), (40, 3000, 128, "bf16"), (9, 260, 2048, "f32")])
def test_long_and_wide(need_gpu, batch, steps, n, name):
    check_case(name, *make(batch, steps, n, TYPES[name], seed=steps))


@gpu
@pytest.mark.parametrize("steps", [5, 40, 300, 3000])
def test_sequences_and_gradients_are_optional(need_gpu, steps):
    x, z, initial, starts, g, g_last = make(3, steps, 24, torch.float32, seed=steps)
    check_case("f32", x, z, None, starts, g, None)
    check_case("f32", x, z, initial, None, g, g_last)
    h, last, none = Q.gated_scan_forward(x, z, initial, starts, states=False)
    want = Q.gated_scan_forward(x, z, initial, starts)
    assert none is None and torch.equal(h, want[0]) and torch.equal(last, want[1])
    a = Q.gated_scan_backward(g, x, z, want[2], starts, want_initial=False)
    b = Q.gated_scan_backward(g, x, z, want[2], starts, torch.zeros_like(last))
    assert a[2] is None and torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@gpu
@pytest.mark.parametrize("name", ["f32", "bf16", "f64"])
@pytest.mark.parametrize("batch,steps,n", [(3, 50, 10), (2, 400, 65), (1, 3000, 12)])
def test_strides(need_gpu, name, batch, steps, n):
    """Halves of one array, steps before sequences, features apart, repeated rows, negatives."""
    x, z, initial, starts, g, g_last = make(batch, steps, n, TYPES[name], seed=n)

    def run(x, z, starts, g):
        h, last, states = Q.gated_scan_forward(x, z, initial, starts)
        return (h, last, *Q.gated_scan_backward(g, x, z, states, starts, g_last))

    want = run(x, z, starts, g)
    both = torch.full((batch, steps, 2 * n + 3), float("nan"), dtype=x.dtype, device="cuda")
    both[..., 1:n + 1], both[..., n + 2:2 * n + 2] = x, z
    turned = lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)  # noqa: E731
    apart = lambda t: t.transpose(1, 2).contiguous().transpose(1, 2)  # noqa: E731
    for args in ((both[..., 1:n + 1], both[..., n + 2:2 * n + 2], starts, g), (turned(x), turned(z), turned(starts), turned(g)),
                 (apart(x), apart(z), starts, apart(g)), (torch._neg_view(-x), torch._neg_view(-z), starts, torch._neg_view(-g))):
        assert all(torch.equal(p, q) for p, q in zip(run(*args), want))
    wide = lambda t: t[:1, :1].expand(batch, steps, n)  # noqa: E731
    assert all(torch.equal(p, q) for p, q in zip(run(wide(x), wide(z), starts[:1].expand(batch, steps), wide(g)),
                                                 run(wide(x).contiguous(), wide(z).contiguous(),
                                                     starts[:1].repeat(batch, 1), wide(g).contiguous())))
    one = torch.ones((), dtype=x.dtype, device="cuda").expand(batch, steps, n)
    assert all(torch.equal(p, q) for p, q in zip(run(x, z, None, one), run(x, z, None, one.contiguous())))


@gpu
def test_no_steps(need_gpu):
    x = torch.empty((3, 0, 5), device="cuda")
    initial, g_last = torch.randn(3, 5, device="cuda"), torch.randn(3, 5, device="cuda")
    h, last, states = Q.gated_scan_forward(x, x, initial)
    assert h.shape == (3, 0, 5) and states.shape == (3, 0, 5) and torch.equal(last, initial)
    assert not Q.gated_scan_forward(x, x)[1].any()
    assert torch.equal(Q.gated_scan_backward(x, x, x, states, None, g_last)[2], g_last)
    h, last = Q.gated_scan(torch.empty((0, 4, 5), device="cuda"), torch.empty((0, 4, 5), device="cuda"))
    assert h.shape == (0, 4, 5) and last.shape == (0, 5)


@gpu
@pytest.mark.parametrize("steps", [40, 600, 5000])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_bad_values_stay_in_their_sequence(need_gpu, steps, bad):
    """In x, in the gate, in a gradient and in the initial state; sequences behind one
    another, of one and of many steps, and beside one another."""
    x, z, initial, starts, g, g_last = make(2, steps, 20, torch.float32, seed=steps)
    starts[:] = False
    bounds = [0, steps // 3, steps // 3 + 1, steps // 2, steps - 3]
    starts[:, bounds[1:]] = True

    def run():
        h, last, states = Q.gated_scan_forward(x, z, initial, starts)
        return (h, last, *Q.gated_scan_backward(g, x, z, states, starts, g_last))

    want = run()
    own = slice(steps // 2, steps - 3)
    inside = torch.zeros(2, steps, dtype=torch.bool, device="cuda")
    inside[0, own] = True
    at = steps // 2 + max(1, (steps - 3 - steps // 2) // 3)
    for t in (x, z, g):
        held = t[0, at].clone()
        t[0, at] = bad
        h, last, gx, gz, gi = run()
        for p, q in ((h, want[0]), (gx, want[2]), (gz, want[3])):
            assert torch.equal(p[~inside], q[~inside])
        assert torch.equal(last, want[1]) and torch.equal(gi, want[4])
        if t is x:
            assert torch.equal(h[0, :at], want[0][0, :at]) and not torch.isfinite(h[0, at:steps - 3]).any()
        if t is g:
            assert torch.equal(h, want[0]) and torch.equal(gx[0, at + 1:], want[2][0, at + 1:])
            assert not torch.isfinite(gx[0, steps // 2:at + 1]).any()
        t[0, at] = held
    initial[1] = bad
    h, last, gx, gz, gi = run()
    first = torch.zeros_like(inside)
    first[1, :bounds[1]] = True
    assert torch.equal(h[~first], want[0][~first]) and torch.equal(last, want[1]) and torch.equal(gi, want[4])
    assert torch.equal(gx, want[2]) and torch.equal(gz[~first], want[3][~first])
    starts[:, 0] = True  # and not at all where a sequence starts at once
    assert torch.isfinite(run()[0]).all() and not run()[4].any()


@gpu
@pytest.mark.parametrize("name", ["f32", "f64", "bf16"])
def test_gates_that_keep_and_forget_all(need_gpu, name):
    """z far from 0 and infinite: a is 1 or 0, and 1 - a the other."""
    x, z, initial, starts, g, g_last = make(2, 300, 16, TYPES[name], seed=4, starts=False)
    z[:, 50:200] = 60.0
    z[:, 100:150, :8] = float("inf")
    z[:, 200:250] = -60.0
    z[:, 220:230] = -float("inf")
    z[:, 280:] = 1e4
    check_case(name, x, z, initial, None, g, g_last)
    h, *_ = Q.gated_scan_forward(x, z, initial)
    # bit by bit inside a block of 16 steps, which runs step by step; the state before
    # a later block comes from the maps of the ones before it, rounded otherwise: the
    # bounds above hold it
    assert torch.equal(h[:, 111, :8], h[:, 100, :8]) and torch.equal(h[:, 220:230], x[:, 220:230])


@gpu
@pytest.mark.parametrize("steps", [7, 100, 3000])
def test_gradients_against_differences(need_gpu, steps):
    """d/dt of sum(g h) + sum(g_last last) along a direction by central differences
    in float64; the step's error is h^2 / 6 of a third derivative, of order 1 for
    every step that a state remembers (some 10 here), plus rounding over h."""
    x, z, initial, starts, g, g_last = make(2, steps, 6, torch.float64, seed=steps)
    dx, dz = torch.randn_like(x), torch.randn_like(z)
    di = torch.randn_like(initial)
    h, last, states = Q.gated_scan_forward(x, z, initial, starts)
    gx, gz, gi = Q.gated_scan_backward(g, x, z, states, starts, g_last)
    eps = 1e-4

    def at(t):
        h, last = Q.gated_scan(x + t * dx, z + t * dz, initial + t * di, starts)
        return ((g * h).sum() + (g_last * last).sum()).item()

    got = ((gx * dx).sum() + (gz * dz).sum() + (gi * di).sum()).item()
    size = (g.abs().sum() + g_last.abs().sum()).item()
    assert abs((at(eps) - at(-eps)) / (2 * eps) - got) <= size * (1000 * eps * eps + 1e-13 / eps)


@gpu
def test_autograd(need_gpu):
    x, z, initial, starts, g, g_last = make(3, 90, 20, torch.float32, seed=2)
    h, last, states = Q.gated_scan_forward(x, z, initial, starts)
    want = Q.gated_scan_backward(g, x, z, states, starts, g_last)
    leaves = [t.requires_grad_() for t in (x, z, initial)]
    a, b = Q.gated_scan(x, z, initial, starts)
    assert torch.equal(a, h) and torch.equal(b, last)
    got = torch.autograd.grad([a, b], leaves, [g, g_last])
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    zero = torch.zeros_like(x)
    for outs, gs, w in (([0], [g], Q.gated_scan_backward(g, x, z, states, starts)),
                        ([1], [g_last], Q.gated_scan_backward(zero, x, z, states, starts, g_last))):
        y = Q.gated_scan(x, z, initial, starts)
        got = torch.autograd.grad([y[o] for o in outs], leaves, gs)
        assert all(torch.equal(p, q) for p, q in zip(got, w))
    # one array for both
    y = Q.gated_scan(x, x, None, None)[0]
    h, _, states = Q.gated_scan_forward(x, x)
    gx, gz, _ = Q.gated_scan_backward(g, x, x, states)
    assert torch.equal(torch.autograd.grad(y, x, g)[0], gx + gz)
    y = Q.gated_scan(x.detach(), z, None, starts)[0]
    assert torch.autograd.grad(y, z, g)[0].shape == z.shape
    with fwd.dual_level(), pytest.raises(RuntimeError, match="forward mode AD"):
        Q.gated_scan(fwd.make_dual(x.detach(), x.detach()), z.detach())
    with torch.no_grad():
        assert torch.equal(Q.gated_scan(x, z, initial, starts)[0], a)
        saved = z * 1
    saved.requires_grad_()
    y = Q.gated_scan(x, saved * 1, initial, starts)[0]
    starts.logical_not_()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


@gpu
def test_in_parts(need_gpu):
    """A long sequence in parts, state handed on, forward and backward."""
    x, z, initial, starts, g, g_last = make(2, 700, 30, torch.float32, seed=6)
    ref = Reference("f32", x, z, initial, starts, g, g_last)
    parts, kept, state = [slice(0, 1), slice(1, 300), slice(300, 316), slice(316, 700)], [], initial
    for p in parts:
        h, state, states = Q.gated_scan_forward(x[:, p], z[:, p], state, starts[:, p])
        kept.append(states)
        near(h, ref.h[:, p], ref.dh[:, p], "h")
    near(state, ref.last, ref.dlast, "last")
    back = g_last
    for p, states in zip(parts[::-1], kept[::-1]):
        gx, gz, back = Q.gated_scan_backward(g[:, p], x[:, p], z[:, p], states, starts[:, p], back)
        near(gx, ref.gx[:, p], ref.dgx[:, p], "grad_x")
        near(gz, ref.gz[:, p], ref.dgz[:, p], "grad_gate")
    near(back, ref.ginitial, ref.dginitial, "grad_initial")


@gpu
@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("batch,n", [(1, 1), (3, 5), (64, 16), (7, 130), (256, 1024)])
def test_steps(need_gpu, name, batch, n):
    """Step by step, each sequence starting where it says so; rows of a wider array."""
    steps = 6
    x, z, initial, starts, *_ = make(batch, steps, n, TYPES[name], seed=n)
    starts[:, 3] = torch.arange(batch, device="cuda") % 2 == 0
    ref = Reference(name, x, z, initial, starts)
    state = initial.clone()
    both = torch.cat((x, z), -1)
    for t in range(steps):
        version = state._version
        h = Q.gated_scan_step(both[:, t, :n], both[:, t, n:], state, starts[:, t])
        near(h, ref.h[:, t], ref.dh[:, t], "h")
        assert state._version > version
    near(state, ref.last, ref.dlast, "state")
    again = initial.clone()
    for t in range(steps):
        assert Q.gated_scan_step(x[:, t].contiguous(), z[:, t].contiguous(), again, starts[:, t].contiguous()).shape == (batch, n)
    assert torch.equal(again, state)
    whole = initial.clone()
    Q.gated_scan_step(x[:, 0], z[:, 0], whole)
    near(whole, *(lambda r: (r.last, r.dlast))(Reference(name, x[:, :1], z[:, :1], initial)), "state")


@gpu
def test_python_refuses(need_gpu):
    x, z, initial, starts, g, g_last = make(2, 40, 6, torch.bfloat16, seed=2)
    h, last, states = Q.gated_scan_forward(x, z, initial, starts)
    for bad in (lambda: Q.gated_scan(x[0], z[0]), lambda: Q.gated_scan(x, z[:1]), lambda: Q.gated_scan(x, z.float()),
                lambda: Q.gated_scan(x, z, initial.bfloat16()), lambda: Q.gated_scan(x, z, initial[:1]),
                lambda: Q.gated_scan(x, z, None, starts.int()), lambda: Q.gated_scan(x, z, None, starts[:, 1:]),
                lambda: Q.gated_scan(x, z, None, starts.cpu()), lambda: Q.gated_scan(x, z.cpu()),
                lambda: Q.gated_scan(x[..., :0], z[..., :0]),
                lambda: Q.gated_scan_backward(g[:, 1:], x, z, states), lambda: Q.gated_scan_backward(g, x, z, states[:, 1:]),
                lambda: Q.gated_scan_backward(g, x, z, states.bfloat16()), lambda: Q.gated_scan_backward(g, x, z, states, None, g_last.half()),
                lambda: Q.gated_scan_step(x, z, initial), lambda: Q.gated_scan_step(x[:, 0], z[:, 0], initial.half()),
                lambda: Q.gated_scan_step(x[:, 0], z[:, 0], initial.t().contiguous().t()),
                lambda: Q.gated_scan_step(x[:, 0], z[:, 0], torch._neg_view(initial)),
                lambda: Q.gated_scan_step(x[:, 0], z[:, 0], initial, starts),
                lambda: Q.gated_scan_step(x[:, 0], z[:, 0], initial.clone().requires_grad_())):
        with pytest.raises(ValueError):
            bad()


@gpu
@pytest.mark.parametrize("steps", [40, 3000])
def test_other_stream_and_graph(need_gpu, steps):
    x, z, initial, starts, g, g_last = make(2, steps, 50, torch.bfloat16, seed=3)
    state = initial.clone()

    def run():
        h, last, states = Q.gated_scan_forward(x, z, initial, starts)
        return (h, last, *Q.gated_scan_backward(g, x, z, states, starts, g_last), Q.gated_scan_step(x[:, 0], z[:, 0], state))

    want = run()
    state.copy_(initial)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        got = run()
    torch.cuda.current_stream().wait_stream(stream)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for seed in range(3):
        for t, v in zip((x, z, initial, starts), make(2, steps, 50, torch.bfloat16, seed=30 + seed)):
            t.copy_(v)
        state.copy_(initial)
        want = run()
        state.copy_(initial)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, want))


@gpu
def test_same_bits_again(need_gpu):
    x, z, initial, starts, g, g_last = make(3, 5000, 40, torch.float32, seed=5)
    h, last, states = Q.gated_scan_forward(x, z, initial, starts)
    first = Q.gated_scan_backward(g, x, z, states, starts, g_last)
    for _ in range(3):
        again = Q.gated_scan_forward(x, z, initial, starts)
        assert all(torch.equal(p, q) for p, q in zip(again, (h, last, states)))
        assert all(torch.equal(p, q) for p, q in zip(Q.gated_scan_backward(g, x, z, states, starts, g_last), first))


@gpu
def test_offsets_past_32_bits(need_gpu):
    batch, steps, n = 2, 40000, 33000
    x = torch.zeros((batch, steps, n), dtype=torch.bfloat16, device="cuda")
    z, g = torch.zeros_like(x), torch.zeros_like(x)
    assert x.numel() > 1 << 31
    at = torch.tensor([0, n // 2, n - 1], device="cuda")
    px, pz, _, _, pg, _ = make(batch, steps, 3, torch.bfloat16, seed=9)
    x[..., at], z[..., at], g[..., at] = px, pz, pg
    h, last, states = Q.gated_scan_forward(x, z)
    gx, gz, _ = Q.gated_scan_backward(g, x, z, states)
    ref = Reference("bf16", px, pz, None, None, pg)
    near(h[..., at], ref.h, ref.dh, "h")
    near(last[..., at], ref.last, ref.dlast, "last")
    near(gx[..., at], ref.gx, ref.dgx, "grad_x")
    near(gz[..., at], ref.gz, ref.dgz, "grad_gate")


@gpu
@pytest.mark.parametrize("steps", [10, 60, 400])
def test_sequences_gigabytes_apart(need_gpu, steps):
    """Their columns lie further from a workgroup's first than 32 bits of bytes: the same bits."""
    x, z, initial, starts, g, g_last = make(2, steps, 10, torch.bfloat16, seed=3)
    far = torch.empty((1 << 32) + 20 * steps, dtype=torch.bfloat16, device="cuda")
    both = far.as_strided((2, steps, 20), (1 << 32, 20, 1))
    both[..., :10], both[..., 10:] = x, z

    def run(x, z):
        h, last, states = Q.gated_scan_forward(x, z, initial, starts)
        return (h, last, *Q.gated_scan_backward(g, x, z, states, starts, g_last))

    assert all(torch.equal(p, q) for p, q in zip(run(both[..., :10], both[..., 10:]), run(x, z)))
