"""Root-mean-square norm with the residual's addition: refusals (CPU), and forward,
8-bit output and backward against the formulas in 64 bits (needs an MI355X).

Tolerances are bounds of the kernels' rounding, element by element. With unit
roundoff u of the arithmetic, a sum of squares of depth d is off by (d + 1) u of
itself, so rstd by rr = (d / 2 + 6) u; the other terms are carried on from there,
and outputs are rounded once more. The sum x + residual is rounded once: its
bits are known.
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
EPS = 1e-6
gpu = pytest.mark.gpu


# ---------------------------------------------------------------------------
# refusals: nothing is launched, so the addresses are never read

@pytest.fixture(scope="module")
def lib():
    return Q.load()


FAKE = ctypes.c_void_p(0x1000)
ODD = ctypes.c_void_p(0x1001)


def _fwd(lib, type_=F32, wtype=F32, rows=2, n=4, x=FAKE, xs=4, res=None, rs=0, w=FAKE, eps=EPS, summed=None, y=FAKE, rstd=None,
         scale=None, ws=None, ws_bytes=0):
    return lib.ql_rms_norm_forward(type_, wtype, rows, n, x, xs, res, rs, w, eps, summed, y, rstd, scale, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(type_=4), -1), (dict(wtype=-1), -1), (dict(wtype=F64), -3), (dict(type_=BF16, wtype=F16), -3),
    (dict(type_=F64, wtype=F64, scale=FAKE), -3),
    (dict(rows=-1), -1), (dict(n=0), -1), (dict(n=(1 << 30) + 1), -1), (dict(rows=1 << 40, n=1 << 20), -1),
    (dict(xs=-4), -1), (dict(rows=1 << 30, xs=1 << 30), -1), (dict(res=FAKE, summed=FAKE, rs=-1), -1),
    (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1), (dict(eps=float("inf")), -1),
    (dict(x=None), -1), (dict(y=None), -1), (dict(res=FAKE), -1), (dict(x=ODD), -1), (dict(y=ODD), -1),
    (dict(w=ODD), -1), (dict(res=ODD, summed=FAKE), -1), (dict(res=FAKE, summed=ODD), -1), (dict(rstd=ODD), -1),
    (dict(scale=ctypes.c_void_p(0x1002)), -1),
    (dict(n=70000, xs=70000), -1), (dict(n=70000, xs=70000, ws=FAKE, ws_bytes=8), -2),
    (dict(n=70000, xs=70000, ws=ctypes.c_void_p(0x1004), ws_bytes=1 << 20), -1),
])
def test_forward_refuses(lib, kw, code):
    assert _fwd(lib, **kw) == code
    assert lib.ql_last_error()


def _bwd(lib, type_=F32, wtype=F32, rows=2, n=4, g=FAKE, gs=4, h=None, hs=0, s=FAKE, ss=4, rstd=FAKE, w=FAKE, gx=FAKE, gw=FAKE,
         ws=FAKE, ws_bytes=1 << 20):
    return lib.ql_rms_norm_backward(type_, wtype, rows, n, g, gs, h, hs, s, ss, rstd, w, gx, gw, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(type_=7), -1), (dict(wtype=BF16), -3), (dict(rows=-2), -1), (dict(n=0), -1), (dict(g=None), -1),
    (dict(s=None), -1), (dict(rstd=None), -1), (dict(gs=-1), -1), (dict(ss=-1), -1), (dict(h=FAKE, hs=-1), -1),
    (dict(g=ODD), -1), (dict(h=ODD), -1), (dict(gx=ODD), -1), (dict(gw=ODD), -1), (dict(ws=None), -1),
    (dict(ws=ctypes.c_void_p(0x1004)), -1), (dict(ws_bytes=0), -2),
])
def test_backward_refuses(lib, kw, code):
    assert _bwd(lib, **kw) == code
    assert lib.ql_last_error()


def test_workspace_bytes(lib):
    out = ctypes.c_size_t()
    assert lib.ql_rms_norm_workspace_bytes(F32, 4, 8, 1, None) == -1
    assert lib.ql_rms_norm_workspace_bytes(F32, 4, 0, 1, ctypes.byref(out)) == -1
    for t, size in ((F32, 4), (F64, 8), (BF16, 4), (F16, 4)):
        for rows, n in ((0, 5), (1, 1), (256, 10), (8192, 1024), (3, 100000)):
            assert lib.ql_rms_norm_workspace_bytes(t, rows, n, 1, ctypes.byref(out)) == 0
            assert n * size <= out.value <= 4096 * n * size
            assert lib.ql_rms_norm_workspace_bytes(t, rows, n, 0, ctypes.byref(out)) == 0
            assert (out.value > 0) == (n == 100000)


def test_no_rows_and_nothing_wanted(lib):
    assert _fwd(lib, rows=0, x=None, y=None) == 0
    assert _bwd(lib, gx=None, gw=None, ws=None, ws_bytes=0) == 0


def test_python_refuses_cpu_and_integer_tensors():
    with pytest.raises(ValueError):
        Q.rms_norm(torch.zeros(2, 4))
    with pytest.raises(ValueError):
        Q.rms_norm_forward(torch.zeros(2, 4, dtype=torch.int64))
    with pytest.raises(ValueError, match="not differentiable"):
        Q.rms_norm_quantized(torch.zeros(2, 4, requires_grad=True))


# ---------------------------------------------------------------------------
# values

@pytest.fixture(scope="module")
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    Q.load()


def _f64(t):
    return None if t is None else t.detach().cpu().double().numpy()


def make(rows, n, dtype, wdtype, seed, weight=True, residual=True):
    r = np.random.default_rng(seed)
    t = lambda a, d: torch.from_numpy(np.asarray(a)).to("cuda", d)  # noqa: E731
    x = t(r.normal(size=(rows, n)) * (0.5 + r.random(n)), dtype)
    w = t(1 + 0.3 * r.normal(size=n), wdtype) if weight else None
    res = t(r.normal(size=(rows, n)), dtype) if residual else None
    g = t(r.normal(size=(rows, n)), dtype)
    gs = t(r.normal(size=(rows, n)), dtype) if residual else None
    return x, w, res, g, gs


def added(x, res):
    """x + residual, rounded to its type: from float32 for 16-bit rows."""
    if res is None:
        return x
    return (x.float() + res.float()).to(x.dtype) if x.element_size() == 2 else x + res


class Reference:
    """The formulas in 64 bits from the rounded sum, and the bounds of a kernel's error."""

    def __init__(self, s, w, g, gs, name, wname, eps=EPS):
        s, w, g, gs = _f64(s), _f64(w), _f64(g), _f64(gs)
        rows, n = s.shape
        w = np.ones(n) if w is None else w
        u = 2.0 ** -53 if name == "f64" else 2.0 ** -24
        out, tiny = 1.01 * OUT_U[name], 1e-7 * (name == "f16")
        # depth of the sums: a lane's share of a row, then the lanes; over rows likewise
        d, drow = 80 + n / 1024, 80 + rows / 16
        r = 1 / np.sqrt((s * s).mean(-1, keepdims=True) + eps)
        rr = (d / 2 + 6) * u
        h = s * r
        self.rstd, self.drstd = r[:, 0], r[:, 0] * rr
        self.y = h * w
        self.dy = np.abs(self.y) * (rr + 3 * u + out) + tiny
        self.scale = np.abs(self.y).max(-1) / 448
        self.dscale = self.scale * (rr + 6 * u)
        with np.errstate(invalid="ignore"):
            self.q = self.y / self.scale[:, None]
        if g is None:
            return
        v = g * w
        c = (v * h).mean(-1, keepdims=True)
        dc = (d + 4) * u * np.abs(v * h).mean(-1, keepdims=True) + rr * np.abs(v * h).mean(-1, keepdims=True)
        core = r * (v - h * c)
        self.gx = core + (0 if gs is None else gs)
        self.dgx = (r * (2 * u * np.abs(v) + np.abs(h * c) * (rr + 4 * u) + np.abs(h) * dc) + np.abs(core) * (rr + 3 * u)
                    + 2 * u * (np.abs(core) + np.abs(self.gx)) + out * np.abs(self.gx) + tiny)
        self.gw = (g * h).sum(0)
        self.dgw = (np.abs(g * h).sum(0) * (rr + (drow + 4) * u) + 1.01 * OUT_U[wname] * np.abs(self.gw)
                    + 1e-7 * (wname == "f16"))


def near(got, want, bound, what):
    got = _f64(got).reshape(np.shape(want))
    assert np.isfinite(got).all(), what
    off = np.abs(got - want) - bound
    assert (off <= 0).all(), f"{what}: {np.max(off):.3e} over the bound at {np.unravel_index(np.argmax(off), off.shape)}"


def e4m3_near(q, want):
    """q is want rounded to e4m3, want itself off by 10 u of its size (s w and the
    two factors, each rounded): no further than the roundings of its two ends."""
    u = 2.0 ** -24
    ends = [torch.from_numpy(want * (1 + k * 10 * u)).float().clamp(-448, 448).to(torch.float8_e4m3fn).double().numpy()
            for k in (-1, 1)]
    got = _f64(q).reshape(want.shape)
    assert (got >= np.minimum(*ends)).all() and (got <= np.maximum(*ends)).all()


def check_case(x, w, res, g, gs, name, wname, eps=EPS):
    y, summed, rstd = Q.rms_norm_forward(x, w, res, eps)
    s = added(x, res)
    assert torch.equal(summed, s) and (res is not None or summed is x)
    ref = Reference(s, w, g, gs, name, wname, eps)
    near(y, ref.y, ref.dy, "y")
    near(rstd, ref.rstd, ref.drstd, "rstd")
    gx, gw = Q.rms_norm_backward(g, summed, rstd, w, gs, weight_dtype=TYPES[wname])
    near(gx, ref.gx, ref.dgx, "grad_x")
    near(gw, ref.gw, ref.dgw, "grad_weight")
    if name != "f64":
        q, scale, again = Q.rms_norm_quantized(x, w, res, eps)
        assert torch.equal(again, s)
        near(scale, ref.scale, ref.dscale, "scale")
        e4m3_near(q, ref.q)


# every length class of a row: groups of 16 lanes, wavefronts, workgroups, and
# past the registers of a workgroup; their ends, one element on either side
SHAPES = [(1, 1), (7, 1), (3, 2), (1, 3), (256, 10), (33, 16), (70, 63), (5, 64), (9, 65), (4, 127), (6, 129), (1037, 257),
          (3, 1000), (2, 1025), (5, 2047), (3, 4097), (2, 8191), (2, 16385), (300, 16400), (1, 33000), (2, 70001)]


@gpu
@pytest.mark.parametrize("name,wname", [("f32", "f32"), ("f64", "f64"), ("bf16", "bf16"), ("bf16", "f32"),
                                        ("f16", "f16"), ("f16", "f32")])
@pytest.mark.parametrize("rows,n", SHAPES)
def test_values(need_gpu, rows, n, name, wname):
    check_case(*make(rows, n, TYPES[name], TYPES[wname], seed=rows * 100003 + n, residual=n % 2 == 0 or n > 60), name, wname)


@gpu
@pytest.mark.parametrize("rows,n,name", [(4100, 33, "f32"), (20000, 7, "f64"), (5000, 520, "bf16"), (70000, 4, "f16"),
                                         (270, 33000, "f32")])
def test_many_rows(need_gpu, rows, n, name):
    check_case(*make(rows, n, TYPES[name], TYPES[name], seed=n), name, name)


@gpu
@pytest.mark.parametrize("weight,residual", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("n", [12, 900, 5000, 66000])
def test_without_weight_or_residual(need_gpu, n, weight, residual):
    for name in ("f32", "bf16"):
        check_case(*make(6, n, TYPES[name], TYPES[name], seed=n, weight=weight, residual=residual), name, name)


@gpu
@pytest.mark.parametrize("name", ["f32", "bf16", "f64"])
@pytest.mark.parametrize("n,pad,shift", [(10, 1, 0), (64, 3, 1), (1001, 7, 5), (4099, 2, 3), (33001, 5, 3)])
def test_strides_and_alignment(need_gpu, name, n, pad, shift):
    """Columns of wider arrays, starting at any element."""
    x, w, res, g, gs = make(37, n, TYPES[name], TYPES[name], seed=n)

    def inside(t, extra):
        wide = torch.full((37, n + extra + shift), float("nan"), dtype=t.dtype, device="cuda")
        wide[:, shift:shift + n] = t
        return wide[:, shift:shift + n]

    views = [inside(t, pad + k) for k, t in enumerate((x, res, g, gs))]
    wv = torch.cat([w[:1], w])[1:]  # one element past an aligned address
    assert not views[0].is_contiguous()
    check_case(views[0], wv, views[1], views[2], views[3], name, name)
    y, summed, rstd = Q.rms_norm_forward(views[0], wv)
    near(Q.rms_norm_backward(views[2], summed, rstd, wv)[0], *(lambda r: (r.gx, r.dgx))(Reference(x, w, g, None, name, name)), "grad_x")


@gpu
def test_orders_of_axes(need_gpu):
    """Leading axes that do not collapse, a transposed matrix, repeated rows, negatives."""
    x, w, res, g, gs = make(24, 40, torch.float32, torch.float32, seed=3)
    want, s = Q.rms_norm(x, w, res)
    turn = lambda t: t.view(2, 3, 4, 40).transpose(0, 2)  # noqa: E731
    y, t = Q.rms_norm(turn(x), w, turn(res))
    assert torch.equal(y, turn(want)) and torch.equal(t, turn(s))
    y, t = Q.rms_norm(x.t().contiguous().t(), w, res.t().contiguous().t())
    assert torch.equal(y, want) and torch.equal(t, s)
    y, t = Q.rms_norm(x, w, res[:1].expand(24, 40))
    assert torch.equal(t, x + res[:1]) and torch.equal(y, Q.rms_norm(x + res[:1], w))
    assert torch.equal(Q.rms_norm(s[0], w), want[0])
    assert torch.equal(Q.rms_norm(torch._neg_view(-s), w), want)
    assert torch.equal(Q.layer_norm(torch._neg_view(-s), w), Q.layer_norm(s, w))
    _, summed, rstd = Q.rms_norm_forward(x, w, res)
    a = Q.rms_norm_backward(g[:1].expand(24, 40), summed, rstd, w, gs[:1].expand(24, 40))
    c = Q.rms_norm_backward(g[:1].repeat(24, 1), summed, rstd, w, gs[:1].repeat(24, 1))
    assert all(torch.equal(p, q) for p, q in zip(a, c))
    ones = torch.ones((), device="cuda").expand(24, 40)
    assert torch.equal(Q.rms_norm_backward(ones, summed, rstd, w)[0], Q.rms_norm_backward(ones.contiguous(), summed, rstd, w)[0])


@gpu
def test_no_rows(need_gpu):
    x = torch.empty((0, 12), device="cuda", requires_grad=True)
    w = torch.ones(12, device="cuda", requires_grad=True)
    y, s = Q.rms_norm(x, w, x)
    (y.sum() + s.sum()).backward()
    assert y.shape == s.shape == (0, 12) and x.grad.shape == (0, 12) and not w.grad.any()
    q, scale, _ = Q.rms_norm_quantized(x.detach(), w.detach())
    assert q.shape == (0, 12) and scale.shape == (0,)


@gpu
@pytest.mark.parametrize("n", [10, 300, 5000, 66000])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_bad_value_stays_in_its_row(need_gpu, n, bad):
    x, w, res, g, gs = make(5, n, torch.float32, torch.float32, seed=n)
    want, s, r = Q.rms_norm_forward(x, w, res)
    gx = Q.rms_norm_backward(g, s, r, w, gs)[0]
    p, scale, _ = Q.rms_norm_quantized(x, w, res)
    x[2, n // 2] = bad
    y, s, r = Q.rms_norm_forward(x, w, res)
    hx = Q.rms_norm_backward(g, s, r, w, gs)[0]
    q, other, _ = Q.rms_norm_quantized(x, w, res)
    keep = [0, 1, 3, 4]
    assert torch.isnan(y[2, n // 2]) and torch.isnan(other[2])
    assert torch.isnan(y[2]).all() if bad != bad else (r[2] == 0)
    assert torch.equal(y[keep], want[keep]) and torch.equal(hx[keep], gx[keep])
    assert torch.equal(q[keep].float(), p[keep].float()) and torch.equal(other[keep], scale[keep])


@gpu
@pytest.mark.parametrize("n", [16, 700, 40000])
def test_rows_of_zeros_and_far_from_one(need_gpu, n):
    """Zeros give scale 0 and zeros; rows of 1e-37, 1e-20 and 1e16 fill the 8 bits as others do."""
    x, w, *_ = make(4, n, torch.float32, torch.float32, seed=n, residual=False)
    x *= torch.tensor([[0.0], [1e-37], [1e-20], [1e16]], device="cuda")
    q, scale, _ = Q.rms_norm_quantized(x, w)
    assert scale[0] == 0 and not q[0].float().any()
    ref = Reference(x[1:], w, None, None, "f32", "f32")
    e4m3_near(q[1:], ref.q)
    near(scale[2:], ref.scale[1:], ref.dscale[1:], "scale")


@gpu
@pytest.mark.parametrize("rows,n", [(3, 5), (4, 130), (2, 1030)])
def test_gradients_against_differences(need_gpu, rows, n):
    """d/dt of sum(g y + gs s) at x + t dx, residual + t dr, w + t dw by central
    differences in float64; the step's error is h^2 / 6 of a third derivative of
    order 1 each term, plus rounding over h."""
    x, w, res, g, gs = make(rows, n, torch.float64, torch.float64, seed=n)
    r = np.random.default_rng(n + 1)
    dx, dr, dw = (torch.from_numpy(r.normal(size=s)).cuda() for s in ((rows, n), (rows, n), n))
    y, s, rstd = Q.rms_norm_forward(x, w, res)
    gx, gw = Q.rms_norm_backward(g, s, rstd, w, gs)
    h = 1e-4

    def at(t):
        y, s = Q.rms_norm(x + t * dx, w + t * dw, res + t * dr)
        return (g * y + gs * s).sum().item()

    got = ((gx * (dx + dr)).sum() + (gw * dw).sum()).item()
    size = (g.abs() * (1 + y.abs()) + (gs * s).abs()).sum().item()
    assert abs((at(h) - at(-h)) / (2 * h) - got) <= size * (100 * h * h + 1e-13 / h)


@gpu
def test_autograd_and_module(need_gpu):
    x, w, res, g, gs = make(12, 48, torch.float32, torch.float32, seed=8)
    layer = Q.RMSNorm(48)
    with torch.no_grad():
        layer.weight.copy_(w)
    z, s, r = Q.rms_norm_forward(x, w, res)
    gx, gw = Q.rms_norm_backward(g, s, r, w, gs)
    x.requires_grad_(), res.requires_grad_()
    y, t = layer(x.view(3, 4, 48), res.view(3, 4, 48))
    torch.autograd.backward([y, t], [g.view(3, 4, 48), gs.view(3, 4, 48)])
    assert torch.equal(y.view(12, 48), z) and torch.equal(t.view(12, 48), s)
    assert torch.equal(x.grad, gx) and torch.equal(res.grad, gx) and torch.equal(layer.weight.grad, gw)
    # gradients of one of the two outputs
    x.grad = res.grad = layer.weight.grad = None
    layer(x, res)[0].backward(g)
    only, gw = Q.rms_norm_backward(g, s, r, w)
    assert torch.equal(x.grad, only) and torch.equal(res.grad, only) and torch.equal(layer.weight.grad, gw)
    x.grad = res.grad = layer.weight.grad = None
    layer(x, res)[1].backward(gs)
    assert torch.equal(x.grad, gs) and torch.equal(res.grad, gs) and layer.weight.grad is None
    x.grad = None
    layer(x.detach(), res)[0].backward(g)
    assert x.grad is None
    assert Q.rms_norm_backward(g, s, r, w, want_x=False)[0] is None and Q.rms_norm_backward(g, s, r, w, want_weight=False)[1] is None
    with torch.no_grad():
        assert torch.equal(layer(x, res)[0], z)


@gpu
def test_what_autograd_cannot_follow(need_gpu):
    x, w, *_ = make(3, 8, torch.float32, torch.float32, seed=8)
    with fwd.dual_level(), pytest.raises(RuntimeError, match="forward mode AD"):
        Q.rms_norm(fwd.make_dual(x, x), w)
    with fwd.dual_level(), pytest.raises(ValueError, match="not differentiable"):
        Q.rms_norm_quantized(fwd.make_dual(x, x), w)
    with pytest.raises(RuntimeError):
        torch.func.vmap(Q.rms_norm)(x[None])
    y, s = Q.rms_norm(x, w.requires_grad_(), x)
    s.mul_(2)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


@gpu
def test_python_refuses(need_gpu):
    x, w, res, g, gs = make(4, 8, torch.float32, torch.float32, seed=1)
    y, s, r = Q.rms_norm_forward(x, w, res)
    for bad in (w[:7], w.cpu(), torch.ones(16, device="cuda")[::2], w[None]):
        with pytest.raises(ValueError):
            Q.rms_norm(x, bad, res)
    for bad in (res[:3], res[0], res.half(), res.cpu()):
        with pytest.raises(ValueError):
            Q.rms_norm(x, w, bad)
    with pytest.raises(Q.QLError):
        Q.rms_norm(x, w.double())
    with pytest.raises(Q.QLError):
        Q.rms_norm(x, w, eps=-1.0)
    with pytest.raises(Q.QLError):
        Q.rms_norm_quantized(x.double(), w.double())
    for bad in (dict(grad_y=g[:3]), dict(rstd=r[:3]), dict(rstd=r.double()), dict(grad_summed=gs.half())):
        with pytest.raises(ValueError):
            Q.rms_norm_backward(**{**dict(grad_y=g, summed=s, rstd=r, weight=w), **bad})


@gpu
@pytest.mark.parametrize("n", [200, 40000])
def test_other_stream_and_graph(need_gpu, n):
    """The current stream, and a captured graph replayed with new inputs between
    eager work."""
    x, w, res, g, gs = make(30, n, torch.bfloat16, torch.float32, seed=5)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())

    def step():
        y, s, r = Q.rms_norm_forward(x, w, res)
        q, scale, _ = Q.rms_norm_quantized(x, w, res)
        return (y, s, q.float(), scale, *Q.rms_norm_backward(g, s, r, w, gs))

    want = step()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        got = step()
    torch.cuda.current_stream().wait_stream(stream)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in range(3):
        x.copy_(make(30, n, torch.bfloat16, torch.float32, seed=50 + seed)[0])
        want = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, want))


@gpu
def test_same_bits_again(need_gpu):
    x, w, res, g, gs = make(3000, 321, torch.float32, torch.float32, seed=5)
    y, s, r = Q.rms_norm_forward(x, w, res)
    first = Q.rms_norm_backward(g, s, r, w, gs)
    for _ in range(3):
        assert all(torch.equal(p, q) for p, q in zip(first, Q.rms_norm_backward(g, s, r, w, gs)))


@gpu
def test_offsets_past_32_bits(need_gpu):
    rows, n = 66000, 33000
    x = torch.zeros((rows, n), dtype=torch.bfloat16, device="cuda")
    g = torch.zeros((rows, n), dtype=torch.bfloat16, device="cuda")
    assert x.numel() > 1 << 31
    at = [0, 1, rows // 2, rows - 2, rows - 1]
    part, w, res, gpart, gs = make(len(at), n, torch.bfloat16, torch.float32, seed=9)
    x[at], g[at] = part, gpart
    other = torch.zeros_like(x)
    other[at] = res
    y, s, r = Q.rms_norm_forward(x, w, other)
    gx, gw = Q.rms_norm_backward(g, s, r, w, s)
    sums = added(part, res)
    assert torch.equal(s[at], sums)
    ref = Reference(sums, w, gpart, sums, "bf16", "f32")
    near(y[at], ref.y, ref.dy, "y")
    near(gx[at], ref.gx, ref.dgx, "grad_x")
    near(gw, ref.gw, ref.dgw, "grad_weight")
    del y, gx, s
    q, scale, _ = Q.rms_norm_quantized(x, w, other)
    near(scale[at], ref.scale, ref.dscale, "scale")
    e4m3_near(q[at], ref.q)
