"""Layer norm: refusals of the C entries (CPU), and forward and backward against
the formulas in 64 bits (needs an MI355X).

Tolerances are bounds of the kernels' rounding, element by element: with unit
roundoff u of the arithmetic and sums of depth s, a mean is off by at most
s u max|x|, so h = (x - mean) rstd by (1 + |h|) (s u max|x| rstd + (s + 4) u), and
what is computed from it by the terms carried on; outputs are rounded once more.
"""

from __future__ import annotations

import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2301_03251_amd as Q  # noqa: E402

F32, F64, BF16, F16 = 0, 1, 2, 3
TYPES = {"f32": torch.float32, "f64": torch.float64, "bf16": torch.bfloat16, "f16": torch.float16}
OUT_U = {"f32": 2.0 ** -24, "f64": 2.0 ** -53, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
EPS = 1e-5


# ---------------------------------------------------------------------------
# refusals: nothing is launched, so the addresses are never read

@pytest.fixture(scope="module")
def lib():
    return Q.load()


FAKE = ctypes.c_void_p(0x1000)
ODD = ctypes.c_void_p(0x1001)


def _fwd(lib, type_=F32, wtype=F32, rows=2, n=4, x=FAKE, stride=4, w=FAKE, b=FAKE, eps=EPS, y=FAKE, mean=None, rstd=None, ws=None,
         ws_bytes=0):
    return lib.ql_layer_norm_forward(type_, wtype, rows, n, x, stride, w, b, eps, y, mean, rstd, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(type_=4), -1), (dict(type_=-1), -1), (dict(wtype=9), -1),
    (dict(wtype=F64), -3), (dict(type_=F64, wtype=F32), -3), (dict(type_=BF16, wtype=F16), -3),
    (dict(rows=-1), -1), (dict(n=0), -1), (dict(n=-3), -1), (dict(n=(1 << 30) + 1), -1),
    (dict(rows=1 << 40, n=1 << 20), -1), (dict(stride=-4), -1), (dict(rows=1 << 30, stride=1 << 30), -1),
    (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1), (dict(eps=float("inf")), -1),
    (dict(x=None), -1), (dict(y=None), -1), (dict(x=ODD), -1), (dict(y=ODD), -1), (dict(w=ODD), -1),
    (dict(n=70000, stride=70000), -1), (dict(n=70000, stride=70000, ws=FAKE, ws_bytes=8), -2),
    (dict(n=70000, stride=70000, ws=ctypes.c_void_p(0x1004), ws_bytes=1 << 20), -1),
    (dict(b=ODD), -1), (dict(mean=ODD), -1), (dict(rstd=ctypes.c_void_p(0x1002)), -1),
])
def test_forward_refuses(lib, kw, code):
    assert _fwd(lib, **kw) == code
    assert lib.ql_last_error()


def _bwd(lib, type_=F32, wtype=F32, rows=2, n=4, g=FAKE, gs=4, x=FAKE, xs=4, mean=FAKE, rstd=FAKE, w=FAKE, gx=FAKE,
         gw=FAKE, gb=FAKE, ws=FAKE, ws_bytes=1 << 20):
    return lib.ql_layer_norm_backward(type_, wtype, rows, n, g, gs, x, xs, mean, rstd, w, gx, gw, gb, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(type_=7), -1), (dict(wtype=BF16), -3), (dict(rows=-2), -1), (dict(n=0), -1), (dict(g=None), -1),
    (dict(x=None), -1), (dict(mean=None), -1), (dict(rstd=None), -1), (dict(gs=-1), -1), (dict(xs=-1), -1),
    (dict(g=ODD), -1), (dict(gx=ODD), -1), (dict(gw=ODD), -1), (dict(gb=ODD), -1),
    (dict(ws=None), -1), (dict(ws=ctypes.c_void_p(0x1004)), -1), (dict(ws_bytes=0), -2),
])
def test_backward_refuses(lib, kw, code):
    assert _bwd(lib, **kw) == code
    assert lib.ql_last_error()


def test_workspace_bytes(lib):
    out = ctypes.c_size_t()
    assert lib.ql_layer_norm_workspace_bytes(F32, 4, 8, 1, None) == -1
    assert lib.ql_layer_norm_workspace_bytes(F32, 4, 0, 1, ctypes.byref(out)) == -1
    for t, size in ((F32, 4), (F64, 8), (BF16, 4), (F16, 4)):
        for rows, n in ((0, 5), (1, 1), (256, 10), (8192, 1024), (3, 100000)):
            assert lib.ql_layer_norm_workspace_bytes(t, rows, n, 1, ctypes.byref(out)) == 0
            assert 2 * n * size <= out.value <= 4096 * 2 * n * size
            assert lib.ql_layer_norm_workspace_bytes(t, rows, n, 0, ctypes.byref(out)) == 0
            assert (out.value > 0) == (n == 100000)


def test_python_refuses_cpu_and_integer_tensors():
    with pytest.raises(ValueError):
        Q.layer_norm(torch.zeros(2, 4))
    with pytest.raises(ValueError):
        Q.layer_norm_forward(torch.zeros(2, 4, dtype=torch.int64))


# ---------------------------------------------------------------------------
# values

gpu = pytest.mark.gpu


@pytest.fixture(scope="module")
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    Q.load()


def _f64(t):
    return None if t is None else t.detach().cpu().double().numpy()


def make(rows, n, dtype, wdtype, seed, offset=1.0, weight=True, bias=True):
    r = np.random.default_rng(seed)
    t = lambda a, d: torch.from_numpy(np.asarray(a)).to("cuda", d)  # noqa: E731
    x = t(r.normal(size=(rows, n)) * (0.5 + r.random(n)) + offset * r.normal(size=n), dtype)
    w = t(1 + 0.3 * r.normal(size=n), wdtype) if weight else None
    b = t(0.3 * r.normal(size=n), wdtype) if bias else None
    g = t(r.normal(size=(rows, n)), dtype)
    return x, w, b, g


class Reference:
    """The formulas in 64 bits, and the bounds of a kernel's error."""

    def __init__(self, x, w, b, g, name, eps=EPS):
        x, w, b, g = _f64(x), _f64(w), _f64(b), _f64(g)
        rows, n = x.shape
        w = np.ones(n) if w is None else w
        b = np.zeros(n) if b is None else b
        u = 2.0 ** -53 if name == "f64" else 2.0 ** -24
        out = OUT_U[name]
        # depth of the sums: a lane's share of a row, then the lanes; over rows likewise
        s = 80 + n / 1024
        srow = 80 + rows / 16
        mean = x.mean(-1, keepdims=True)
        rstd = 1 / np.sqrt(((x - mean) ** 2).mean(-1, keepdims=True) + eps)
        h = (x - mean) * rstd
        dh = (1 + np.abs(h)) * (s * u * np.abs(x).max(-1, keepdims=True) * rstd + (s + 4) * u)
        self.y = h * w + b
        self.dy = np.abs(w) * dh + 3 * u * (np.abs(h * w) + np.abs(b)) + 1.01 * out * np.abs(self.y) + 1e-7 * (name == "f16")
        self.mean, self.rstd = mean[:, 0], rstd[:, 0]
        rel_rstd = 2 * (s * u * np.abs(x).max(-1, keepdims=True) * rstd + (s + 4) * u)
        v = g * w
        c1, c2 = v.mean(-1, keepdims=True), (v * h).mean(-1, keepdims=True)
        self.gx = rstd * (v - c1 - h * c2)
        e1 = (s + 2) * u * np.abs(v).mean(-1, keepdims=True)
        e2 = (s + 4) * u * np.abs(v * h).mean(-1, keepdims=True) + (np.abs(v) * dh).mean(-1, keepdims=True)
        self.dgx = (rstd * (4 * u * (np.abs(v) + np.abs(c1) + np.abs(h * c2)) + e1 + np.abs(h) * e2 + np.abs(c2) * dh)
                    + np.abs(self.gx) * (rel_rstd + 1.01 * out) + 1e-7 * (name == "f16"))
        self.gw, self.gb = (g * h).sum(0), g.sum(0)
        self.dgw = (np.abs(g) * dh).sum(0) + (srow + 3) * u * np.abs(g * h).sum(0)
        self.dgb = (srow + 3) * u * np.abs(g).sum(0)
        self.rel_rstd = rel_rstd[:, 0]
        self.dmean = s * u * np.abs(x).max(-1)


def near(got, want, bound, what):
    got = _f64(got).reshape(np.shape(want))
    assert np.isfinite(got).all(), what
    off = np.abs(got - want) - bound
    assert (off <= 0).all(), f"{what}: {np.max(off):.3e} over the bound at {np.unravel_index(np.argmax(off), off.shape)}"


def check_case(x, w, b, g, name, wname, eps=EPS):
    ref = Reference(x, w, b, g, name, eps)
    y, mean, rstd = Q.layer_norm_forward(x, w, b, eps)
    near(y, ref.y, ref.dy, "y")
    near(mean, ref.mean, ref.dmean, "mean")
    near(rstd, ref.rstd, ref.rstd * ref.rel_rstd, "rstd")
    gx, gw, gb = Q.layer_norm_backward(g, x, mean, rstd, w, weight_dtype=TYPES[wname])
    near(gx, ref.gx, ref.dgx, "grad_x")
    near(gw, ref.gw, ref.dgw + 1.01 * OUT_U[wname] * np.abs(ref.gw) + 1e-7 * (wname == "f16"), "grad_weight")
    near(gb, ref.gb, ref.dgb + 1.01 * OUT_U[wname] * np.abs(ref.gb) + 1e-7 * (wname == "f16"), "grad_bias")


# every length class of a row: groups of 16 lanes, wavefronts, workgroups, and
# past the registers of a workgroup; their ends, one element on either side
SHAPES = [(1, 1), (7, 1), (3, 2), (1, 10), (256, 10), (33, 16), (70, 63), (5, 64), (9, 65), (4, 127), (6, 129),
          (1037, 257), (3, 1000), (2, 1025), (5, 2047), (3, 4097), (2, 8191), (2, 16385), (1, 33000), (2, 70001)]


@gpu
@pytest.mark.parametrize("name,wname", [("f32", "f32"), ("f64", "f64"), ("bf16", "bf16"), ("bf16", "f32"),
                                        ("f16", "f16"), ("f16", "f32")])
@pytest.mark.parametrize("rows,n", SHAPES)
def test_values(need_gpu, rows, n, name, wname):
    x, w, b, g = make(rows, n, TYPES[name], TYPES[wname], seed=rows * 100003 + n)
    check_case(x, w, b, g, name, wname)


@gpu
@pytest.mark.parametrize("rows,n,name", [(4100, 33, "f32"), (20000, 7, "f64"), (5000, 520, "bf16"), (70000, 4, "f16")])
def test_many_rows(need_gpu, rows, n, name):
    x, w, b, g = make(rows, n, TYPES[name], TYPES[name], seed=n)
    check_case(x, w, b, g, name, name)


@gpu
@pytest.mark.parametrize("weight,bias", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("n", [12, 900, 5000, 66000])
def test_without_weight_or_bias(need_gpu, n, weight, bias):
    x, w, b, g = make(6, n, torch.float32, torch.float32, seed=n, weight=weight, bias=bias)
    check_case(x, w, b, g, "f32", "f32")


@gpu
@pytest.mark.parametrize("n", [10, 515, 3001])
def test_large_offset_keeps_the_variance(need_gpu, n):
    """Features 1000 times further from zero than from each other."""
    x, w, b, g = make(20, n, torch.float32, torch.float32, seed=n, offset=0.0)
    check_case(x + 1000, w, b, g, "f32", "f32")


@gpu
@pytest.mark.parametrize("name", ["f32", "bf16", "f64"])
@pytest.mark.parametrize("n,pad,shift", [(10, 1, 0), (64, 3, 1), (1001, 7, 5), (4099, 2, 3)])
def test_strides_and_alignment(need_gpu, name, n, pad, shift):
    """Columns of a wider array, starting at any element."""
    x, w, b, g = make(37, n, TYPES[name], TYPES[name], seed=n)
    wide = torch.full((37, n + pad + shift), float("nan"), dtype=x.dtype, device="cuda")
    wide[:, shift:shift + n] = x
    grad = torch.full((37, n + 2 * shift + 1), float("nan"), dtype=x.dtype, device="cuda")
    grad[:, shift:shift + n] = g
    xv, gv = wide[:, shift:shift + n], grad[:, shift:shift + n]
    wv = torch.cat([w[:1], w])[1:]  # one element past an aligned address
    assert not xv.is_contiguous()
    check_case(xv, wv, b, gv, name, name)


@gpu
def test_orders_of_axes(need_gpu):
    """Leading axes that do not collapse, a transposed matrix, repeated rows."""
    x, w, b, g = make(24, 40, torch.float32, torch.float32, seed=3)
    want = Q.layer_norm(x, w, b)
    assert torch.equal(Q.layer_norm(x.view(2, 3, 4, 40).transpose(0, 2), w, b), want.view(2, 3, 4, 40).transpose(0, 2))
    t = x.t().contiguous().t()
    assert torch.equal(Q.layer_norm(t, w, b), want)
    one = x[:1].expand(24, 40)
    assert torch.equal(Q.layer_norm(one, w, b), want[:1].expand(24, 40))
    assert torch.equal(Q.layer_norm(x[0], w, b), want[0])
    wide = torch.full((24, 80), float("nan"), device="cuda")
    wide[:, ::2] = x
    assert torch.equal(Q.layer_norm(wide[:, ::2], w, b), want) and torch.equal(Q.layer_norm(wide[3, ::2], w, b), want[3])
    cube = torch.full((2, 12, 41), float("nan"), device="cuda")
    cube[..., :40] = x.view(2, 12, 40)
    assert torch.equal(Q.layer_norm(cube[..., :40], w, b).view(24, 40), want)
    column = x[:, :1]
    assert torch.equal(Q.layer_norm(column, w[:1], b[:1]), Q.layer_norm(column.contiguous(), w[:1], b[:1]))
    y, mean, rstd = Q.layer_norm_forward(x, w, b)
    a = Q.layer_norm_backward(g[:1].expand(24, 40), x, mean, rstd, w)
    c = Q.layer_norm_backward(g[:1].repeat(24, 1), x, mean, rstd, w)
    assert all(torch.equal(p, q) for p, q in zip(a, c))


@gpu
def test_no_rows(need_gpu):
    x = torch.empty((0, 12), device="cuda", requires_grad=True)
    w, b = torch.ones(12, device="cuda", requires_grad=True), torch.zeros(12, device="cuda", requires_grad=True)
    y = Q.layer_norm(x, w, b)
    assert y.shape == (0, 12)
    y.sum().backward()
    assert x.grad.shape == (0, 12) and not w.grad.any() and not b.grad.any()


@gpu
@pytest.mark.parametrize("n", [10, 300, 5000, 66000])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_bad_value_stays_in_its_row(need_gpu, n, bad):
    x, w, b, g = make(5, n, torch.float32, torch.float32, seed=n)
    want, m, r = Q.layer_norm_forward(x, w, b)
    gx = Q.layer_norm_backward(g, x, m, r, w)[0]
    x[2, n // 2] = bad
    y, m, r = Q.layer_norm_forward(x, w, b)
    hx = Q.layer_norm_backward(g, x, m, r, w)[0]
    keep = [0, 1, 3, 4]
    assert torch.isnan(y[2]).all() and torch.isnan(hx[2]).all()
    assert torch.equal(y[keep], want[keep]) and torch.equal(hx[keep], gx[keep])


@gpu
def test_constant_rows(need_gpu):
    """No variance: h is 0, y the bias, and dx what is left of g w without its mean."""
    x, w, b, g = make(4, 96, torch.float32, torch.float32, seed=1)
    x[:] = torch.tensor([[0.0], [3.0], [-0.25], [1e6]], device="cuda")
    y, m, r = Q.layer_norm_forward(x, w, b)
    assert torch.equal(y, b.expand(4, 96))
    gx, gw, gb = Q.layer_norm_backward(g, x, m, r, w)
    v = (g * w).double()
    want = (v - v.mean(-1, keepdim=True)) / np.sqrt(EPS)
    assert (gx.double() - want).abs().max().item() <= 200 * 2.0 ** -24 * v.abs().max().item() / np.sqrt(EPS)
    assert not gw.any()


@gpu
@pytest.mark.parametrize("rows,n", [(3, 5), (4, 130), (2, 1030)])
def test_gradients_against_differences(need_gpu, rows, n):
    """d/dt of sum(g y(x + t dx, w + t dw, b + t db)) at t = 0 by central
    differences in float64, against the gradients; the step's error is
    h^2 / 6 of a third derivative of order 1 each term, plus rounding over h."""
    x, w, b, g = make(rows, n, torch.float64, torch.float64, seed=n)
    r = np.random.default_rng(n + 1)
    dx, dw, db = (torch.from_numpy(r.normal(size=s)).cuda() for s in ((rows, n), n, n))
    y, m, s = Q.layer_norm_forward(x, w, b)
    gx, gw, gb = Q.layer_norm_backward(g, x, m, s, w)
    h = 1e-4
    up = (g * Q.layer_norm(x + h * dx, w + h * dw, b + h * db)).sum()
    lo = (g * Q.layer_norm(x - h * dx, w - h * dw, b - h * db)).sum()
    got = ((gx * dx).sum() + (gw * dw).sum() + (gb * db).sum()).item()
    size = (g.abs() * (1 + y.abs())).sum().item()
    assert abs((up - lo).item() / (2 * h) - got) <= size * (100 * h * h + 1e-13 / h)


@gpu
def test_autograd_and_module(need_gpu):
    x, w, b, g = make(12, 48, torch.float32, torch.float32, seed=8)
    layer = Q.LayerNorm(48)
    with torch.no_grad():
        layer.weight.copy_(w)
        layer.bias.copy_(b)
    x.requires_grad_()
    y = layer(x.view(3, 4, 48))
    y.backward(g.view(3, 4, 48))
    z, m, r = Q.layer_norm_forward(x.detach(), w, b)
    gx, gw, gb = Q.layer_norm_backward(g, x.detach(), m, r, w)
    assert torch.equal(y.view(12, 48), z) and torch.equal(x.grad, gx)
    assert torch.equal(layer.weight.grad, gw) and torch.equal(layer.bias.grad, gb)
    plain = Q.LayerNorm(48, bias=False)
    assert plain.bias is None and torch.equal(plain(x), Q.layer_norm(x, plain.weight))
    only = Q.layer_norm_backward(g, x.detach(), m, r, w, want_x=False, want_bias=False)
    assert only[0] is None and only[2] is None and torch.equal(only[1], gw)
    with torch.no_grad():
        assert torch.equal(layer(x), z)


@gpu
def test_python_refuses(need_gpu):
    x, w, b, g = make(4, 8, torch.float32, torch.float32, seed=1)
    y, m, r = Q.layer_norm_forward(x, w, b)
    for bad in (w[:7], w.cpu(), torch.ones(16, device="cuda")[::2]):
        with pytest.raises(ValueError):
            Q.layer_norm(x, bad, b)
    with pytest.raises(ValueError):
        Q.layer_norm(x, w, b.double())
    with pytest.raises(Q.QLError):
        Q.layer_norm(x, w.double(), b.double())
    with pytest.raises(Q.QLError):
        Q.layer_norm(x, w, b, eps=-1.0)
    with pytest.raises(ValueError):
        Q.layer_norm_backward(g[:3], x, m, r, w)
    with pytest.raises(ValueError):
        Q.layer_norm_backward(g, x, m[:3], r, w)
    with pytest.raises(ValueError):
        Q.layer_norm_backward(g, x, m.double(), r, w)


@gpu
def test_other_stream_and_graph(need_gpu):
    """The current stream, and a captured graph replayed with new inputs between
    eager work."""
    x, w, b, g = make(300, 200, torch.bfloat16, torch.float32, seed=5)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())

    def step():
        y, m, r = Q.layer_norm_forward(x, w, b)
        return (y, *Q.layer_norm_backward(g, x, m, r, w))

    want = step()
    with torch.cuda.stream(stream):
        got = step()
    torch.cuda.current_stream().wait_stream(stream)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in range(3):
        x.copy_(make(300, 200, torch.bfloat16, torch.float32, seed=50 + seed)[0])
        want = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, want))


@gpu
def test_same_bits_again(need_gpu):
    x, w, b, g = make(3000, 321, torch.float32, torch.float32, seed=5)
    y, m, r = Q.layer_norm_forward(x, w, b)
    first = Q.layer_norm_backward(g, x, m, r, w)
    for _ in range(3):
        again = Q.layer_norm_backward(g, x, m, r, w)
        assert all(torch.equal(p, q) for p, q in zip(first, again))


@gpu
def test_offsets_past_32_bits(need_gpu):
    """An array of more than 2^32 elements' bytes, and a view whose rows lie further apart."""
    rows, n = 66000, 33000
    x = torch.zeros((rows, n), dtype=torch.bfloat16, device="cuda")
    g = torch.zeros((rows, n), dtype=torch.bfloat16, device="cuda")
    assert x.numel() > 1 << 31
    at = [0, 1, rows // 2, rows - 2, rows - 1]
    part, w, b, gpart = make(len(at), n, torch.bfloat16, torch.float32, seed=9)
    x[at], g[at] = part, gpart
    y, m, r = Q.layer_norm_forward(x, w, b)
    gx, gw, gb = Q.layer_norm_backward(g, x, m, r, w)
    ref = Reference(part, w, b, gpart, "bf16")
    near(y[at], ref.y, ref.dy, "y")
    near(gx[at], ref.gx, ref.dgx, "grad_x")
    near(gw, ref.gw, ref.dgw + 2.0 ** -24 * np.abs(ref.gw), "grad_weight")
    near(gb, ref.gb, ref.dgb + 2.0 ** -24 * np.abs(ref.gb), "grad_bias")
