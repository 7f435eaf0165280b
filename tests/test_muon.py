"""Orthogonalised updates and the optimiser's step: refusals of the C entries
(CPU), and values against the formulas in 64 bits (needs an MI355X).

Tolerances come from a model of the kernels' rounding, run on the CPU on the
same inputs: the formulas in float64 with X, A and B rounded after every product
as the kernels hold them (fp32 for small matrices, 22 bits in two fp16 parts, 11
bits in one). Its distance from the exact values, element by element at its
largest and in the Frobenius norm, is what a kernel's should be: three times
that, plus 2^-24 sqrt(terms) for sums in fp32 and the output's own rounding, is
what it may be.
"""

from __future__ import annotations

import array
import ctypes
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2301_03251_amd as Q  # noqa: E402

F32, F64, BF16, F16 = 0, 1, 2, 3
TYPES = {"f32": torch.float32, "f64": torch.float64, "bf16": torch.bfloat16, "f16": torch.float16}
OUT_U = {"f32": 2.0 ** -24, "f64": 2.0 ** -53, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
COEF = (3.4445, -4.7750, 2.0315)
EPS = 1e-7
FAKE = 0x1000


# ---------------------------------------------------------------------------
# refusals: nothing is launched, so the addresses are never read

@pytest.fixture(scope="module")
def lib():
    return Q.load()


class Ortho(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("a", "b", "c", "eps")] + [("steps", ctypes.c_int32)]


class Step(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("lr", "momentum", "weight_decay")] + [("nesterov", ctypes.c_int32)]


def entry(rows=200, cols=300, batch=1, grad=FAKE, gs=None, momentum=FAKE, ms=None, out=FAKE, os=None):
    s = [rows * cols, cols, 1]
    return [rows, cols, batch, grad, *(gs or s), momentum, *(ms or s), out, *(os or s)]


def _call(lib, entries, muon=False, type_=F32, count=None, ortho=None, step=None, ws=FAKE, ws_bytes=1 << 40):
    words = array.array("q", [v for e in entries for v in e])
    mats = words.buffer_info()[0] if words else None
    o = ctypes.byref(ortho) if ortho is not None else None
    n = len(entries) if count is None else count
    if muon:
        s = ctypes.byref(step) if step is not None else None
        return lib.ql_muon_step(type_, mats, n, s, o, ws, ws_bytes, None)
    return lib.ql_orthogonalize(type_, mats, n, o, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(entries=[entry()], type_=4), -1), (dict(entries=[entry()], type_=-1), -1),
    (dict(entries=[], count=-1), -1), (dict(entries=[], count=2), -1),
    (dict(entries=[entry(rows=0)]), -1), (dict(entries=[entry(cols=-1)]), -1), (dict(entries=[entry(rows=65537)]), -1),
    (dict(entries=[entry(batch=-1)]), -1), (dict(entries=[entry(batch=1 << 31)]), -1),
    (dict(entries=[entry(batch=1 << 22)] * 3), -1),
    (dict(entries=[entry(grad=0)]), -1), (dict(entries=[entry(out=0)]), -1),
    (dict(entries=[entry(grad=FAKE + 2)]), -1), (dict(entries=[entry(out=FAKE + 1)]), -1),
    (dict(entries=[entry(gs=[0, -300, 1])]), -1), (dict(entries=[entry(os=[0, 0, 1])]), -1),
    (dict(entries=[entry(os=[0, 1, 0])]), -1), (dict(entries=[entry(batch=2, os=[0, 300, 1])]), -1),
    (dict(entries=[entry(gs=[0, 1 << 60, 1])]), -1),
    (dict(entries=[entry()], ortho=Ortho(*COEF, -1.0, 5)), -1),
    (dict(entries=[entry()], ortho=Ortho(*COEF, float("nan"), 5)), -1),
    (dict(entries=[entry()], ortho=Ortho(*COEF, EPS, 0)), -1), (dict(entries=[entry()], ortho=Ortho(*COEF, EPS, 65)), -1),
    (dict(entries=[entry()], ortho=Ortho(float("nan"), 0, 0, EPS, 5)), -1),
    (dict(entries=[entry()], ortho=Ortho(9.0, 0, 0, EPS, 5)), -1),
    (dict(entries=[entry()], ortho=Ortho(3.4445, -4.7750, 20.0, EPS, 5)), -1),
    (dict(entries=[entry()], ws=None), -1), (dict(entries=[entry()], ws=FAKE + 8), -1),
    (dict(entries=[entry()], ws_bytes=100), -2),
    (dict(entries=[entry(momentum=0)], muon=True), -1), (dict(entries=[entry(momentum=FAKE + 2)], muon=True), -1),
    (dict(entries=[entry(ms=[0, 0, 1])], muon=True), -1),
    (dict(entries=[entry()], muon=True, step=Step(float("inf"), 0.9, 0, 1)), -1),
    (dict(entries=[entry()], muon=True, step=Step(0.1, float("nan"), 0, 1)), -1),
    (dict(entries=[entry()], muon=True, ws_bytes=100), -2),
])
def test_refuses(lib, kw, code):
    assert _call(lib, **kw) == code
    assert lib.ql_last_error()


def test_nothing_to_do(lib):
    assert _call(lib, []) == 0
    assert _call(lib, [entry(batch=0, grad=0, out=0)]) == 0
    assert _call(lib, [entry(batch=0)], muon=True) == 0


def test_workspace_bytes(lib):
    out = ctypes.c_size_t()

    def size(t, *e):
        words = array.array("q", [v for x in e for v in x])
        return lib.ql_orthogonalize_workspace_bytes(t, words.buffer_info()[0], len(e), ctypes.byref(out)), out.value

    assert lib.ql_orthogonalize_workspace_bytes(F32, None, 1, ctypes.byref(out)) == -1
    assert lib.ql_orthogonalize_workspace_bytes(F32, None, 0, None) == -1
    assert size(F32, entry(20, 72)) == (0, 0)  # one workgroup's LDS holds it
    for t, unit in ((F32, 4), (F16, 4), (BF16, 2), (F64, 8)):
        rc, one = size(t, entry(200, 300))
        assert rc == 0 and one >= unit * (3 * 256 * 320 + 2 * 256 * 256)
        assert size(t, entry(300, 200)) == (0, one)
        assert size(t, entry(200, 300, batch=3)) == (0, 3 * one)
        assert size(t, entry(200, 300), entry(200, 300)) == (0, 2 * one)


def test_python_refuses_on_the_cpu():
    g = torch.zeros(4, 4)
    with pytest.raises(ValueError):
        Q.orthogonalize(g)
    with pytest.raises(ValueError):
        Q.muon_step([g], [g], [g])
    with pytest.raises(ValueError):
        Q.muon_step([g], [g], [])
    with pytest.raises(ValueError):
        Q.Muon([torch.nn.Parameter(torch.zeros(8))])
    assert Q.muon_step([], [], []) is None


# ---------------------------------------------------------------------------
# values

gpu = pytest.mark.gpu


@pytest.fixture(scope="module")
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    Q.load()


def _f64(t):
    return t.detach().cpu().double().numpy()


def steps_of(u, steps, coef, eps, hold=lambda v, size: v):
    """The formulas; hold(v, size) is v as it is kept between products."""
    a, b, c = coef
    turned = u.shape[0] > u.shape[1]
    u = u.T if turned else u
    x = hold(u / (np.sqrt((u * u).sum()) + eps), 1.0)
    for _ in range(steps):
        g = hold(x @ x.T, 1.0)
        x = hold(a * x + hold(b * g + c * (g @ g), 4.0) @ x, 1.0)
    return x.T if turned else x


def _fp16_parts(parts):
    def hold(v, size):
        s = 2.0 ** 14 / size
        hi = (v * s).astype(np.float16).astype(np.float64)
        if parts == 2:
            hi += (v * s - hi).astype(np.float16).astype(np.float64)
        return hi / s
    return hold


def small(m, n):
    return min(m, n) <= 64 and max(m, n) <= 400


def exact_and_bounds(u, name, steps=5, coef=COEF, eps=EPS):
    """(exact O, bound of a norm of the difference, bound of an element's)."""
    want = steps_of(u, steps, coef, eps)
    if name == "f64":
        hold = lambda v, size: v * (1 + 2.0 ** -52 * np.cos(np.arange(v.size)).reshape(v.shape))  # noqa: E731
    elif name == "bf16" and not small(*u.shape):
        hold = _fp16_parts(1)
    else:
        hold = _fp16_parts(2)  # of a small matrix too, which is held in fp32 where it runs by itself
    off = steps_of(u, steps, coef, eps, hold) - want
    terms = max(u.shape)
    unit = (2.0 ** -53 if name == "f64" else 2.0 ** -24) * math.sqrt(terms) * 4
    norm, size = np.linalg.norm(want), np.abs(want).max() if want.size else 0.0
    out = 1.01 * OUT_U[name]
    tiny = 3e-8 if name == "f16" else 0.0
    grow = max(1.0, 4.0 ** steps / 64)  # what a sum's rounding grows by in the steps behind it
    return (want, 3 * np.linalg.norm(off) + (out + unit * grow) * norm + tiny * math.sqrt(want.size),
            3 * np.abs(off).max() + (out + unit * grow) * size + tiny)


def near(got, u, name, what="", **kw):
    want, norm, each = exact_and_bounds(u, name, **kw)
    off = got - want
    assert np.isfinite(got).all(), what
    assert np.linalg.norm(off) <= norm, f"{what}: norm {np.linalg.norm(off):.3e} > {norm:.3e}"
    assert np.abs(off).max() <= each, f"{what}: largest {np.abs(off).max():.3e} > {each:.3e}"


def gradient(shape, dtype, seed, decay=0.5):
    r = np.random.default_rng(seed)
    g = r.normal(size=shape)
    for axis in (-1, -2):
        n = shape[axis]
        s = r.permutation(np.arange(1, n + 1) ** -decay)
        g = g * (s if axis == -1 else s[:, None])
    return torch.from_numpy(0.05 * g).to("cuda", dtype)


SHAPES = [(1, 1), (1, 7), (5, 1), (2, 2), (6, 30), (8, 32), (16, 16), (17, 15), (20, 72), (64, 64), (64, 256), (33, 410),
          (63, 500), (3, 3000), (65, 65), (70, 64), (100, 130), (128, 128), (129, 200), (257, 70), (500, 300)]


@gpu
@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_orthogonalize(need_gpu, rows, cols, name):
    g = gradient((rows, cols), TYPES[name], seed=rows * 1000 + cols)
    near(_f64(Q.orthogonalize(g)), _f64(g), name, f"{rows}x{cols}")


@gpu
@pytest.mark.parametrize("name,rows,cols", [("f32", 1111, 1500), ("bf16", 2050, 1030), ("f16", 1200, 1200), ("f64", 600, 900),
                                            ("bf16", 64, 9000), ("f32", 9000, 130)])
def test_large(need_gpu, name, rows, cols):
    g = gradient((rows, cols), TYPES[name], seed=rows)
    near(_f64(Q.orthogonalize(g)), _f64(g), name, f"{rows}x{cols}")


def _fp16_parts_torch(parts):
    def hold(v, size):
        s = 2.0 ** 14 / size
        hi = (v * s).half().double()
        if parts == 2:
            hi = hi + (v * s - hi).half().double()
        return hi / s
    return hold


def steps_on_gpu(u, hold=lambda v, size: v):
    """steps_of with the default options, in torch's float64."""
    a, b, c = COEF
    turned = u.shape[0] > u.shape[1]
    u = u.T.contiguous() if turned else u
    x = hold(u / (u.square().sum().sqrt() + EPS), 1.0)
    for _ in range(5):
        g = hold(x @ x.T.contiguous(), 1.0)
        x = hold(a * x + hold(b * g + c * (g @ g), 4.0) @ x, 1.0)
    return x.T if turned else x


# each tile size, a long K that is split, and matrices beside smaller ones
@gpu
@pytest.mark.parametrize("name,rows,cols", [("bf16", 4096, 4096), ("bf16", 2900, 3500), ("f32", 2048, 8192), ("f32", 3500, 2900),
                                            ("f16", 1500, 4100), ("f32", 64, 9000), ("bf16", 20, 6000), ("f32", 300, 8200),
                                            ("f64", 70, 5000)])
def test_tile_sizes_and_splits(need_gpu, name, rows, cols):
    """The model's bounds as above, both computed on the GPU in torch's float64."""
    g = gradient((rows, cols), TYPES[name], seed=rows + cols)
    u = g.double()
    want = steps_on_gpu(u)
    unit, out = (2.0 ** -53 if name == "f64" else 2.0 ** -24) * math.sqrt(cols) * 4 * 16, 1.01 * OUT_U[name]
    off = steps_on_gpu(u, _fp16_parts_torch(1 if name == "bf16" else 2)) - want if name != "f64" else 0 * want
    norm = 3 * off.norm().item() + (out + unit) * want.norm().item() + 3e-8 * math.sqrt(want.numel()) * (name == "f16")
    each = 3 * off.abs().max().item() + (out + unit) * want.abs().max().item() + 3e-8 * (name == "f16")
    for v in (g, g.t().contiguous().t()):
        got = Q.orthogonalize(v).double() - want
        assert got.norm().item() <= norm and got.abs().max().item() <= each
    p, m = torch.zeros_like(g), torch.zeros_like(g, dtype=torch.float64 if name == "f64" else torch.float32)
    Q.muon_step([p], [g], [m], lr=1.0, momentum=0.0)
    got = p.double() + max(1.0, rows / cols) ** 0.5 * want
    assert got.norm().item() <= max(1.0, rows / cols) ** 0.5 * norm and got.abs().max().item() <= max(1.0, rows / cols) ** 0.5 * each


@gpu
@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(3, 10, 20), (2, 3, 40, 30), (5, 100, 140), (40, 70, 66)])
def test_batches(need_gpu, shape, name):
    g = gradient(shape, TYPES[name], seed=shape[-1])
    got = Q.orthogonalize(g)
    assert got.shape == g.shape
    for o, q in zip(got.reshape(-1, *shape[-2:]), g.reshape(-1, *shape[-2:])):
        near(_f64(o), _f64(q), name, str(shape))


@gpu
@pytest.mark.parametrize("rows,cols", [(12, 30), (30, 12), (90, 140), (140, 90)])
@pytest.mark.parametrize("name", ["f32", "f64", "bf16"])
def test_strides(need_gpu, rows, cols, name):
    """Transposed, spaced and shifted arrays, in and out; and in place."""
    g = gradient((rows, cols), TYPES[name], seed=rows)
    want = Q.orthogonalize(g)
    views = [g.t().contiguous().t()]
    wide = torch.full((rows, 2 * cols + 3), float("nan"), dtype=g.dtype, device="cuda")
    wide[:, 3::2] = g
    views.append(wide[:, 3::2])
    tall = torch.full((2 * rows + 1, cols + 1), float("nan"), dtype=g.dtype, device="cuda")
    tall[1::2, 1:] = g
    views.append(tall[1::2, 1:])
    for v in views:
        assert torch.equal(Q.orthogonalize(v), want)
        out = torch.empty_strided(v.shape, v.stride(), dtype=v.dtype, device="cuda").fill_(0)
        assert torch.equal(Q.orthogonalize(g, out=out), want)
    same = g.clone()
    assert Q.orthogonalize(same, out=same) is same and torch.equal(same, want)


@gpu
@pytest.mark.parametrize("rows,cols", [(9, 20), (150, 100)])
@pytest.mark.parametrize("name", list(TYPES))
def test_zeros_infinities_and_nan(need_gpu, rows, cols, name):
    g = gradient((rows, cols), TYPES[name], seed=1)
    assert not Q.orthogonalize(torch.zeros_like(g)).any()
    for bad in (float("inf"), -float("inf"), float("nan")):
        h = g.clone()
        h[rows - 1, 3] = bad
        assert torch.isnan(Q.orthogonalize(h)).all()
    pair = torch.stack([h, g])  # the matrix beside it keeps its values
    assert torch.equal(Q.orthogonalize(pair)[1], Q.orthogonalize(torch.stack([g, g]))[1])


@gpu
@pytest.mark.parametrize("rows,cols", [(12, 30), (100, 130)])
@pytest.mark.parametrize("scale", [1e-18, 1e18])
def test_scale_of_the_gradient(need_gpu, rows, cols, scale):
    """Squares past the range of fp32; the result is the same but for the
    rounding of the inputs (a power of two: none) and eps."""
    g = gradient((rows, cols), torch.float32, seed=2) * 2.0 ** round(math.log2(scale))
    near(_f64(Q.orthogonalize(g, eps=0.0)), _f64(g), "f32", eps=0.0)
    near(_f64(Q.orthogonalize(g)), _f64(g), "f32")


@gpu
@pytest.mark.parametrize("steps,coef", [(1, COEF), (8, COEF), (10, (1.5, -0.5, 0.0)), (3, (2.0, -1.5, 0.5)), (2, (6.0, -8.0, 3.0))])
@pytest.mark.parametrize("rows,cols", [(24, 40), (130, 200)])
def test_steps_and_coefficients(need_gpu, rows, cols, steps, coef):
    g = gradient((rows, cols), torch.float32, seed=4, decay=0.1)
    near(_f64(Q.orthogonalize(g, steps, coef)), _f64(g), "f32", steps=steps, coef=coef)


@gpu
@pytest.mark.parametrize("rows,cols", [(40, 60), (200, 90)])
def test_cubic_steps_give_the_polar_factor(need_gpu, rows, cols):
    """1.5 s - 0.5 s^3 takes every singular value to 1: O = U V^T."""
    g = gradient((rows, cols), torch.float64, seed=6, decay=0.0)
    u, _, vt = np.linalg.svd(_f64(g), full_matrices=False)
    got = _f64(Q.orthogonalize(g, 40, (1.5, -0.5, 0.0)))
    assert np.abs(got - u @ vt).max() <= 1e-11


def check_step(shapes, name, lr, mu, nesterov, decay, seed, rounds=2):
    dtype, wide = TYPES[name], torch.float64 if name == "f64" else torch.float32
    p = [gradient(s, dtype, seed + k, 0.0) * 10 for k, s in enumerate(shapes)]
    m = [gradient(s, wide, seed + 50 + k) for k, s in enumerate(shapes)]
    for turn in range(rounds):
        g = [gradient(s, dtype, seed + 100 + 10 * turn + k) for k, s in enumerate(shapes)]
        p0, m0 = [_f64(t) for t in p], [_f64(t) for t in m]
        Q.muon_step(p, g, m, lr=lr, momentum=mu, nesterov=nesterov, weight_decay=decay)
        for k, (rows, cols) in enumerate(shapes):
            gk, unit = _f64(g[k]), 2.0 ** -53 if name == "f64" else 2.0 ** -24
            want_m = mu * m0[k] + gk
            assert (np.abs(_f64(m[k]) - want_m) <= 3 * unit * (np.abs(mu * m0[k]) + np.abs(gk))).all()
            now = _f64(m[k])
            u = gk + mu * now if nesterov else now
            o, norm, each = exact_and_bounds(u, name)
            step = lr * math.sqrt(max(1.0, rows / cols))
            want = (1 - lr * decay) * p0[k] - step * o
            out = 1.01 * OUT_U[name]
            off = _f64(p[k]) - want
            assert np.abs(off).max() <= step * each + (out + 4 * unit) * np.abs(want).max() + 1e-7 * (name == "f16")
            assert np.linalg.norm(off) <= step * norm + (out + 4 * unit) * np.linalg.norm(want) + 1e-7 * (name == "f16") * math.sqrt(off.size)


@gpu
@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("shapes", [[(20, 72)], [(6, 30), (64, 256), (10, 3)], [(100, 300)],
                                    [(6, 30), (256, 64), (130, 70), (1, 9), (200, 200)]])
def test_muon_step(need_gpu, shapes, name):
    check_step(shapes, name, 0.03, 0.9, True, 0.1, 7)


@gpu
@pytest.mark.parametrize("lr,mu,nesterov,decay", [(0.02, 0.95, False, 0.0), (0.5, 0.0, True, 0.5), (0.0, 0.9, True, 0.1)])
def test_muon_options(need_gpu, lr, mu, nesterov, decay):
    check_step([(12, 20), (30, 9)], "f32", lr, mu, nesterov, decay, 70)
    check_step([(120, 90)], "f32", lr, mu, nesterov, decay, 71)


@gpu
def test_more_matrices_than_a_launch_takes(need_gpu):
    shapes = [(5 + k % 7, 9 + k) for k in range(60)]
    check_step(shapes, "f32", 0.05, 0.9, True, 0.0, 300, rounds=1)
    check_step([*shapes, (70, 80)], "f32", 0.05, 0.9, True, 0.0, 300, rounds=1)


@gpu
def test_optimizer(need_gpu):
    """The module's steps are muon_step's, flat weights among them; state is kept."""
    torch.manual_seed(0)
    w = [torch.nn.Parameter(torch.randn(s, device="cuda")) for s in ((12, 30), (70, 90), (3, 5, 8))]
    flat = torch.nn.Parameter(torch.randn(6 * 30, device="cuda"))
    idle = torch.nn.Parameter(torch.randn(4, 4, device="cuda"))
    opt = Q.Muon([{"params": [*w, idle]}, {"params": [flat], "matrix": (6, 30)}], lr=0.1, weight_decay=0.2)
    p = [t.detach().clone() for t in (*w, flat.view(6, 30))]
    m = [torch.zeros_like(t) for t in p]
    for turn in range(3):
        g = [torch.randn_like(t) for t in p]
        for t, q in zip((*w, flat), g):
            t.grad = q.view(t.shape).clone()
        version = flat._version
        opt.step()
        assert flat._version > version
        Q.muon_step(p[:3], g[:3], m[:3], lr=0.1, weight_decay=0.2)
        Q.muon_step(p[3:], g[3:], m[3:], lr=0.1, weight_decay=0.2)
        assert all(torch.equal(a.view(b.shape), b) for a, b in zip((*w, flat), p))
    assert opt.step(lambda: 3.0) == 3.0


@gpu
def test_optimizer_state_is_saved_whole(need_gpu):
    """A bfloat16 weight's momentum is float32 after saving and loading too."""
    w = [torch.nn.Parameter(torch.randn(12, 20, device="cuda").bfloat16()) for _ in range(2)]
    w[1].data.copy_(w[0].data)
    a, b = Q.Muon([w[0]], lr=0.1), Q.Muon([w[1]], lr=0.1)
    for turn in range(3):
        g = torch.randn(12, 20, device="cuda").bfloat16()
        w[0].grad = g
        if turn == 2:
            b.load_state_dict(a.state_dict())
            w[1].data.copy_(w[0].data)
            w[1].grad = g.clone()
            b.step()
        a.step()
    assert b.state[w[1]]["momentum"].dtype == torch.float32
    assert torch.equal(w[0], w[1]) and torch.equal(a.state[w[0]]["momentum"], b.state[w[1]]["momentum"])


@gpu
def test_python_refuses(need_gpu):
    g = torch.randn(8, 12, device="cuda")
    m = torch.zeros_like(g)
    for bad in (g[0], g.to(torch.int32)):
        with pytest.raises(ValueError):
            Q.orthogonalize(bad)
    with pytest.raises(ValueError):
        Q.orthogonalize(g, out=torch.empty(12, 8, device="cuda"))
    for args in (([g], [g[:4]], [m]), ([g], [g.double()], [m]), ([g], [g], [m.double()]), ([g], [g], [m.cpu()]),
                 ([g, g.double()], [g, g.double()], [m, m.double()]), ([g[0]], [g[0]], [m[0]])):
        with pytest.raises(ValueError):
            Q.muon_step(*args)
    for kw in (dict(steps=0), dict(eps=-1.0), dict(coefficients=(9.0, 0.0, 0.0))):
        with pytest.raises(Q.QLError):
            Q.orthogonalize(g, **kw)
    with pytest.raises(Q.QLError):
        Q.muon_step([g], [g], [m], lr=float("nan"))
    with pytest.raises(Q.QLError):  # a weight whose rows are one row
        Q.muon_step([g[:1].expand(8, 12)], [g], [m])
    assert Q.orthogonalize(torch.empty(0, 4, 5, device="cuda")).shape == (0, 4, 5)
    assert not m.any()


@gpu
@pytest.mark.parametrize("rows,cols", [(20, 50), (180, 260)])
def test_other_stream_graph_and_same_bits(need_gpu, rows, cols):
    g = gradient((rows, cols), torch.float32, seed=1)
    want = Q.orthogonalize(g)
    assert all(torch.equal(Q.orthogonalize(g), want) for _ in range(3))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        got = Q.orthogonalize(g)
    torch.cuda.current_stream().wait_stream(stream)
    assert torch.equal(got, want)
    p, m = torch.randn_like(g), torch.zeros_like(g)
    q, n = p.clone(), m.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        Q.muon_step([p], [g], [m])
    for turn in range(3):
        g.copy_(gradient((rows, cols), torch.float32, seed=10 + turn))
        Q.muon_step([q], [g], [n])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(p, q) and torch.equal(m, n)


@gpu
@pytest.mark.parametrize("rows,cols", [(8, 16), (80, 100)])
def test_offsets_past_32_bits(need_gpu, rows, cols):
    """A batch whose matrices lie 2^30 elements apart."""
    far = torch.zeros((1 << 30) * 3 + 20000, dtype=torch.bfloat16, device="cuda")
    v = far.as_strided((4, rows, cols), (1 << 30, cols, 1))
    g = gradient((4, rows, cols), torch.bfloat16, seed=3)
    v.copy_(g)
    assert torch.equal(Q.orthogonalize(v), Q.orthogonalize(g))
