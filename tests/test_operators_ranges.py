"""The ends of the ranges that the operators' C entries take: rows of more
features and batches of more matrices than one launch's threads (2^32), and what
is refused before anything is launched."""

from __future__ import annotations

import array
import ctypes
import math

import pytest

torch = pytest.importorskip("torch")
import paper_2301_03251_amd as Q  # noqa: E402

F32, F64, BF16, F16 = 0, 1, 2, 3
gpu = pytest.mark.gpu


@pytest.fixture(scope="module")
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    Q.load()


def within(got, want, bound, what):
    off = (got.double() - want).abs_().sub_(bound)
    assert off.max().item() <= 0, f"{what}: {off.max().item():.3e} over the bound"


@gpu
@pytest.mark.parametrize("n", [(1 << 27) + 5])
def test_norm_of_very_long_rows(need_gpu, n):
    """Column sums of 2^28 columns, which take more threads than a launch has.
    The bounds are test_norm's, with the depth of a segment's sums (8 elements,
    then 256 lanes) and of the lane that joins 1/64 of the segments."""
    torch.manual_seed(0)
    x = (torch.randn(2, n, device="cuda") + 0.5).bfloat16()
    g = torch.randn(2, n, device="cuda").bfloat16()
    y, mean, rstd = Q.layer_norm_forward(x)
    gx, gw, gb = Q.layer_norm_backward(g, x, mean, rstd, weight_dtype=torch.float32)
    u, out, s = 2.0 ** -24, 1.01 * 2.0 ** -8, 80 + n / 2048 / 64
    assert gw.shape == gb.shape == (n,)
    sums = torch.zeros(2, n, dtype=torch.float64, device="cuda")
    slack = torch.zeros(n, dtype=torch.float64, device="cuda")
    size = torch.zeros(2, n, dtype=torch.float64, device="cuda")
    for row in range(2):
        xr, gr = x[row].double(), g[row].double()
        m = xr.mean()
        r = 1 / ((xr - m).square().mean() + 1e-5).sqrt()
        h = (xr - m) * r
        off = (s * u * xr.abs().max() * r + (s + 4) * u)
        dh = (1 + h.abs()) * off
        within(y[row], h, dh + out * h.abs(), "y")
        c1, c2 = gr.mean(), (gr * h).mean()
        want = r * (gr - c1 - h * c2)
        e1, e2 = (s + 2) * u * gr.abs().mean(), (s + 4) * u * (gr * h).abs().mean() + (gr.abs() * dh).mean()
        bound = r * (4 * u * (gr.abs() + c1.abs() + (h * c2).abs()) + e1 + h.abs() * e2 + c2.abs() * dh)
        within(gx[row], want, bound + want.abs() * (2 * off + out), "grad_x")
        sums[0] += gr * h
        sums[1] += gr
        slack += gr.abs() * dh
        size[0] += (gr * h).abs()
        size[1] += gr.abs()
    within(gw, sums[0], slack + 8 * u * size[0], "grad_weight")
    within(gb, sums[1], 8 * u * size[1], "grad_bias")


class Ortho(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("a", "b", "c", "eps")] + [("steps", ctypes.c_int32)]


class Step(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("lr", "momentum", "weight_decay")] + [("nesterov", ctypes.c_int32)]


FAKE = 0x1000


def orthogonalize(entries, type_=F32, ortho=None, ws=None, ws_bytes=0):
    words = array.array("q", [v for r, c, b in entries for v in (r, c, b, FAKE, r * c, c, 1, 0, 0, 0, 0, FAKE, r * c, c, 1)])
    return Q.load().ql_orthogonalize(type_, words.buffer_info()[0], len(entries),
                                     ctypes.byref(ortho) if ortho is not None else None, ws, ws_bytes, None)


@pytest.mark.parametrize("a,b,c", [(-200.0, 200.0, 1e-16), (30.0, -30.0, 1e-17), (-30.0, 30.0, -1e-17), (200.0, -200.0, 0.0)])
def test_growth_between_zero_and_one_is_seen(a, b, c):
    """a x + b x^3 is 0 at both ends of [0, 1], and past 64 or a few steps from it
    between them: the two roots of its slope may differ by 16 orders of magnitude."""
    reach = 1.0
    for _ in range(3):
        reach = max(abs(x * (a + x * x * (b + c * x * x))) for x in (reach * i / 1000 for i in range(1001)))
    assert reach > 64
    assert orthogonalize([(200, 300, 1)], ortho=Ortho(a, b, c, 1e-7, 4), ws=FAKE, ws_bytes=1 << 40) == -1


def workspace(entries, type_=F32):
    words = array.array("q", [v for r, c, b in entries for v in (r, c, b, *(0,) * 12)])
    out = ctypes.c_size_t()
    return Q.load().ql_orthogonalize_workspace_bytes(type_, words.buffer_info()[0], len(entries), ctypes.byref(out)), out.value


@pytest.mark.parametrize("type_", [F32, F64, BF16])
def test_matrices_of_a_call(type_):
    """2^32 threads in workgroups of 512, one for each 64x64: 2^23 of them are refused before anything runs."""
    most = (1 << 23) - 1
    assert workspace([(65, 65, most // 4)], type_)[0] == 0
    assert workspace([(65, 65, most // 4 + 1)], type_)[0] == -1
    assert workspace([(65, 65, 1), (3, 3, most - 4)], type_)[0] == 0
    assert workspace([(65, 65, 1), (3, 3, most - 3)], type_)[0] == -1
    assert orthogonalize([(65, 65, most // 4 + 1)], type_, ws=FAKE, ws_bytes=1 << 62) == -1
    # matrices that one workgroup holds go in as many launches as it takes
    assert workspace([(3, 3, 1 << 28)], type_) == (0, 0)


@gpu
@pytest.mark.parametrize("name,rows,cols,batch", [("float32", 2, 2, (1 << 23) + 5), ("float64", 1, 2, (1 << 23) + 5),
                                                  ("bfloat16", 33, 64, (1 << 22) + 5)])
def test_batches_of_more_threads_than_a_launch(need_gpu, name, rows, cols, batch):
    """As the same matrices in a smaller batch, bit by bit, past the first launch too."""
    torch.manual_seed(0)
    dtype = getattr(torch, name)
    few = torch.randn(7, rows, cols, device="cuda").to(dtype)
    want = Q.orthogonalize(few)
    out = torch.zeros(batch, rows, cols, dtype=dtype, device="cuda")
    if rows * cols < 10:
        g = few.repeat(batch // 7 + 1, 1, 1)[:batch]
        Q.orthogonalize(g, out=out)
        assert torch.equal(out, want.repeat(batch // 7 + 1, 1, 1)[:batch])
    else:  # one matrix throughout: 18 GB of results are enough
        Q.orthogonalize(few[:1].expand(batch, rows, cols), out=out)
        assert (out == want[:1]).all()


@gpu
def test_muon_steps_of_more_threads_than_a_launch(need_gpu):
    torch.manual_seed(1)
    batch = (1 << 22) + 9
    p = [torch.randn(s, device="cuda") for s in ((3, 2, 3), (batch, 2, 2), (5, 4, 4))]
    g, m = [torch.randn_like(t) for t in p], [torch.randn_like(t) for t in p]
    q, n = [t.clone() for t in p], [t.clone() for t in m]
    Q.muon_step(p, g, m)
    half = batch // 2
    for part in (slice(0, half), slice(half, None)):
        Q.muon_step([q[1][part]], [g[1][part]], [n[1][part]])
    Q.muon_step([q[0], q[2]], [g[0], g[2]], [n[0], n[2]])
    assert all(torch.equal(a, b) for a, b in zip(p + m, q + n))


def norm_near(rows, n, dtype, segment):
    """y, grad_x and the column sums of n features in segments, against 64 bits; the bounds as above."""
    torch.manual_seed(n)
    x = (torch.randn(rows, n, device="cuda") + 0.5).to(dtype)
    w = (1 + 0.2 * torch.randn(n, device="cuda")).to(dtype)
    g = torch.randn(rows, n, device="cuda").to(dtype)
    y, mean, rstd = Q.layer_norm_forward(x, w)
    gx, gw, gb = Q.layer_norm_backward(g, x, mean, rstd, w)
    u = 2.0 ** -53 if dtype == torch.float64 else 2.0 ** -24
    out = 1.01 * {torch.float64: 2.0 ** -53, torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}[dtype]
    s = 80 + n / segment / 64
    xd, gd, wd = x.double(), g.double(), w.double()
    m = xd.mean(1, keepdim=True)
    r = 1 / ((xd - m).square().mean(1, keepdim=True) + 1e-5).sqrt()
    h = (xd - m) * r
    off = s * u * xd.abs().amax(1, keepdim=True) * r + (s + 4) * u
    dh = (1 + h.abs()) * off
    v = gd * wd
    within(y, h * wd, wd.abs() * dh + (3 * u + out) * (h * wd).abs(), "y")
    c1, c2 = v.mean(1, keepdim=True), (v * h).mean(1, keepdim=True)
    want = r * (v - c1 - h * c2)
    e1 = (s + 2) * u * v.abs().mean(1, keepdim=True)
    e2 = (s + 4) * u * (v * h).abs().mean(1, keepdim=True) + (v.abs() * dh).mean(1, keepdim=True)
    bound = r * (4 * u * (v.abs() + c1.abs() + (h * c2).abs()) + e1 + h.abs() * e2 + c2.abs() * dh)
    within(gx, want, bound + want.abs() * (2 * off + out), "grad_x")
    gh = gd * h
    within(gw, gh.sum(0), (gd.abs() * dh).sum(0) + (rows + 7) * u * gh.abs().sum(0) + out * gh.sum(0).abs(), "grad_weight")
    within(gb, gd.sum(0), (rows + 7) * u * gd.abs().sum(0) + out * gd.sum(0).abs(), "grad_bias")


@gpu
@pytest.mark.parametrize("name,segment", [("float32", 1024), ("float64", 512), ("bfloat16", 2048)])
@pytest.mark.parametrize("rows", [1, 3])
@pytest.mark.parametrize("past", [-1, 0, 1, 700])
def test_norm_where_segments_are_joined_apart(need_gpu, name, segment, rows, past):
    norm_near(rows, 256 * segment + past, getattr(torch, name), segment)


@gpu
def test_norm_takes_time_as_its_row_is_long(need_gpu):
    """Four times the features take about four times as long: joined again for every
    segment they took 13 times, and 2^30 of them seconds."""
    times = []
    for n in (1 << 24, 1 << 26):
        x, g = torch.randn(1, n, device="cuda"), torch.randn(1, n, device="cuda")
        y, m, r = Q.layer_norm_forward(x)
        ways = (lambda: Q.layer_norm_forward(x), lambda: Q.layer_norm_backward(g, x, m, r))
        for f in ways:
            f()
            least = math.inf
            for _ in range(3):
                a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
                a.record()
                f()
                b.record()
                torch.cuda.synchronize()
                least = min(least, a.elapsed_time(b))
            times.append(least)
    assert times[2] < 8 * times[0] and times[3] < 8 * times[1], times
