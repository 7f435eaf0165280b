"""Embedding lookup and its gradient: refusals (CPU), and values against 64 bits
(needs an MI355X).

A row is one product and one rounding: off by u and half a step. A gradient sums
at most two chunks of 64 rows in the arithmetic's unit roundoff u (24 bits: 2^-24), or the
sums of chunks in fp64: off by (128 + 3) u of the sum of magnitudes, and half a step.
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


def _fwd(lib, type_=F32, wide=1, n=3, rows=5, d=4, t=FAKE, w=FAKE, ws=4, scale=1.0, y=FAKE):
    return lib.ql_embedding_forward(type_, wide, n, rows, d, t, w, ws, scale, 0, 0, y, None)


@pytest.mark.parametrize("kw", [
    dict(type_=4), dict(type_=-1), dict(n=-1), dict(n=1 << 31), dict(rows=0), dict(rows=1 << 31), dict(d=0),
    dict(d=(1 << 22) + 1), dict(rows=1 << 30, d=1 << 20), dict(n=1 << 30, d=1 << 20), dict(scale=float("nan")),
    dict(scale=float("inf")), dict(ws=-1), dict(rows=1 << 30, ws=1 << 30), dict(t=None), dict(w=None), dict(y=None),
    dict(t=ctypes.c_void_p(0x1004)), dict(t=ctypes.c_void_p(0x1002), wide=0), dict(w=ODD), dict(y=ODD),
])
def test_forward_refuses(lib, kw):
    assert _fwd(lib, **kw) == -1
    assert lib.ql_last_error()


def _bwd(lib, type_=F32, wide=1, n=3, rows=5, d=4, t=FAKE, g=FAKE, gs=4, scale=1.0, out=FAKE, ws=FAKE, ws_bytes=1 << 20):
    return lib.ql_embedding_backward(type_, wide, n, rows, d, t, g, gs, scale, 0, 0, out, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(type_=9), -1), (dict(n=-1), -1), (dict(rows=0), -1), (dict(d=0), -1), (dict(scale=float("-inf")), -1),
    (dict(gs=-1), -1), (dict(t=None), -1), (dict(g=None), -1), (dict(out=None), -1), (dict(out=None, n=0), -1),
    (dict(t=ODD, wide=0), -1), (dict(g=ODD), -1), (dict(out=ODD), -1), (dict(ws=None), -1),
    (dict(ws=ctypes.c_void_p(0x1008)), -1), (dict(ws_bytes=16), -2),
])
def test_backward_refuses(lib, kw, code):
    assert _bwd(lib, **kw) == code
    assert lib.ql_last_error()


def test_workspace_bytes(lib):
    out = ctypes.c_size_t()
    assert lib.ql_embedding_workspace_bytes(F32, 4, 8, 1, None) == -1
    assert lib.ql_embedding_workspace_bytes(F32, -4, 8, 1, ctypes.byref(out)) == -1
    for n in (0, 1, 64, 65, 8192, 8193, 1 << 20, (1 << 31) - 1):
        for rows in (1, 255, 1 << 20, (1 << 31) - 1):
            assert lib.ql_embedding_workspace_bytes(BF16, n, rows, 16, ctypes.byref(out)) == 0
            chunk = max(8, min(64, n // 2048 // 8 * 8))
            assert 8 * n <= out.value <= 16 * n + (n // chunk + 1) * 2 * 16 * 4 + (n // 1024 + 2) * 4096 + 4096


def test_no_tokens(lib):
    assert _fwd(lib, n=0, t=None, w=None, y=None) == 0


def test_python_refuses_without_a_gpu():
    w, t = torch.zeros(4, 3), torch.zeros(2, dtype=torch.int64)
    for bad in (lambda: Q.embedding(t, w), lambda: Q.embedding(t, w[0]), lambda: Q.embedding(t, w.long()),
                lambda: Q.embedding_backward(torch.zeros(2, 3), t, 4)):
        with pytest.raises(ValueError):
            bad()


# ---------------------------------------------------------------------------
# values

@pytest.fixture(scope="module")
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    Q.load()


def make(n, rows, d, dtype, seed, kind="even"):
    g = torch.Generator().manual_seed(seed)
    if kind == "even":
        t = torch.randint(rows, (n,), generator=g)
    elif kind == "one":
        t = torch.full((n,), rows // 2)
    elif kind == "few":
        t = torch.randint(min(rows, 3), (n,), generator=g) * ((rows - 1) // 2)
    else:  # frequent and rare ones
        t = (rows ** torch.rand(n, generator=g, dtype=torch.float64)).long().clamp_(1, rows) - 1
    w = torch.randn(rows, d, generator=g).to(dtype)
    return t.cuda(), w.cuda(), torch.randn(n, d, generator=g).to(dtype).cuda()


def check(t, w, grad, name, scale=1.0, padding=None):
    rows, d = w.shape
    n, out = t.numel(), 1.01 * OUT_U[name]
    tiny = 6e-8 * (name == "f16")
    u = 2.0 ** -53 if name == "f64" else 2.0 ** -24
    y = Q.embedding_forward(t, w, scale, padding)
    keep = torch.ones(n, dtype=torch.bool, device="cuda") if padding is None else t != padding
    want = torch.where(keep[:, None], w.double()[t.long().clamp(0, rows - 1)] * scale, 0.0)
    assert y.dtype == w.dtype and y.shape == (n, d)
    assert ((y.double() - want).abs() <= want.abs() * (u + out) + tiny).all()
    got = Q.embedding_backward(grad, t, rows, scale, padding)
    # summed on the host, in order
    at, kept = t.long()[keep].cpu(), grad.double()[keep].cpu()
    total = torch.zeros(rows, d, dtype=torch.float64).index_add_(0, at, kept).cuda()
    size = torch.zeros(rows, d, dtype=torch.float64).index_add_(0, at, kept.abs()).cuda()
    bound = (size * 131 * u + total.abs() * out) * abs(scale) + tiny
    if name == "f64":  # the order of the reference's own sums counts too
        bound += size * abs(scale) * 2.0 ** -53 * (8 + torch.bincount(t.long()[keep], minlength=rows).max().item())
    assert got.dtype == grad.dtype and got.shape == (rows, d)
    assert ((got.double() - total * scale).abs() <= bound).all()
    assert not got[torch.bincount(t.long()[keep], minlength=rows) == 0].any()


@gpu
@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("n,rows,d", [(1, 1, 1), (1, 9, 3), (3, 2, 4), (63, 5, 8), (64, 300, 10), (65, 3, 16), (129, 1000, 65),
                                      (1000, 257, 33), (4096, 1000, 64), (4095, 70000, 7), (300, 32, 1031), (20, 12, 5000)])
def test_values(need_gpu, n, rows, d, name):
    t, w, g = make(n, rows, d, TYPES[name], seed=n + d)
    check(t, w, g, name)
    check(t.int(), w, g, name, scale=-1.7, padding=int(t[0]))


@gpu
@pytest.mark.parametrize("kind", ["even", "one", "few", "frequent"])
@pytest.mark.parametrize("n,rows,d,name", [(4096, 50, 20, "f32"), (4097, 3, 12, "f32"), (5000, 200, 7, "f16"), (20001, 1500, 66, "bf16"),
                                           (70000, 300000, 16, "f32"), (8191, 40, 9, "f64"), (8192, 3000, 24, "bf16"), (8193, 700, 17, "f32"), (9000, 1 << 21, 4, "f64"), (140000, 1023, 130, "bf16"),
                                           (300000, 1024, 5, "f32")])
def test_sorts_and_runs(need_gpu, n, rows, d, name, kind):
    """Both sorts, one to three digits, tokens of one place and of nearly all."""
    t, w, g = make(n, rows, d, TYPES[name], seed=rows, kind=kind)
    check(t, w, g, name, scale=0.3)


@gpu
@pytest.mark.parametrize("n", [60, 4096, 8192, 10000])
def test_tokens_outside_the_table(need_gpu, n):
    """They have rows of NaN and no gradient; the padding may be one of them."""
    t, w, g = make(n, 40, 24, torch.float32, seed=n)
    bad = torch.tensor([-1, 40, 41, -(1 << 62), (1 << 32) + 3, (1 << 63) - 1], device="cuda")
    at = torch.randperm(n, generator=torch.Generator().manual_seed(n))[:6].cuda()
    want = Q.embedding_forward(t, w)
    inside = torch.ones(n, dtype=torch.bool, device="cuda")
    inside[at] = False
    left = torch.zeros_like(g)
    left[inside] = g[inside]
    total = Q.embedding_backward(left, torch.where(inside, t, torch.zeros_like(t)), 40)
    t[at] = bad
    g[at] = float("nan")
    y = Q.embedding_forward(t, w)
    assert torch.isnan(y[at]).all() and torch.equal(y[inside], want[inside])
    got = Q.embedding_backward(g, t, 40)
    # the same sums but for zeros among them, whose chunks may end elsewhere
    size = torch.zeros_like(total).index_add_(0, t[inside], g[inside].abs())
    assert ((got - total).abs() <= size * 262 * 2.0 ** -24).all()
    y = Q.embedding_forward(t, w, padding=-1)
    assert not y[at[0]].any() and torch.isnan(y[at[1:]]).all()
    assert torch.equal(Q.embedding_backward(g, t, 40, padding=-1), got)
    everywhere = torch.full((n,), 1 << 40, device="cuda")
    assert not Q.embedding_backward(g, everywhere, 40).any() and torch.isnan(Q.embedding_forward(everywhere, w)).all()


@gpu
def test_padding(need_gpu):
    """Zeros whatever the row holds, and gradients of padded places that are never read as numbers."""
    t, w, g = make(500, 20, 12, torch.float32, seed=2)
    w[7] = float("nan")
    t[:100] = 7
    g[:100] = float("nan")
    g[t == 7] = float("inf")
    y = Q.embedding_forward(t, w, 2.0, 7)
    assert not y[t == 7].any() and torch.isfinite(y).all()
    got = Q.embedding_backward(g, t, 20, 2.0, 7)
    assert torch.isfinite(got).all() and not got[7].any()
    assert not Q.embedding_backward(g, torch.full_like(t, 7), 20, 2.0, 7).any()


@gpu
def test_bad_gradients_stay_in_their_row(need_gpu):
    t, w, g = make(20000, 300, 40, torch.float32, seed=5, kind="frequent")
    want = Q.embedding_backward(g, t, 300)
    g[777, 3] = float("nan")
    g[778, 4] = float("inf")
    got = Q.embedding_backward(g, t, 300)
    assert torch.isnan(got[t[777], 3]) and torch.isinf(got[t[778], 4])
    want[t[777], 3] = got[t[777], 3] = 0
    want[t[778], 4] = got[t[778], 4] = 0
    assert torch.equal(got, want)


@gpu
@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("d,pad,shift", [(5, 1, 0), (24, 3, 1), (1001, 7, 5)])
def test_strides_and_alignment(need_gpu, name, d, pad, shift):
    t, w, g = make(300, 50, d, TYPES[name], seed=d)

    def inside(x):
        wide = torch.full((x.shape[0], d + pad + shift), float("nan"), dtype=x.dtype, device="cuda")
        wide[:, shift:shift + d] = x
        return wide[:, shift:shift + d]

    want, total = Q.embedding_forward(t, w, 0.7), Q.embedding_backward(g, t, 50, 0.7)
    assert torch.equal(Q.embedding_forward(t, inside(w), 0.7), want)
    assert torch.equal(Q.embedding_backward(inside(g), t, 50, 0.7), total)
    assert torch.equal(Q.embedding_forward(t, w.t().contiguous().t(), 0.7), want)
    assert torch.equal(Q.embedding_forward(t, torch._neg_view(-w), 0.7), want)
    assert torch.equal(Q.embedding_backward(torch._neg_view(-g), t, 50, 0.7), total)
    assert torch.equal(Q.embedding_forward(t.view(3, 100).t(), w, 0.7), want.view(3, 100, d).transpose(0, 1))
    assert torch.equal(Q.embedding_backward(g.view(3, 100, d).transpose(0, 1), t.view(3, 100).t(), 50, 0.7),
                       Q.embedding_backward(g.view(3, 100, d).transpose(0, 1).contiguous(), t.view(3, 100).t().contiguous(), 50, 0.7))
    assert torch.equal(Q.embedding_forward(torch.stack((t, t), 1)[:, 0].int(), w, 0.7), want)
    assert torch.equal(Q.embedding_backward(g[:1].expand(300, d), t, 50), Q.embedding_backward(g[:1].repeat(300, 1), t, 50))
    one = torch.ones((), dtype=g.dtype, device="cuda").expand(300, d)
    assert torch.equal(Q.embedding_backward(one, t, 50), Q.embedding_backward(one.contiguous(), t, 50))
    assert torch.equal(Q.embedding_forward(t[0], w, 0.7), want[0])
    assert torch.equal(Q.embedding_forward(t, w[:1].expand(50, d), 0.7), Q.embedding_forward(torch.zeros_like(t), w, 0.7))


@gpu
def test_nothing_to_look_up(need_gpu):
    t = torch.empty((0, 4), dtype=torch.int64, device="cuda")
    w = torch.randn(6, 3, device="cuda", requires_grad=True)
    y = Q.embedding(t, w)
    assert y.shape == (0, 4, 3)
    y.sum().backward()
    assert w.grad.shape == (6, 3) and not w.grad.any()


@gpu
def test_autograd_and_module(need_gpu):
    layer = Q.Embedding(30, 12, scale=3.0, padding=0)
    t = torch.randint(30, (5, 7), device="cuda")
    g = torch.randn(5, 7, 12, device="cuda")
    y = layer(t)
    assert torch.equal(y, Q.embedding_forward(t, layer.weight, 3.0, 0))
    y.backward(g)
    assert torch.equal(layer.weight.grad, Q.embedding_backward(g, t, 30, 3.0, 0))
    with torch.no_grad():
        assert torch.equal(layer(t), y)
    # linear in the table: differences of any size agree, in float64 to its rounding
    w = torch.randn(30, 12, dtype=torch.float64, device="cuda", requires_grad=True)
    dw = torch.randn_like(w)
    Q.embedding(t, w, 3.0, 0).backward(g.double())
    with torch.no_grad():
        change = (g * (Q.embedding(t, w + dw, 3.0, 0) - Q.embedding(t, w - dw, 3.0, 0))).sum() / 2
    assert (change - (w.grad * dw).sum()).abs() <= 1e-13 * 3 * (g.abs().sum() * (dw.abs().max() + w.abs().max()))
    y = Q.embedding(t, w)
    t.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    with fwd.dual_level(), pytest.raises(RuntimeError, match="forward mode AD"):
        Q.embedding(t, fwd.make_dual(w.detach(), dw))


@gpu
def test_python_refuses(need_gpu):
    t, w, g = make(10, 6, 4, torch.float32, seed=1)
    for bad in (lambda: Q.embedding(t.cpu(), w), lambda: Q.embedding(t.float(), w), lambda: Q.embedding(t.short(), w),
                lambda: Q.embedding(t, w[0]), lambda: Q.embedding(t, w.int()), lambda: Q.embedding_backward(g[:9], t, 6),
                lambda: Q.embedding_backward(g.cpu(), t, 6), lambda: Q.embedding(t, w, padding=1 << 63)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: Q.embedding(t, w[:0]), lambda: Q.embedding(t, w, float("nan")), lambda: Q.embedding_backward(g, t, 0),
                lambda: Q.embedding_backward(g, t, 1 << 31), lambda: Q.embedding(t, w[:, :0])):
        with pytest.raises(Q.QLError):
            bad()


@gpu
@pytest.mark.parametrize("n", [900, 30000])
def test_other_stream_and_graph(need_gpu, n):
    t, w, g = make(n, 500, 48, torch.bfloat16, seed=5, kind="frequent")

    def step():
        return Q.embedding_forward(t, w, 2.0, 3), Q.embedding_backward(g, t, 500, 2.0, 3)

    want = step()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        got = step()
    torch.cuda.current_stream().wait_stream(stream)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in range(3):
        t.copy_(make(n, 500, 48, torch.bfloat16, seed=50 + seed, kind=("one", "even", "few")[seed])[0])
        want = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, want))


@gpu
def test_same_bits_again(need_gpu):
    t, w, g = make(100000, 900, 70, torch.float32, seed=8, kind="frequent")
    first = Q.embedding_backward(g, t, 900)
    for _ in range(3):
        assert torch.equal(Q.embedding_backward(g, t, 900), first)
    # and whatever columns there are beside it
    assert torch.equal(Q.embedding_backward(g[:, :20], t, 900), first[:, :20])


@gpu
def test_offsets_past_32_bits(need_gpu):
    rows, d = 70000, 33000
    w = torch.zeros((rows, d), dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([0, 1, rows // 2, rows - 2, rows - 1], device="cuda")
    w[at] = torch.randn(5, d, device="cuda").bfloat16()
    assert w.numel() > 1 << 31
    y = Q.embedding_forward(at, w)
    assert torch.equal(y, w[at])
    got = Q.embedding_backward(y, at, rows)
    assert torch.equal(got[at], y) and not got[2:rows // 2].any()
    del got, w
    t = torch.arange(rows, device="cuda") % 8
    g = torch.ones((), dtype=torch.bfloat16, device="cuda").expand(rows, 1).repeat(1, d)
    assert g.numel() > 1 << 31
    g[-1] = 3
    total = Q.embedding_backward(g, t, 8)
    count = torch.full((8, 1), rows // 8, device="cuda", dtype=torch.float32)
    count[(rows - 1) % 8] += 2
    assert torch.equal(total, count.bfloat16().expand(8, d))
