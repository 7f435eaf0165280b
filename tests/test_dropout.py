"""Dropout: refusals (CPU), the generator against its published answers and the
kernel against it (needs an MI355X).

A kept element is x times 1 / (1 - p), each rounded to the arithmetic's unit
roundoff u, and their product rounded to x's type: off by 2 u and half a step.
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
KEY = (0x0123456789ABCDEF, 0xFEDCBA9876543210)
gpu = pytest.mark.gpu


def philox(counters, offset, seed):
    """Four words for each counter (uint64), [n, 4]."""
    low = np.uint64(0xFFFFFFFF)
    s = np.uint64(32)
    c = [counters & low, counters >> s, np.full_like(counters, offset & 0xFFFFFFFF), np.full_like(counters, offset >> 32)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> s) ^ c[1] ^ np.uint64(k[0]), q & low, (p >> s) ^ c[3] ^ np.uint64(k[1]), p & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, -1)


def kept(first, n, p, key=KEY):
    """The mask of elements first ... first + n - 1."""
    counters = np.arange(first // 4, (first + n + 3) // 4, dtype=np.uint64)
    words = philox(counters, key[1], key[0]).reshape(-1)[first % 4:first % 4 + n]
    return torch.from_numpy(words.astype(np.int64) >= round(p * 2.0 ** 32))


def test_the_generators_published_answers():
    """Known answers of Philox 4x32-10 that its authors publish with it."""
    def words(c0, c1, c2, c3, k0, k1):
        return [int(w) for w in philox(np.array([c1 << 32 | c0], np.uint64), c3 << 32 | c2, k1 << 32 | k0)[0]]
    assert words(0, 0, 0, 0, 0, 0) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    assert words(*[0xffffffff] * 6) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]
    assert words(0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344, 0xa4093822, 0x299f31d0) == [
        0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1]


# ---------------------------------------------------------------------------
# refusals: nothing is launched, so the addresses are never read

@pytest.fixture(scope="module")
def lib():
    return Q.load()


FAKE = ctypes.c_void_p(0x1000)
ODD = ctypes.c_void_p(0x1001)


def _call(lib, type_=F32, rows=2, n=4, x=FAKE, stride=4, p=0.5, key=None, y=FAKE):
    return lib.ql_dropout(type_, rows, n, x, stride, p, 1, 2, key, y, None)


@pytest.mark.parametrize("kw", [
    dict(type_=4), dict(rows=-1), dict(n=0), dict(n=(1 << 30) + 1), dict(rows=1 << 40, n=1 << 20), dict(stride=-1),
    dict(rows=1 << 30, stride=1 << 30), dict(p=-1e-9), dict(p=1.0000001), dict(p=float("nan")), dict(x=None), dict(y=None),
    dict(x=ODD), dict(y=ODD), dict(key=ctypes.c_void_p(0x1004)),
])
def test_refuses(lib, kw):
    assert _call(lib, **kw) == -1
    assert lib.ql_last_error()


def test_no_rows(lib):
    assert _call(lib, rows=0, x=None, y=None) == 0


def test_python_refuses():
    with pytest.raises(ValueError):
        Q.dropout(torch.zeros(2, 4), 0.5, KEY)
    for p in (-0.1, 1.1, float("nan")):
        with pytest.raises(ValueError):
            Q.Dropout(p, device="cpu")


def test_module_without_a_gpu():
    """Evaluation and p = 0 are the identity; the key is part of the state."""
    x = torch.randn(3, 4)
    layer = Q.Dropout(0.5, seed=7, device="cpu").eval()
    assert layer(x) is x and Q.Dropout(0.0, device="cpu")(x) is x
    assert layer.state_dict()["key"].tolist() == [7, 0]
    torch.manual_seed(3)
    first = Q.Dropout(0.5, device="cpu").key.tolist()
    assert Q.Dropout(0.5, device="cpu").key.tolist() != first
    torch.manual_seed(3)
    assert Q.Dropout(0.5, device="cpu").key.tolist() == first


# ---------------------------------------------------------------------------
# values

@pytest.fixture(scope="module")
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    Q.load()


def check(x, p, y, keep, name):
    x, y = x.double().cpu(), y.double().cpu()
    keep = keep.view(x.shape)
    want = torch.where(keep, x / (1 - p) if p < 1 else x, torch.zeros_like(x))
    u = 2.0 ** -53 if name == "f64" else 2.0 ** -24
    # float64 results are compared in their own arithmetic, whose rounding counts too
    bound = want.abs() * (2 * u + 1.01 * OUT_U[name] + 2 * 2.0 ** -53) + 6e-8 * (name == "f16")
    assert ((y - want).abs() <= bound).all()
    assert (y[~keep] == 0).all()


@gpu
@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("rows,n", [(1, 1), (1, 3), (1, 4), (2, 5), (3, 7), (1, 8), (5, 9), (33, 31), (64, 256), (1037, 1001), (2, 70001)])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.999, 1.0])
def test_values(need_gpu, rows, n, p, name):
    torch.manual_seed(rows + n)
    x = torch.randn(rows, n, device="cuda").to(TYPES[name])
    y = Q.dropout_forward(x, p, KEY)
    check(x, p, y, kept(0, rows * n, p), name)


@gpu
@pytest.mark.parametrize("name", ["f32", "bf16", "f64"])
@pytest.mark.parametrize("n,pad,shift", [(5, 1, 0), (8, 3, 1), (64, 8, 0), (999, 7, 5)])
def test_strides_and_alignment(need_gpu, name, n, pad, shift):
    """The mask goes by the place in x, not in memory."""
    x = torch.randn(37, n, device="cuda").to(TYPES[name])
    wide = torch.full((37, n + pad + shift), float("nan"), dtype=x.dtype, device="cuda")
    wide[:, shift:shift + n] = x
    want = Q.dropout_forward(x, 0.3, KEY)
    assert torch.equal(Q.dropout_forward(wide[:, shift:shift + n], 0.3, KEY), want)
    assert torch.equal(Q.dropout_forward(x.t().contiguous().t(), 0.3, KEY), want)
    assert torch.equal(Q.dropout_forward(x.view(37, 1, n), 0.3, KEY).view(37, n), want)
    assert torch.equal(Q.dropout_forward(x[:1].expand(37, n), 0.3, KEY), Q.dropout_forward(x[:1].repeat(37, 1), 0.3, KEY))
    assert torch.equal(Q.dropout_forward(torch._neg_view(-x), 0.3, KEY), want)
    assert torch.equal(Q.dropout_forward(x.view(-1)[1:], 0.3, KEY), Q.dropout_forward(x.view(-1)[1:].clone(), 0.3, KEY))


@gpu
def test_what_is_dropped_is_zero(need_gpu):
    x = torch.tensor([float("nan"), float("inf"), -float("inf"), 3e38], device="cuda").repeat(4000)
    keep = kept(0, x.numel(), 0.5).cuda()
    y = Q.dropout_forward(x, 0.5, KEY)
    assert not y[~keep].any()
    assert torch.isnan(y[keep & x.isnan()]).all() and y[keep & ~x.isnan()].isinf().all()
    assert not Q.dropout_forward(x, 1.0, KEY).any()
    assert not Q.dropout_forward(x, 1 - 1e-15, KEY).any()


@gpu
def test_keys(need_gpu):
    """As numbers and on the device; other seeds and offsets are other masks."""
    x = torch.ones(100, 33, device="cuda")
    want = Q.dropout_forward(x, 0.5, (5, 9))
    assert torch.equal(Q.dropout_forward(x, 0.5, torch.tensor([5, 9], device="cuda")), want)
    for key in ((6, 9), (5, 8), (5 + (1 << 32), 9), (5, 9 + (1 << 32)), ((1 << 64) - 1, 9), (5, (1 << 64) - 1)):
        y = Q.dropout_forward(x, 0.5, key)
        assert torch.equal(y.view(-1).cpu() != 0, kept(0, 3300, 0.5, key)) and not torch.equal(y, want)
    big = torch.tensor([-1, -2], device="cuda")  # the bits of 2^64 - 1 and 2^64 - 2
    assert torch.equal(Q.dropout_forward(x, 0.5, big), Q.dropout_forward(x, 0.5, ((1 << 64) - 1, (1 << 64) - 2)))


@gpu
def test_shares(need_gpu):
    """n masks of probability q: their mean is within 5 standard deviations."""
    n = 1 << 22
    x = torch.ones(n, device="cuda")
    for p in (0.1, 0.5, 0.9):
        share = (Q.dropout_forward(x, p, KEY) != 0).double().mean().item()
        assert abs(share - (1 - p)) <= 5 * (p * (1 - p) / n) ** 0.5


@gpu
def test_python_refuses_on_the_gpu(need_gpu):
    x = torch.ones(4, 8, device="cuda")
    for key in ((1,), (-1, 0), (0, 1 << 64), torch.tensor([1, 2]), torch.tensor([1, 2], device="cuda", dtype=torch.int32),
                torch.tensor([1, 2, 3], device="cuda"), torch.tensor([1, 0, 2, 0], device="cuda")[::2]):
        with pytest.raises(ValueError):
            Q.dropout(x, 0.5, key)
    with pytest.raises(Q.QLError):
        Q.dropout(x, 1.5, KEY)
    with pytest.raises(ValueError):
        Q.dropout(x.long(), 0.5, KEY)
    assert Q.dropout(x[:0], 0.5, KEY).shape == (0, 8)


@gpu
def test_autograd(need_gpu):
    """The gradient goes through the elements that were kept; it is linear, so
    differences of any size agree: 2 u from each of the two products."""
    x = torch.randn(20, 30, dtype=torch.float64, device="cuda", requires_grad=True)
    g, d = torch.randn_like(x), torch.randn_like(x)
    key = torch.tensor([3, 4], device="cuda")
    y = Q.dropout(x, 0.25, key)
    y.backward(g)
    assert torch.equal(x.grad, Q.dropout_forward(g, 0.25, (3, 4)))
    with torch.no_grad():
        change = (g * (Q.dropout(x + d, 0.25, key) - Q.dropout(x - d, 0.25, key))).sum() / 2
        size = (g.abs() * (x.abs() + d.abs())).sum() / 0.75
    assert (change - (x.grad * d).sum()).abs() <= 1e-14 * size * 20
    y = Q.dropout(x, 0.25, key)
    key.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward(g)
    x.grad = None
    Q.dropout(x, 0.25, (3, 4)).sum().backward()
    assert torch.equal(x.grad, Q.dropout_forward(torch.ones_like(x), 0.25, (3, 4)))
    with fwd.dual_level(), pytest.raises(RuntimeError, match="forward mode AD"):
        Q.dropout(fwd.make_dual(x.detach(), g), 0.5, KEY)


@gpu
def test_module(need_gpu):
    x = torch.randn(50, 40, device="cuda", requires_grad=True)
    layer = Q.Dropout(0.4, seed=11)
    ys = [layer(x) for _ in range(3)]
    for k, y in enumerate(ys):
        assert torch.equal(y, Q.dropout_forward(x, 0.4, (11, k)))
    # backward passes after later calls draw their own masks
    torch.autograd.grad(ys[0].sum(), x, retain_graph=True)
    for k in (1, 0, 2):
        assert torch.equal(torch.autograd.grad(ys[k].sum(), x)[0], Q.dropout_forward(torch.ones_like(x), 0.4, (11, k)))
    other = Q.Dropout(0.4)
    other.load_state_dict(layer.state_dict())
    assert torch.equal(other(x), Q.dropout_forward(x, 0.4, (11, 3)))
    assert layer.eval()(x) is x


@gpu
def test_graph_draws_new_masks(need_gpu):
    """Forward and backward captured together: each replay is the eager call of the next offset."""
    x = torch.randn(64, 100, device="cuda").bfloat16()
    g = torch.randn_like(x)
    layer = Q.Dropout(0.3, seed=5)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        Q.dropout_forward(x, 0.3, layer.key)
        assert torch.equal(Q.dropout_forward(x, 0.3, (5, 0)), Q.dropout_forward(x, 0.3, layer.key))
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        key = layer.key.clone()
        y = layer(x)
        gx = Q.dropout_forward(g, 0.3, key)
    before = int(layer.key[1])
    for k in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, Q.dropout_forward(x, 0.3, (5, before + k)))
        assert torch.equal(gx, Q.dropout_forward(g, 0.3, (5, before + k)))
        torch.cuda.synchronize()


@gpu
@pytest.mark.parametrize("stride", [0, 7])
def test_places_past_32_bits(need_gpu, stride):
    rows, n = 66000, 66001
    x = torch.ones((rows, n + stride), dtype=torch.bfloat16, device="cuda")[:, :n]
    assert x.numel() > 1 << 32
    y = Q.dropout_forward(x, 0.5, KEY)
    for row in (0, 1, rows // 2, rows - 1):
        assert torch.equal(y[row].cpu() != 0, kept(row * n, n, 0.5))
    assert abs((y[::1000] != 0).double().mean().item() - 0.5) < 0.01
