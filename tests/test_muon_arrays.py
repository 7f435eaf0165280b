"""What ``muon_step`` and ``orthogonalize`` hand to the C entries for weights and
gradients of any strides (CPU, with the entry replaced by one that reads the
arrays where the kernels would), and their results (needs an MI355X)."""

from __future__ import annotations

import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2301_03251_amd as Q  # noqa: E402
from paper_2301_03251_amd import muon, norm  # noqa: E402


class Posing(torch.Tensor):
    """A CPU tensor that passes the binding's checks for a GPU's."""

    is_cuda = True


def posing(t):
    return t.as_subclass(Posing)


class Arrays:
    """In the library's place: the float32 matrices of a call's entries, by their
    addresses and strides."""

    def __init__(self):
        self.entries = []

    def _read(self, type_, words, count, *_):
        words = ctypes.cast(words, ctypes.POINTER(ctypes.c_int64))
        at = [words[i] for i in range(15 * count)]
        for k in range(count):
            e = at[15 * k:15 * k + 15]
            self.entries.append({"shape": (e[2], e[0], e[1]),
                                 **{name: self._matrices(e, p) for name, p in (("grad", 3), ("momentum", 7), ("out", 11))}})
        return 0

    @staticmethod
    def _matrices(e, p):
        if not e[p]:
            return None
        b, i, j = np.indices((e[2], e[0], e[1]))
        offsets = b * e[p + 1] + i * e[p + 2] + j * e[p + 3]
        return np.array([ctypes.c_float.from_address(e[p] + 4 * int(o)).value for o in offsets.ravel()],
                        np.float32).reshape(offsets.shape)

    ql_muon_step = ql_orthogonalize = _read


@pytest.fixture
def arrays(monkeypatch):
    a = Arrays()
    monkeypatch.setattr(muon, "load", lambda: a)
    monkeypatch.setattr(muon, "_stream", lambda device: None)
    monkeypatch.setattr(muon, "_workspace_bytes", lambda type_, shapes: 4096)
    return a


def weights(count, shape):
    return [posing(torch.arange(float(np.prod(shape))).view(shape) + 1000 * k) for k in range(count)]


def orders(name, shape, device="cpu"):
    """A gradient of the shape whose leading axes do not collapse."""
    if name == "channels_last":
        return torch.randn(shape, device=device).contiguous(memory_format=torch.channels_last)
    if name == "permuted":
        return torch.randn(shape[1], shape[0], *shape[2:], device=device).transpose(0, 1)
    return torch.randn(1, shape[1], *shape[2:], device=device).expand(shape)


@pytest.mark.parametrize("order", ["channels_last", "permuted", "expanded"])
def test_every_gradient_is_there_when_the_step_is_launched(arrays, order):
    """Copies of gradients, and the workspace, lie side by side in memory until then."""
    torch.manual_seed(0)
    p = weights(5, (8, 4, 3, 3))
    g = [posing(orders(order, (8, 4, 3, 3))) for _ in p]
    m = [posing(torch.zeros(8, 4, 3, 3)) for _ in p]
    muon.muon_step(p, g, m)
    assert len(arrays.entries) == 5
    for e, want in zip(arrays.entries, g):
        assert np.array_equal(e["grad"], want.as_subclass(torch.Tensor).reshape(-1, 3, 3).numpy())


@pytest.mark.parametrize("order", ["channels_last", "permuted"])
def test_leading_axes_that_do_not_collapse(arrays, order):
    """Weights, momenta and outputs are written where they lie, each matrix once."""
    torch.manual_seed(0)
    shape = (6, 5, 3, 4)
    p, g, m, o = (orders(order, shape) for _ in range(4))
    muon.muon_step([posing(p)], [posing(g)], [posing(m)])
    for name, t in (("grad", g), ("momentum", m), ("out", p)):
        assert np.array_equal(np.concatenate([e[name] for e in arrays.entries]), t.reshape(-1, 3, 4).numpy())
    arrays.entries.clear()
    assert muon.orthogonalize(posing(g), out=posing(o)).data_ptr() == o.data_ptr()
    for name, t in (("grad", g), ("out", o)):
        assert np.array_equal(np.concatenate([e[name] for e in arrays.entries]), t.reshape(-1, 3, 4).numpy())


def negated(*shape, device="cpu"):
    """A view whose memory holds the values' negatives: the imaginary part of a conjugate."""
    t = torch.randn(*shape, dtype=torch.complex64, device=device).conj().imag
    assert t.is_neg()
    return t


@pytest.mark.parametrize("shape", [(4, 5), (2, 4, 5), (2, 3, 4, 5)])
def test_views_of_negatives(arrays, shape):
    """Read as the values they stand for; not written through."""
    torch.manual_seed(0)
    g = negated(*shape)
    want = g.clone().reshape(-1, *shape[-2:]).numpy()
    muon.orthogonalize(posing(g))
    muon.muon_step([posing(torch.zeros(shape))], [posing(g)], [posing(torch.zeros(shape))])
    assert all(np.array_equal(e["grad"], want) for e in arrays.entries)
    plain = posing(torch.zeros(shape))
    for call in (lambda: muon.orthogonalize(plain, out=posing(g)), lambda: muon.muon_step([posing(g)], [plain], [plain]),
                 lambda: muon.muon_step([plain], [plain], [posing(g)])):
        with pytest.raises(ValueError, match="negative"):
            call()


# ---------------------------------------------------------------------------
# results

gpu = pytest.mark.gpu


@pytest.fixture
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    Q.load()


@gpu
@pytest.mark.parametrize("order", ["channels_last", "permuted", "expanded"])
@pytest.mark.parametrize("beside", [(20, 30), (150, 210)])  # without a workspace, and with one
def test_gradients_of_any_order(need_gpu, order, beside):
    """The same step as with contiguous gradients, bit by bit."""
    torch.manual_seed(1)
    shapes = [(8, 4, 3, 3)] * 5 + [beside]
    p = [torch.randn(s, device="cuda") for s in shapes]
    g = [orders(order, s, "cuda") if len(s) == 4 else torch.randn(s, device="cuda") for s in shapes]
    m = [torch.randn(s, device="cuda") for s in shapes]
    q, n = [t.clone() for t in p], [t.clone() for t in m]
    Q.muon_step(p, g, m)
    Q.muon_step(q, [t.contiguous() for t in g], n)
    assert all(torch.equal(a, b) for a, b in zip(p + m, q + n))


@gpu
@pytest.mark.parametrize("order", ["channels_last", "permuted"])
def test_weights_of_any_order(need_gpu, order):
    torch.manual_seed(2)
    shape = (6, 5, 3, 4)
    p, g, m = ([orders(order, shape, "cuda") for _ in range(2)] for _ in range(3))
    q, h, n = ([t.contiguous() for t in ts] for ts in (p, g, m))
    Q.muon_step(p, g, m)
    Q.muon_step(q, h, n)
    assert all(torch.equal(a, b) for a, b in zip(p + m, q + n))
    out = orders(order, shape, "cuda")
    assert Q.orthogonalize(g[0], out=out) is out
    assert torch.equal(out, Q.orthogonalize(h[0]))
    assert torch.equal(Q.orthogonalize(g[0], out=g[0]), out)
    w = torch.nn.Parameter(orders(order, shape, "cuda"))
    w.grad = orders("expanded", shape, "cuda")
    opt = Q.Muon([w], lr=0.1)
    want, state = w.detach().contiguous(), torch.zeros(shape, device="cuda")
    opt.step()
    Q.muon_step([want], [w.grad.contiguous()], [state], lr=0.1)
    assert torch.equal(w, want)


@pytest.mark.parametrize("shape", [(7, 12), (3, 5, 12), (7, 1), (3, 5, 1), (1,)])
def test_norm_rows_of_views_of_negatives(shape):
    x = negated(*shape)
    rows, count, stride = norm._rows(x, x.shape)
    there = torch.empty(0).set_(rows.untyped_storage(), rows.storage_offset(), (count, shape[-1]), (stride, 1))
    assert torch.equal(there, x.reshape(count, shape[-1]))
    with pytest.raises(ValueError):
        norm._parameter(negated(1), x.get_device(), 1, "weight")


@gpu
def test_norm_of_views_of_negatives(need_gpu):
    torch.manual_seed(3)
    for shape in ((7, 12), (3, 5, 12), (7, 1), (3, 5, 1)):
        x, g = negated(*shape, device="cuda"), negated(*shape, device="cuda")
        y, mean, rstd = Q.layer_norm_forward(x)
        want, m, r = Q.layer_norm_forward(x.clone())
        assert torch.equal(y, want) and torch.equal(mean, m)
        assert torch.equal(Q.layer_norm_backward(g, x, mean, rstd)[0], Q.layer_norm_backward(g.clone(), x.clone(), m, r)[0])
