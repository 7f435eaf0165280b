"""What autograd sees of the operators around a quantum layer: tangents of
forward mode, vmap, and writes to tensors that a graph has saved. The dispatch
is checked on the CPU with the kernels' part replaced, the rest needs an MI355X."""

from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")
import torch.autograd.forward_ad as fwd  # noqa: E402

import paper_2301_03251_amd as Q  # noqa: E402
from paper_2301_03251_amd import muon, norm  # noqa: E402

gpu = pytest.mark.gpu


@pytest.fixture
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    Q.load()


@pytest.fixture
def plain_forward(monkeypatch):
    def forward(x, weight=None, bias=None, eps=1e-5, stats=True):
        return x.detach().clone(), x.detach()[..., 0], x.detach()[..., 0]
    monkeypatch.setattr(norm, "layer_norm_forward", forward)


def lost_tangent(device, which, grad):
    """layer_norm of a dual tensor has no tangent to give: it says so."""
    ts = [torch.randn(3, 4, device=device), torch.randn(4, device=device), torch.randn(4, device=device)]
    with torch.set_grad_enabled(grad), fwd.dual_level():
        ts[which] = fwd.make_dual(ts[which], torch.ones_like(ts[which]))
        with pytest.raises(RuntimeError, match="forward mode AD"):
            Q.layer_norm(*ts)
        ts[which] = fwd.unpack_dual(ts[which]).primal
        Q.layer_norm(*ts)  # no tangent, no error


@pytest.mark.parametrize("which", [0, 1, 2])
@pytest.mark.parametrize("grad", [True, False])
def test_a_tangent_is_not_dropped(plain_forward, which, grad):
    lost_tangent("cpu", which, grad)


@gpu
@pytest.mark.parametrize("which", [0, 1, 2])
@pytest.mark.parametrize("grad", [True, False])
def test_a_tangent_is_not_dropped_on_the_gpu(need_gpu, which, grad):
    lost_tangent("cuda", which, grad)


@gpu
def test_transforms_are_refused(need_gpu):
    x = torch.randn(3, 4, 5, device="cuda")
    with pytest.raises(RuntimeError):
        torch.func.vmap(Q.layer_norm)(x)
    with pytest.raises(RuntimeError):
        torch.func.jvp(Q.layer_norm, (x,), (x,))
    with pytest.raises(RuntimeError):
        torch.func.grad(lambda t: Q.layer_norm(t).sum())(x)


class Posing(torch.Tensor):
    """A CPU tensor that passes the binding's checks for a GPU's."""

    is_cuda = True


class Idle:
    """In the library's place: entries that do nothing."""

    def ql_orthogonalize(self, *_):
        return 0

    ql_muon_step = ql_orthogonalize


@pytest.fixture
def idle(monkeypatch):
    monkeypatch.setattr(muon, "load", Idle)
    monkeypatch.setattr(muon, "_stream", lambda device: None)
    monkeypatch.setattr(muon, "_workspace_bytes", lambda type_, shapes: 0)


def saved_out_is_seen(make):
    """out= is a write like any in place: a graph that has saved the array says so."""
    w = make(6, 4)
    for out_is_input in (False, True):
        y = (torch.ones(6, 4, device=w.device, requires_grad=True) * w).sum()
        version = w._version
        Q.orthogonalize(w if out_is_input else make(6, 4), out=w)
        assert w._version > version
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()


def inference_tensors(make):
    """They have no version to count."""
    with torch.inference_mode():
        p, g, m = make(6, 4), make(6, 4), make(6, 4)
        Q.muon_step([p], [g], [m])
        assert Q.orthogonalize(g, out=p) is p


def graph_is_not_dropped(make):
    """What autograd would have to follow is refused; under no_grad and detached it runs."""
    g = make(6, 4).requires_grad_()
    for call in (lambda: Q.orthogonalize(g), lambda: Q.orthogonalize(g * 2), lambda: Q.orthogonalize(make(6, 4), out=g)):
        with pytest.raises(ValueError, match="not differentiable"):
            call()
    with fwd.dual_level(), pytest.raises(ValueError, match="not differentiable"):
        Q.orthogonalize(fwd.make_dual(make(6, 4), make(6, 4)))
    assert not Q.orthogonalize(g.detach()).requires_grad
    with torch.no_grad():
        assert not Q.orthogonalize(g).requires_grad


def test_orthogonalize_is_seen_by_autograd(idle):
    saved_out_is_seen(lambda *s: torch.randn(s).as_subclass(Posing))
    inference_tensors(lambda *s: torch.randn(s).as_subclass(Posing))


def test_orthogonalize_does_not_drop_a_graph(idle):
    graph_is_not_dropped(lambda *s: torch.randn(s).as_subclass(Posing))


@gpu
def test_orthogonalize_is_seen_by_autograd_on_the_gpu(need_gpu):
    saved_out_is_seen(lambda *s: torch.randn(s, device="cuda"))
    inference_tensors(lambda *s: torch.randn(s, device="cuda"))


@gpu
def test_orthogonalize_does_not_drop_a_graph_on_the_gpu(need_gpu):
    graph_is_not_dropped(lambda *s: torch.randn(s, device="cuda"))
