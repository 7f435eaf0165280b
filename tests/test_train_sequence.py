"""The sequence operators together, as the example uses them: embedding, dropout,
norm with the residual, recurrence, quantum layer (needs an MI355X)."""

from __future__ import annotations

import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
import paper_2301_03251_amd as Q  # noqa: E402

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("train_sequence", os.path.join(ROOT, "examples", "train_sequence.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("dtype,qubits,batch", [("c64", 8, 32), ("c128", 4, 16)])
def test_runs(example, dtype, qubits, batch):
    model, losses = example.train(steps=5, qubits=qubits, batch=batch, length=70, dtype=dtype, log=lambda *_: None)
    assert all(v == v and v != float("inf") for v in losses)
    assert all(torch.isfinite(p).all() for p in model.parameters())


def test_same_run_again(example):
    """Every operator sums in a fixed order and masks come from counters: two runs agree bit by bit."""
    runs = [example.train(steps=4, qubits=5, batch=16, length=40, log=lambda *_: None) for _ in range(2)]
    assert runs[0][1] == runs[1][1]
    assert all(torch.equal(p, q) for p, q in zip(runs[0][0].parameters(), runs[1][0].parameters()))


def plain(model, tokens, lengths, params):
    """The same network from elementary operations, in the model's float64."""
    x = 0.5 * params["embedding.weight"][tokens] * (tokens != 0)[..., None]

    def masked(module, t, name):
        if not model.training:
            return t
        keep = (Q.dropout_forward(torch.ones_like(t), module.p, tuple(model.drawn[name])) != 0).to(t.dtype)
        return t * keep / (1 - module.p)

    def norm(v, w):
        return v / (v.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w

    x = masked(model.dropout, x, "dropout")
    residual = torch.zeros_like(x)
    for i, block in enumerate(model.blocks):
        residual = x + residual
        y = norm(residual, params[f"blocks.{i}.norm.weight"])
        v, z = (y @ params[f"blocks.{i}.split.weight"].t()).chunk(2, -1)
        a, h, hs = torch.sigmoid(z), torch.zeros_like(v[:, 0]), []
        for t in range(v.shape[1]):
            h = a[:, t] * h + (1 - a[:, t]) * v[:, t]
            hs.append(h)
        x = torch.stack(hs, 1) @ params[f"blocks.{i}.join.weight"].t()
        x = masked(block.dropout, x, f"blocks.{i}.dropout")
    at = (torch.arange(len(tokens), device=tokens.device), lengths - 1)
    s = norm(x[at] + residual[at], params["norm.weight"])
    return model.decode(model.node(s @ params["encode.weight"].t()))


def test_gradients_of_the_whole(example):
    """float64: every parameter's gradient against the same network in elementary
    operations. Both round in float64 along some 10^3 operations of magnitudes up to
    10^2 between a parameter and the loss; 1e-9 of a gradient's size leaves room."""
    torch.manual_seed(4)
    model = example.SequenceClassifier(50, 3, features=12, qubits=4, dtype="c128")
    tokens, lengths, label = example.samples(6, 21, 50, 3)
    lengths[1] = 1
    model.drawn = {n: (int(m.key[0]), int(m.key[1])) for n, m in model.named_modules() if hasattr(m, "key")}
    params = dict(model.named_parameters())
    loss = torch.nn.functional.cross_entropy(model(tokens, lengths), label)
    got = torch.autograd.grad(loss, list(params.values()))
    other = torch.nn.functional.cross_entropy(plain(model, tokens, lengths, params), label)
    want = torch.autograd.grad(other, list(params.values()))
    assert (loss - other).abs() <= 1e-10
    for name, g, w in zip(params, got, want):
        assert (g - w).norm() <= 1e-9 * w.norm(), name
    assert not dict(zip(params, got))["embedding.weight"][example.PADDING].any()


def test_gradients_against_differences(example):
    """Along a random direction of all parameters, in float64."""
    torch.manual_seed(5)
    model = example.SequenceClassifier(40, 3, features=10, qubits=4, dtype="c128").eval()
    tokens, lengths, label = example.samples(5, 18, 40, 3)
    params = list(model.parameters())
    loss = lambda: torch.nn.functional.cross_entropy(model(tokens, lengths), label)  # noqa: E731
    grads = torch.autograd.grad(loss(), params)
    d = [torch.randn_like(p) / p.numel() ** 0.5 for p in params]
    eps = 1e-5
    with torch.no_grad():
        ends = []
        for sign in (1, -2):
            for p, v in zip(params, d):
                p.add_(sign * eps * v)
            ends.append(loss().item())
    slope = (ends[0] - ends[1]) / (2 * eps)
    want = sum((g * v).sum().item() for g, v in zip(grads, d))
    # eps^2 of a third derivative, and the losses' rounding over eps
    assert abs(slope - want) <= 1e-6 * max(1, abs(want))


def test_steps_give_what_the_whole_gives(example):
    """Serving: token by token with states, against the whole sequence at each length."""
    torch.manual_seed(6)
    model = example.SequenceClassifier(60, 3, features=16, qubits=4, dtype="c128").eval()
    tokens = torch.randint(1, 60, (4, 20), device="cuda")
    states = model.states(4)
    for t in range(20):
        got = model.step(tokens[:, t], states)
        with torch.no_grad():
            want = model(tokens, torch.full((4,), t + 1, device="cuda"))
        assert (got - want).abs().max() <= 1e-11 * (1 + want.abs().max())


def test_captured_step(example):
    """A serving step in a graph, replayed with eager work between, against eager steps."""
    torch.manual_seed(7)
    model = example.SequenceClassifier(60, 3, features=16, qubits=4).eval()
    blocks, norm, embedding = model.blocks, model.norm, model.embedding

    def features(token, states):
        x = embedding(token)
        residual = torch.zeros_like(x)
        for block, state in zip(blocks, states):
            x, residual = block.step(x, residual, state)
        return norm(x, residual)[0]

    token, states, eager = torch.ones(4, dtype=torch.int64, device="cuda"), model.states(4), model.states(4)
    with torch.no_grad():
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            features(token, model.states(4))
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = features(token, states)
        for t in range(5):
            token.copy_(torch.randint(1, 60, (4,), device="cuda"))
            want = features(token, eager)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want) and all(torch.equal(a, b) for a, b in zip(states, eager))
