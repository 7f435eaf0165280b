"""The operators together: a hybrid network trained with the norm in front of its
quantum layer and orthogonalised updates of its matrices (needs an MI355X)."""

from __future__ import annotations

import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("train_hybrid", os.path.join(ROOT, "examples", "train_hybrid.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("dtype,qubits,batch", [("c64", 10, 128), ("c128", 4, 64)])
def test_trains(example, dtype, qubits, batch):
    """Four classes far apart: chance is a loss of log 4 = 1.39 and an accuracy of 0.25."""
    losses, accuracy = example.train(steps=60, qubits=qubits, batch=batch, dtype=dtype, log=lambda *_: None)
    assert all(v == v for v in losses)
    assert sum(losses[-5:]) / 5 < 0.7 * losses[0]
    assert accuracy > 0.6


def test_same_run_again(example):
    """Every operator sums in a fixed order: two runs agree bit by bit."""
    runs = [example.train(steps=8, qubits=6, batch=64, log=lambda *_: None)[0] for _ in range(2)]
    assert runs[0] == runs[1]
