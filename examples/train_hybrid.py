"""Training of a small hybrid network with the library's operators.

    features -> Linear -> LayerNorm -> QuantumLayer -> Linear -> classes

The norm brings the first layer's outputs to the range of the encoding's angles
(a weight of pi / 4, a bias of pi / 2), and its backward takes the quantum
layer's input gradients on. The matrices are stepped by Muon, the quantum
layer's angles among them as [layers, angles of a layer]; vectors by SGD.
Synthetic data: noisy samples around one centre for each class.

    python examples/train_hybrid.py [--steps 60] [--qubits 10] [--batch 256]
"""

from __future__ import annotations

import argparse
import math
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2301_03251_amd as Q  # noqa: E402
import workloads as W  # noqa: E402


class Hybrid(torch.nn.Module):
    def __init__(self, features, classes, qubits=10, layers=3, dtype="c64", device="cuda"):
        super().__init__()
        real = torch.float32 if dtype == "c64" else torch.float64
        self.encode = torch.nn.Linear(features, qubits, bias=False, device=device, dtype=real)
        self.norm = Q.LayerNorm(qubits, dtype=real, device=device)
        with torch.no_grad():
            self.norm.weight.fill_(math.pi / 4)
            self.norm.bias.fill_(math.pi / 2)
        gates = W.layered_circuit(qubits, "ry", layers, (W.RY, W.RZ), W.CNOT, "ring")
        self.angles = (layers, 2 * qubits)
        self.node = Q.QuantumLayer(gates, qubits, qubits, layers * 2 * qubits, dtype=dtype, device=device,
                                   weights=0.3 * torch.randn(layers * 2 * qubits, dtype=torch.float64))
        self.decode = torch.nn.Linear(qubits, classes, device=device, dtype=real)

    def forward(self, x):
        return self.decode(self.node(self.norm(self.encode(x))))

    def optimizers(self, lr=0.05):
        muon = Q.Muon([{"params": [self.encode.weight, self.decode.weight]},
                       {"params": [self.node.weights], "matrix": self.angles}], lr=lr, momentum=0.9)
        vectors = torch.optim.SGD([self.norm.weight, self.norm.bias, self.decode.bias], lr=lr, momentum=0.9)
        return muon, vectors


def samples(batch, features, classes, centres, real):
    label = torch.randint(classes, (batch,), device=centres.device)
    return (centres[label] + 0.7 * torch.randn(batch, features, device=centres.device)).to(real), label


def train(steps=60, qubits=10, batch=256, features=64, classes=4, dtype="c64", seed=0, log=print):
    """(losses of all steps, accuracy on a last batch)."""
    torch.manual_seed(seed)
    model = Hybrid(features, classes, qubits, dtype=dtype)
    optimizers = model.optimizers()
    centres = torch.randn(classes, features, device="cuda")
    real = model.decode.weight.dtype
    losses = []
    for step in range(steps):
        x, label = samples(batch, features, classes, centres, real)
        loss = torch.nn.functional.cross_entropy(model(x), label)
        for o in optimizers:
            o.zero_grad()
        loss.backward()
        for o in optimizers:
            o.step()
        losses.append(loss.item())
        if step % 10 == 0 or step + 1 == steps:
            log(f"step {step:4d}  loss {losses[-1]:.4f}")
    with torch.no_grad():
        x, label = samples(1024, features, classes, centres, real)
        accuracy = (model(x).argmax(1) == label).double().mean().item()
    return losses, accuracy


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--qubits", type=int, default=10)
    ap.add_argument("--batch", type=int, default=256)
    ap.add_argument("--dtype", choices=("c64", "c128"), default="c64")
    a = ap.parse_args()
    began = time.perf_counter()
    losses, accuracy = train(a.steps, a.qubits, a.batch, dtype=a.dtype)
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f}, accuracy {accuracy:.3f}, "
          f"{(time.perf_counter() - began) / a.steps * 1e3:.2f} ms a step")


if __name__ == "__main__":
    main()
