"""Training of a hybrid network on sequences of tokens with the library's operators.

    tokens -> Embedding -> Dropout -> blocks -> last step -> RMSNorm -> Linear
           -> QuantumLayer -> Linear -> classes

A block is RMSNorm with the residual's addition, a projection to x and gate, the
gated recurrence over the steps, a projection back, and dropout. Sequences of a
batch have different lengths: padded places have the padding's zeros as features,
and a sequence is read at its last own step. The matrices are stepped by Muon, the quantum
layer's angles among them; the table and the vectors by SGD. Synthetic data: each
class has tokens that it draws more often than others.

    python examples/train_sequence.py [--steps 40] [--qubits 8] [--batch 64]
"""

from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2301_03251_amd as Q  # noqa: E402
import workloads as W  # noqa: E402

PADDING = 0


class Block(torch.nn.Module):
    def __init__(self, features, dropout, device, dtype):
        super().__init__()
        self.norm = Q.RMSNorm(features, device=device, dtype=dtype)
        self.split = torch.nn.Linear(features, 2 * features, bias=False, device=device, dtype=dtype)
        self.join = torch.nn.Linear(features, features, bias=False, device=device, dtype=dtype)
        self.dropout = Q.Dropout(dropout, device=device)

    def project(self, x, residual):
        """(what the recurrence takes: x and gate, the next residual)."""
        y, residual = self.norm(x, residual)
        return (*self.split(y).chunk(2, -1), residual)

    def forward(self, x, residual):
        x, gate, residual = self.project(x, residual)
        h, _ = Q.gated_scan(x, gate)
        return self.dropout(self.join(h)), residual

    def step(self, x, residual, state):
        """One step of every sequence; its state changes in place."""
        x, gate, residual = self.project(x, residual)
        return self.join(Q.gated_scan_step(x, gate, state)), residual


class SequenceClassifier(torch.nn.Module):
    def __init__(self, vocabulary, classes, features=32, qubits=8, layers=2, blocks=2, dropout=0.1, dtype="c64", device="cuda"):
        super().__init__()
        real = torch.float32 if dtype == "c64" else torch.float64
        self.features = features
        self.embedding = Q.Embedding(vocabulary, features, scale=0.5, padding=PADDING, device=device, dtype=real)
        self.dropout = Q.Dropout(dropout, device=device)
        self.blocks = torch.nn.ModuleList(Block(features, dropout, device, real) for _ in range(blocks))
        self.norm = Q.RMSNorm(features, device=device, dtype=real)
        self.encode = torch.nn.Linear(features, qubits, bias=False, device=device, dtype=real)
        gates = W.layered_circuit(qubits, "ry", layers, (W.RY, W.RZ), W.CNOT, "ring")
        self.angles = (layers, 2 * qubits)
        self.node = Q.QuantumLayer(gates, qubits, qubits, layers * 2 * qubits, dtype=dtype, device=device,
                                   weights=0.3 * torch.randn(layers * 2 * qubits, dtype=torch.float64))
        self.decode = torch.nn.Linear(qubits, classes, device=device, dtype=real)

    def head(self, x, residual):
        """Logits of rows [batch, features]."""
        return self.decode(self.node(self.encode(self.norm(x, residual)[0])))

    def forward(self, tokens, lengths):
        x = self.dropout(self.embedding(tokens))
        residual = torch.zeros_like(x)
        for block in self.blocks:
            x, residual = block(x, residual)
        at = (torch.arange(len(tokens), device=tokens.device), lengths - 1)
        return self.head(x[at], residual[at])

    @torch.no_grad()
    def states(self, batch):
        """States before the first token, for ``step``."""
        wide = self.decode.weight.dtype
        return [torch.zeros(batch, self.features, dtype=wide, device=self.decode.weight.device) for _ in self.blocks]

    @torch.no_grad()
    def step(self, tokens, states):
        """Logits after one more token [batch] of every sequence."""
        x = self.embedding(tokens)
        residual = torch.zeros_like(x)
        for block, state in zip(self.blocks, states):
            x, residual = block.step(x, residual, state)
        return self.head(x, residual)

    def optimizers(self, lr=0.02):
        matrices = [p for b in self.blocks for p in (b.split.weight, b.join.weight)] + [self.encode.weight, self.decode.weight]
        muon = Q.Muon([{"params": matrices}, {"params": [self.node.weights], "matrix": self.angles}], lr=lr, momentum=0.9)
        others = [self.embedding.weight, self.norm.weight, self.decode.bias] + [b.norm.weight for b in self.blocks]
        return muon, torch.optim.SGD(others, lr=lr, momentum=0.9)


def samples(batch, steps, vocabulary, classes, device="cuda"):
    """(tokens [batch, steps] padded at their ends, lengths, labels)."""
    label = torch.randint(classes, (batch,), device=device)
    lengths = torch.randint(1, steps + 1, (batch,), device=device)
    lengths[0] = steps
    tokens = torch.randint(1, vocabulary, (batch, steps), device=device)
    own = 1 + (tokens - 1) // classes * classes + label[:, None]  # of the label's share of the vocabulary
    tokens = torch.where((torch.rand(batch, steps, device=device) < 0.5) & (own < vocabulary), own, tokens)
    padded = torch.arange(steps, device=device) >= lengths[:, None]
    return tokens.masked_fill_(padded, PADDING), lengths, label


def train(steps=40, qubits=8, batch=64, length=100, vocabulary=200, classes=4, dtype="c64", seed=0, log=print):
    """(the model, losses of all steps)."""
    torch.manual_seed(seed)
    model = SequenceClassifier(vocabulary, classes, qubits=qubits, dtype=dtype)
    optimizers = model.optimizers()
    losses = []
    for step in range(steps):
        tokens, lengths, label = samples(batch, length, vocabulary, classes)
        loss = torch.nn.functional.cross_entropy(model(tokens, lengths), label)
        for o in optimizers:
            o.zero_grad()
        loss.backward()
        for o in optimizers:
            o.step()
        losses.append(loss.item())
        if step % 10 == 0 or step + 1 == steps:
            log(f"step {step:4d}  loss {losses[-1]:.4f}")
    return model, losses


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--qubits", type=int, default=8)
    ap.add_argument("--batch", type=int, default=64)
    ap.add_argument("--dtype", choices=("c64", "c128"), default="c64")
    a = ap.parse_args()
    began = time.perf_counter()
    _, losses = train(a.steps, a.qubits, a.batch, dtype=a.dtype)
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f}, {(time.perf_counter() - began) / a.steps * 1e3:.2f} ms a step")


if __name__ == "__main__":
    main()
