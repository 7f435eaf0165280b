"""Batched quantum-layer simulation on MI355X (gfx950): forward <Z_i> and adjoint
VJP gradients of parameterised circuits, in hand-written HIP kernels behind a
C ABI (``include/qlayer.h``). See ``qlayer.py`` for the Python binding,
``norm.py`` and ``muon.py`` for the operators around a quantum layer."""

from .qlayer import (C64, C128, MODE_FWD, MODE_FWD_BWD, MODE_FWD_BWD_KEEP, STATIC_SCRATCH_BYTES, Circuit, QLError, Runner,  # noqa: F401
                     sample, sample_workspace_bytes,
                     load, quantum_layer_function, QuantumLayer)
from .muon import Muon, muon_step, orthogonalize  # noqa: F401
from .norm import LayerNorm, layer_norm, layer_norm_backward, layer_norm_forward  # noqa: F401

__all__ = ["C64", "C128", "MODE_FWD", "MODE_FWD_BWD", "MODE_FWD_BWD_KEEP", "STATIC_SCRATCH_BYTES", "Circuit", "QLError", "Runner", "load", "sample", "sample_workspace_bytes",
           "quantum_layer_function", "QuantumLayer", "LayerNorm", "layer_norm", "layer_norm_backward",
           "layer_norm_forward", "Muon", "muon_step", "orthogonalize"]
