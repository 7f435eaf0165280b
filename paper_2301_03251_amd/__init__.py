"""Batched quantum-layer simulation on MI355X (gfx950): forward <Z_i> and adjoint
VJP gradients of parameterised circuits, in hand-written HIP kernels behind a
C ABI (``include/qlayer.h``). See ``qlayer.py`` for the Python binding,
``norm.py`` and ``muon.py`` for the operators around a quantum layer, ``rms.py``,
``drop.py``, ``tokens.py`` and ``scan.py`` for those of a network that reads sequences in front of it."""

from .qlayer import (C64, C128, MODE_FWD, MODE_FWD_BWD, MODE_FWD_BWD_KEEP, STATIC_SCRATCH_BYTES, Circuit, QLError, Runner,  # noqa: F401
                     sample, sample_workspace_bytes,
                     load, quantum_layer_function, QuantumLayer)
from .drop import Dropout, dropout, dropout_forward  # noqa: F401
from .muon import Muon, muon_step, orthogonalize  # noqa: F401
from .norm import LayerNorm, layer_norm, layer_norm_backward, layer_norm_forward  # noqa: F401
from .rms import RMSNorm, rms_norm, rms_norm_backward, rms_norm_forward, rms_norm_quantized  # noqa: F401
from .scan import gated_scan, gated_scan_backward, gated_scan_forward, gated_scan_step  # noqa: F401
from .tokens import Embedding, embedding, embedding_backward, embedding_forward  # noqa: F401

__all__ = ["C64", "C128", "MODE_FWD", "MODE_FWD_BWD", "MODE_FWD_BWD_KEEP", "STATIC_SCRATCH_BYTES", "Circuit", "QLError", "Runner", "load", "sample", "sample_workspace_bytes",
           "quantum_layer_function", "QuantumLayer", "LayerNorm", "layer_norm", "layer_norm_backward",
           "layer_norm_forward", "Muon", "muon_step", "orthogonalize", "RMSNorm", "rms_norm", "rms_norm_backward",
           "rms_norm_forward", "rms_norm_quantized", "Dropout", "dropout", "dropout_forward",
           "Embedding", "embedding", "embedding_backward", "embedding_forward",
           "gated_scan", "gated_scan_backward", "gated_scan_forward", "gated_scan_step"]
