"""Arguments of the sequence operators whose memory is not what it looks like, and
numbers that their arithmetic cannot hold."""

from __future__ import annotations

import ctypes

import pytest

torch = pytest.importorskip("torch")
import paper_2301_03251_amd as Q  # noqa: E402

F32, F64, BF16, F16 = 0, 1, 2, 3
FAKE = ctypes.c_void_p(0x1000)


def _scaled(lib, type_, scale):
    """(code of the forward entry, of the backward entry) of no tokens: nothing is launched by the first."""
    fwd = lib.ql_embedding_forward(type_, 1, 0, 5, 4, None, None, 4, scale, 0, 0, None, None)
    bwd = lib.ql_embedding_backward(type_, 1, 3, 5, 4, FAKE, FAKE, 4, scale, 0, 0, FAKE, None, 0, None)
    return fwd, bwd, lib.ql_last_error().decode()


def test_embedding_scales_past_the_arithmetic_are_refused():
    """float32 holds no 1e39: rows of zeros times what it becomes would be NaN."""
    lib = Q.load()
    for t in (F32, BF16, F16):
        for scale in (1e39, -1e39, 3.5e38):
            fwd, bwd, message = _scaled(lib, t, scale)
            assert (fwd, bwd) == (-1, -1) and "scale" in message
        # the backward call then stops at its missing workspace
        fwd, bwd, message = _scaled(lib, t, 3.4e38)
        assert (fwd, bwd) == (0, -1) and "workspace" in message
    fwd, bwd, message = _scaled(lib, F64, 1e300)
    assert (fwd, bwd) == (0, -1) and "workspace" in message
