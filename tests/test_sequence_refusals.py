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


@pytest.fixture
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    Q.load()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.int64, torch.int32])
def test_negative_views_of_tokens(need_gpu, dtype):
    t = torch.randint(1, 20, (50,), device="cuda", dtype=dtype)
    w, g = torch.randn(20, 12, device="cuda"), torch.randn(50, 12, device="cuda")
    view = torch._neg_view(-t)
    assert torch.equal(view, t)
    assert torch.equal(Q.embedding_forward(view, w), Q.embedding_forward(t, w))
    assert torch.equal(Q.embedding_backward(g, view, 20), Q.embedding_backward(g, t, 20))


@pytest.mark.gpu
def test_negative_views_of_what_must_be_contiguous(need_gpu):
    """A key, the norms' statistics and the recurrence's states are read as they lie: refused."""
    x, g = torch.randn(6, 40, device="cuda"), torch.randn(6, 40, device="cuda")
    with pytest.raises(ValueError, match="key"):
        Q.dropout(x, 0.5, torch._neg_view(torch.tensor([5, 9], device="cuda")))
    _, s, r = Q.rms_norm_forward(x)
    with pytest.raises(ValueError, match="rstd"):
        Q.rms_norm_backward(g, s, torch._neg_view(-r))
    _, mean, rstd = Q.layer_norm_forward(x)
    for a, b in ((torch._neg_view(-mean), rstd), (mean, torch._neg_view(-rstd))):
        with pytest.raises(ValueError, match="rstd"):
            Q.layer_norm_backward(g, x, a, b)
    x, z, g = torch.randn(3, 2, 40, 8, device="cuda").unbind(0)
    _, _, states = Q.gated_scan_forward(x, z)
    with pytest.raises(ValueError, match="states"):
        Q.gated_scan_backward(g, x, z, torch._neg_view(-states))
