"""The ends of the ranges that the operators' C entries take: rows of more
features and batches of more matrices than one launch's threads (2^32), and what
is refused before anything is launched."""

from __future__ import annotations

import array
import ctypes
import math

import pytest

torch = pytest.importorskip("torch")
import paper_2301_03251_amd as Q  # noqa: E402

F32, F64, BF16, F16 = 0, 1, 2, 3
gpu = pytest.mark.gpu


@pytest.fixture(scope="module")
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    Q.load()


def within(got, want, bound, what):
    off = (got.double() - want).abs_().sub_(bound)
    assert off.max().item() <= 0, f"{what}: {off.max().item():.3e} over the bound"


@gpu
@pytest.mark.parametrize("n", [(1 << 27) + 5])
def test_norm_of_very_long_rows(need_gpu, n):
    """Column sums of 2^28 columns, which take more threads than a launch has.
    The bounds are test_norm's, with the depth of a segment's sums (8 elements,
    then 256 lanes) and of the lane that joins 1/64 of the segments."""
    torch.manual_seed(0)
    x = (torch.randn(2, n, device="cuda") + 0.5).bfloat16()
    g = torch.randn(2, n, device="cuda").bfloat16()
    y, mean, rstd = Q.layer_norm_forward(x)
    gx, gw, gb = Q.layer_norm_backward(g, x, mean, rstd, weight_dtype=torch.float32)
    u, out, s = 2.0 ** -24, 1.01 * 2.0 ** -8, 80 + n / 2048 / 64
    assert gw.shape == gb.shape == (n,)
    sums = torch.zeros(2, n, dtype=torch.float64, device="cuda")
    slack = torch.zeros(n, dtype=torch.float64, device="cuda")
    size = torch.zeros(2, n, dtype=torch.float64, device="cuda")
    for row in range(2):
        xr, gr = x[row].double(), g[row].double()
        m = xr.mean()
        r = 1 / ((xr - m).square().mean() + 1e-5).sqrt()
        h = (xr - m) * r
        off = (s * u * xr.abs().max() * r + (s + 4) * u)
        dh = (1 + h.abs()) * off
        within(y[row], h, dh + out * h.abs(), "y")
        c1, c2 = gr.mean(), (gr * h).mean()
        want = r * (gr - c1 - h * c2)
        e1, e2 = (s + 2) * u * gr.abs().mean(), (s + 4) * u * (gr * h).abs().mean() + (gr.abs() * dh).mean()
        bound = r * (4 * u * (gr.abs() + c1.abs() + (h * c2).abs()) + e1 + h.abs() * e2 + c2.abs() * dh)
        within(gx[row], want, bound + want.abs() * (2 * off + out), "grad_x")
        sums[0] += gr * h
        sums[1] += gr
        slack += gr.abs() * dh
        size[0] += (gr * h).abs()
        size[1] += gr.abs()
    within(gw, sums[0], slack + 8 * u * size[0], "grad_weight")
    within(gb, sums[1], 8 * u * size[1], "grad_bias")
