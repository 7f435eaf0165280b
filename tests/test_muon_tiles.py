"""Every tile size and split that orthogonalised updates come to. On the CPU: the
calls below reach all of them (the plan is compiled alone, with sanitizers). On
an MI355X: their results, in every type, order of the arrays and with a momentum.
"""

from __future__ import annotations

import math
import os
import re
import shutil
import subprocess

import pytest

torch = pytest.importorskip("torch")
import paper_2301_03251_amd as Q  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HERE = os.path.join(ROOT, "tests", "sanitize")
CSRC = os.path.join(ROOT, "paper_2301_03251_amd", "csrc")
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
OUT_U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
COEF = (3.4445, -4.7750, 2.0315)
EPS = 1e-7
gpu = pytest.mark.gpu

# (batch, rows, cols) of a call's entries
CALLS = {
    "64": [(1, 301, 499)],
    "64, Gram product split": [(1, 64, 9000)],
    "Gram 128": [(184, 66, 1046)],
    "Gram 128 split": [(87, 4966, 66)],
    "Gram and polynomial 192": [(35, 521, 537)],
    "Gram 256": [(84, 450, 388)],
    "polynomial 128": [(158, 193, 218)],
    "polynomial 256": [(79, 455, 459)],
    "apply 128": [(193, 207, 66)],
    "apply 192": [(68, 129, 519)],
    "apply 256": [(105, 194, 397)],
    "one large": [(1, 3001, 2111)],
    "small ones beside": [(1, 1501, 1499), (3, 30, 6), (2, 9, 901), (1, 1, 77), (5, 64, 64)],
}


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_every_tile_size_is_reached(tmp_path):
    exe = str(tmp_path / "ortho_driver")
    subprocess.run(["g++", "-std=c++17", "-g", "-O1", "-Wall", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    "-D__HIP_PLATFORM_AMD__", "-isystem", "/opt/rocm/include", f"-I{os.path.join(ROOT, 'include')}", f"-I{CSRC}",
                    os.path.join(HERE, "ortho_driver.cpp"), os.path.join(CSRC, "ortho_plan.cpp"), "-o", exe], check=True)

    def plan(*calls):
        text = "".join(f"{t} " + " ".join(f"{r} {c} {b}" for b, r, c in call) + "\n" for t, call in calls)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, timeout=100)
        assert out.returncode == 0, out.stderr[-2000:]
        return out.stdout.splitlines()

    seen = set()
    for line in plan(*((0, c) for c in CALLS.values())):
        for g, splits, p, a in re.findall(r"gram (\d+) splits (\d+) bytes \d+ poly (\d+) apply (\d+)", line):
            seen |= {("gram", int(g), int(splits) > 1), ("poly", int(p)), ("apply", int(a))}
    assert seen == {("gram", t, False) for t in (64, 128, 192, 256)} | {("gram", t, True) for t in (64, 128)} | {
        (m, t) for m in ("poly", "apply") for t in (64, 128, 192, 256)}
    # the ends of the ranges: nothing overflows, and what is too much is refused
    assert plan((0, [(1, 65536, 65536)]), (1, [(3, 65536, 1)]), (2, [((1 << 31) // 3, 1, 1)]), (0, [((1 << 23) - 1, 2, 65)] * 2),
                (3, [(0, 9, 9)] * 60), (0, [(1, 65, 65)] * 60))[2:] == [
        "small workspace 0", plan((0, [((1 << 23) - 1, 2, 65)] * 2))[0], "small workspace 0", plan((0, [(1, 65, 65)] * 60))[0]]
    assert plan((0, [(1 << 21, 65, 65)])) == ["refused"]

    # a long side beside a large matrix keeps the Gram products to the tiles that fold their sums; a short one does not
    gram = [int(re.search(r"gram (\d+)", line)[1]) for line in plan(*((0, [(1, 4096, 4096), *also]) for also in (
        (), ((1, 6, 30),), ((1, 100, 512),), ((1, 12, 5992),), ((2, 700, 100),))))]
    assert gram[0] > 128 and gram[1] == gram[2] == gram[0] and gram[3] <= 128 and gram[4] <= 128


# ---------------------------------------------------------------------------
# results

@pytest.fixture(scope="module")
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    Q.load()


def held(v, size):
    s = 2.0 ** 14 / size
    hi = (v * s).half().double()
    return (hi + (v * s - hi).half().double()) / s


def steps_of(u, hold=lambda v, size: v, product=torch.bmm):
    """The formulas of a batch u, in torch's float64 on the GPU."""
    if u.shape[-2] > u.shape[-1]:
        return steps_of(u.mT.contiguous(), hold, product).mT.contiguous()
    a, b, c = COEF
    x = hold(u / (u.square().sum((-2, -1), keepdim=True).sqrt() + EPS), 1.0)
    for _ in range(5):
        g = hold(product(x, x.mT.contiguous()), 1.0)
        x = hold(a * x + product(hold(b * g + c * product(g, g), 4.0), x), 1.0)
    return x


def bounds(u, dtype):
    """(exact, bound of each matrix's norm of the difference): as in
    test_muon_precision, the model's products in torch's float32."""
    want = steps_of(u)
    off = steps_of(u, held, lambda p, q: torch.bmm(p.float(), q.float()).double()) - want
    norm = lambda t: torch.linalg.matrix_norm(t)  # noqa: E731
    return want, 3 * norm(off) + 2e-6 * norm(want) + 1.1 * norm(want.to(dtype).double() - want)


def update(shape, dtype, seed):
    r = torch.Generator(device="cuda").manual_seed(seed)
    u = torch.randn(shape, generator=r, device="cuda")
    u *= (1 + torch.randperm(shape[-1], generator=r, device="cuda")).rsqrt()
    return (0.03 * u).to(dtype)


def ordered(t, order):
    """t's values in rows, in columns, or spaced in both directions (with NaN between)."""
    if order == "rows":
        return t.contiguous()
    if order == "columns":
        return t.mT.contiguous().mT
    wide = torch.full((t.shape[0], 2 * t.shape[1], 3 * t.shape[2] + 1), float("nan"), dtype=t.dtype, device=t.device)
    v = wide[:, 1::2, 1::3]
    return v.copy_(t)


@gpu
@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("call", list(CALLS))
def test_values(need_gpu, call, name):
    """Updates in rows and in columns, results likewise; the step with a momentum,
    whose weights, gradients and momenta all lie in different orders."""
    dtype = TYPES[name]
    us = [update(s, dtype, k) for k, s in enumerate(CALLS[call])]
    limits = [bounds(u.double(), dtype) for u in us]
    if len(us) == 1:
        (want, bound), u = limits[0], us[0]
        for g, o in (("rows", "rows"), ("columns", "rows"), ("rows", "columns")):
            out = ordered(torch.zeros_like(u), o)
            assert Q.orthogonalize(ordered(u, g), out=out) is out
            assert (torch.linalg.matrix_norm(out.double() - want) <= bound).all(), (g, o)
    doubled = [bounds(2 * u.double(), dtype) for u in us]
    for p_, g_, m_ in (("rows", "columns", "rows"), ("columns", "rows", "spaced"), ("spaced", "spaced", "columns")):
        # m = 0.5 m0 + g with m0 = 2 g, so m = 2 g, and the update is g + 0.5 m = 2 g, exactly
        p = [ordered(torch.zeros_like(u), p_) for u in us]
        m = [ordered(2 * u.float(), m_) for u in us]
        Q.muon_step(p, [ordered(u, g_) for u in us], m, lr=1.0, momentum=0.5)
        for t, u, v, (want, bound) in zip(m, us, p, doubled):
            assert torch.equal(t, 2 * u.float())
            grow = math.sqrt(max(1.0, u.shape[1] / u.shape[2]))
            off = torch.linalg.matrix_norm(-v.double() / grow - want)
            # the rounding is that of the result times grow: at most half a unit of each value
            assert (off <= bound + OUT_U[name] * torch.linalg.matrix_norm(want)).all(), (p_, g_, m_)
