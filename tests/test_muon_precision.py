"""How far orthogonalised updates are from the formulas in 64 bits (needs an MI355X).

The bound is relative and in the Frobenius norm. A model of the rounding runs on
the CPU on the same inputs: the formulas with X, A and B held in 22 bits (two
fp16 parts) between products of 32-bit sums. A kernel, whose sums run in another
order, may be three times as far off as the model, plus 2e-6 of the result (with
few rows single roundings do not average out), plus the rounding of the output:
that of the exact result to its type, which a value so near to it repeats but for
ties that fall the other way (a tenth more).
"""

from __future__ import annotations

import math

import pytest

torch = pytest.importorskip("torch")
import paper_2301_03251_amd as Q  # noqa: E402

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
COEF = (3.4445, -4.7750, 2.0315)
EPS = 1e-7
gpu = pytest.mark.gpu


@pytest.fixture(scope="module")
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    Q.load()


def held(v, size):
    s = 2.0 ** 14 / size
    hi = (v * s).half().double()
    return (hi + (v * s - hi).half().double()) / s


def exact(u, steps=5, eps=EPS):
    return _steps(u, steps, eps, lambda v, size: v, torch.matmul)


def model(u, steps=5, eps=EPS):
    return _steps(u, steps, eps, held, lambda a, b: torch.matmul(a.float(), b.float()).double())


def _steps(u, steps, eps, hold, product):
    if u.shape[0] > u.shape[1]:
        return _steps(u.T.contiguous(), steps, eps, hold, product).T
    a, b, c = COEF
    x = hold(u / (u.norm() + eps), 1.0)
    for _ in range(steps):
        g = hold(product(x, x.T.contiguous()), 1.0)
        x = hold(a * x + product(hold(b * g + c * product(g, g), 4.0), x), 1.0)
    return x


def update(rows, cols, kind, dtype, seed):
    """An update as weights get them: noise; rows and columns of decaying scale; a
    few directions with little beside them, which the steps raise by 3.4 each."""
    r = torch.Generator().manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=r, dtype=torch.float64)  # noqa: E731
    u = normal(rows, cols)
    if kind == "decaying":
        u *= (1 + torch.randperm(cols, generator=r)).double().rsqrt()
        u *= (1 + torch.randperm(rows, generator=r)).double().rsqrt()[:, None]
    elif kind == "few directions":
        few = max(1, min(rows, cols) // 16)
        u = normal(rows, few) @ normal(few, cols) + 1e-3 * u
    return (0.03 * u).to(dtype)


def near(got, u, dtype, what, sign=1.0):
    u = u.double()
    want = exact(u)
    size = want.norm().item()
    rounding = (want.to(dtype).double() - want).norm().item()
    bound = 3 * (model(u) - want).norm().item() + 2e-6 * size + 1.1 * rounding
    off = (sign * got.cpu().double() - want).norm().item()
    assert off <= bound, f"{what}: {off / size:.3e} of the result, bound {bound / size:.3e}, rounding {rounding / size:.3e}"


KINDS = ["noise", "decaying", "few directions"]


@gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("rows,cols", [(2, 50), (8, 32), (72, 20), (64, 256), (500, 63), (33, 410), (3, 3000), (65, 65),
                                       (100, 130), (200, 129), (300, 500), (900, 600), (64, 9000)])
def test_orthogonalize(need_gpu, rows, cols, name, kind):
    u = update(rows, cols, kind, TYPES[name], seed=rows * 1000 + cols)
    near(Q.orthogonalize(u.cuda()), u, TYPES[name], f"{rows}x{cols} {kind}")


@gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("name", list(TYPES))
def test_a_matrix_beside_a_large_one(need_gpu, name, kind):
    """Few rows and small matrices are as near in a call with much work as by themselves."""
    shapes = [(1500, 1500), (12, 5992), (64, 16), (2, 50), (6, 30)]
    u = [update(*s, kind, TYPES[name], seed=k) for k, s in enumerate(shapes)]
    p = [torch.zeros(s, dtype=TYPES[name], device="cuda") for s in shapes]
    m = [torch.zeros(s, device="cuda") for s in shapes]
    # out = -lr sqrt(max(1, rows / cols)) O, with the factor 1 or (64x16) 2
    Q.muon_step(p, [t.cuda() for t in u], m, lr=1.0, momentum=0.0)
    for q, t, (rows, cols) in zip(p, u, shapes):
        near(q, t, TYPES[name], f"{rows}x{cols} {kind}", sign=-1 / math.sqrt(max(1.0, rows / cols)))


@gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("beside,batch", [((4096, 4096), 1), ((20, 30), 600)])
@pytest.mark.parametrize("rows,cols", [(12, 5992), (3000, 65)])
def test_long_sums_of_few_rows(need_gpu, rows, cols, beside, batch, kind):
    """However many tiles the rest of a call gives the chip, so that no sum is split."""
    u = torch.stack([update(rows, cols, kind, torch.float32, seed=k % 3) for k in range(batch)]).cuda()
    other = update(*beside, kind, torch.float32, seed=9).cuda()
    p = [torch.zeros_like(u), torch.zeros_like(other)]
    m = [torch.zeros_like(t) for t in p]
    Q.muon_step(p, [u, other], m, lr=1.0, momentum=0.0)
    grow = math.sqrt(max(1.0, rows / cols))
    for k in (0, batch // 2, batch - 1):
        near(p[0][k], u[k].cpu(), torch.float32, f"{rows}x{cols} {kind}, matrix {k}", sign=-1 / grow)


def low_model(u, steps, coef, eps):
    """The model with X held as finely below 1 as at 1: at its own norm's bound,
    which no step raises by more than the polynomial's largest slope from 0."""
    if u.shape[0] > u.shape[1]:
        return low_model(u.T.contiguous(), steps, coef, eps).T
    a, b, c = coef
    product = lambda p, q: torch.matmul((p * 2.0 ** 40).float(), q.float()).double() * 2.0 ** -40  # noqa: E731
    size = min(1.0, (u.norm() / (u.norm() + eps)).item())
    x = held(u / (u.norm() + eps), size)
    for _ in range(steps):
        x1 = x / size
        g = held(product(x1, x1.T.contiguous()) * size * size, 1.0)
        grown = min(1.0, size * a)
        x = held(a * x + product(held(b * g + c * product(g, g), 4.0), x1) * size, grown)
        size = grown
    return x


@gpu
@pytest.mark.parametrize("steps,coef", [(5, COEF), (1, COEF), (64, (1.5, -0.5, 0.0))])
@pytest.mark.parametrize("norm", [1e-5, 1e-7, 3e-10, 1e-12, 1e-15, 3e-17, 1e-20, 1e-30])
@pytest.mark.parametrize("name,rows,cols", [("f32", 12, 30), ("bf16", 40, 30), ("f32", 100, 130), ("f32", 500, 300), ("f32", 40, 3000)])
def test_updates_far_below_eps(need_gpu, name, rows, cols, norm, steps, coef):
    """X = U / (|U| + eps) is then small, and so is the result: no fewer of its
    bits are right for that."""
    u = update(rows, cols, "noise", torch.float64, seed=rows)
    u = (u * (norm / u.norm())).to(TYPES[name])
    got = Q.orthogonalize(u.cuda(), steps, coef).cpu().double()
    d = u.double()
    want = d if rows <= cols else d.T
    want = want / (d.norm() + EPS)
    for _ in range(steps):
        g = want @ want.T
        want = coef[0] * want + (coef[1] * g + coef[2] * g @ g) @ want
    want = want if rows <= cols else want.T
    size = want.norm().item()
    bound = (3 * (low_model(d, steps, coef, EPS) - want).norm().item() + 2e-6 * size
             + 1.1 * (want.to(TYPES[name]).double() - want).norm().item())
    off = (got - want).norm().item()
    assert off <= bound, f"{off / size:.3e} of the result, bound {bound / size:.3e}"
