"""Rows in 8 bits at the borders of their rounding and of the range (needs an MI355X).

The definition in 64 bits: p = s w (48 bits, exact there), q = p 448 / max |p| rounded
to e4m3, scale = rstd max |p| / 448.
"""

from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")
import paper_2301_03251_amd as Q  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6
U = 2.0 ** -24
# 16 lanes, a wavefront, a workgroup, and past a workgroup's registers
SIZES = [24, 700, 5000, 40000]


@pytest.fixture(scope="module", autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    Q.load()


def steps_of(v):
    """|v| in steps of e4m3 around it: three bits behind the leading one, 2^-9 at least."""
    e = torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6)))
    return v.abs() / torch.exp2(e - 3), torch.exp2(e - 3)


def e4m3(v):
    """v (float64) to e4m3, to nearest, halves to even."""
    n, step = steps_of(v)
    return torch.round(n) * step * torch.sign(v)


def halves(v):
    n, _ = steps_of(v)
    return n - n.floor() == 0.5


def definition(s, w, eps=EPS):
    """(p 448 / max |p|, rstd max |p| / 448), a row of zeros giving zeros."""
    s = s.double()
    p = s if w is None else s * w.double()
    most = p.abs().amax(-1, keepdim=True)
    rstd = 1 / torch.sqrt(s.square().mean(-1) + eps)
    q = torch.where(most > 0, p * 448 / torch.where(most > 0, most, 1), torch.zeros_like(p))
    return q, torch.where(most[..., 0] > 0, rstd * most[..., 0] / 448, torch.zeros_like(rstd))


def check(s, w, q, scale, eps=EPS):
    """q is the definition's value before its rounding to e4m3 times 1 to 1 + 4 u (a factor
    up to 3 u up, and a rounding), u for p, and up to 2^-21 = 8 u less where two bits go. rstd is off by (depth / 2 + 6) u (a sum of squares of depth 80 + n / 1024), the
    scale by 4 u more and half a step where it ends below the normal range."""
    want, wide = definition(s, w, eps)
    ends = [e4m3((want * (1 + k * U)).float().double()) for k in (-9.1, 5.1)]
    got = q.double()
    assert (got >= torch.minimum(*ends)).all() and (got <= torch.maximum(*ends)).all()
    rr = ((80 + s.shape[-1] / 1024) / 2 + 10) * U
    assert ((scale.double() - wide).abs() <= wide * rr + 2.0 ** -150 * 1.01).all()


@pytest.mark.parametrize("weight,residual", [(True, True), (False, False)])
@pytest.mark.parametrize("n", SIZES)
def test_halves_of_bfloat16_go_to_the_even_value(n, weight, residual):
    """bfloat16 rows and weights: p has 16 bits and p 448 has 19, so a quotient in 24 bits
    that is no half of two e4m3 values is at least 2^-21 of itself away from one:
    every value is the definition's, the halves among them too."""
    g = torch.Generator().manual_seed(n)
    rows = 512 if n < 10000 else 24
    x = (torch.randn(rows, n, generator=g) * (0.5 + 2 * torch.rand(n, generator=g))).bfloat16().cuda()
    w = (1 + 0.2 * torch.randn(n, generator=g)).bfloat16().cuda() if weight else None
    res = torch.randn(rows, n, generator=g).bfloat16().cuda() if residual else None
    q, scale, s = Q.rms_norm_quantized(x, w, res, EPS)
    want, _ = definition(s, w)
    assert halves(want).any()
    assert torch.equal(q.double(), e4m3(want))
    check(s, w, q, scale)


@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("n", SIZES)
def test_halves_of_all_types_go_to_the_even_value(n, name):
    """Rows whose largest value is 448 c, c odd, with elements c times a half of two e4m3
    values: integers of at most 16 bits in float32, c = 1, 3, 5 and 7 in 16-bit types."""
    g = torch.Generator().manual_seed(n)
    cs = torch.tensor([1, 3, 5, 7] if name != "f32" else [1, 3, 5, 7, 11, 49, 85, 93, 101, 127])
    rows = 40
    c = cs[torch.arange(rows) % len(cs)][:, None].double()
    # 2 k + 1 sixteenths of a power of two, 8 <= k < 16: halves; those that bfloat16 holds when times 3, 5, 7
    h = (2 * torch.randint(8, 16, (rows, n), generator=g) + 1).double() * torch.exp2(torch.randint(-2, 3, (rows, n), generator=g).double())
    s = h * c * torch.where(torch.rand(rows, n, generator=g) < 0.5, 1.0, -1.0)
    s[:, n // 2] = 448 * c[:, 0]
    x = s.to(TYPES[name]).cuda()
    q, scale, _ = Q.rms_norm_quantized(x)
    want, _ = definition(x, None)
    exact = halves(want)
    assert exact.double().mean() > 0.5
    assert torch.equal(q.double()[exact], e4m3(want)[exact])
    check(x, None, q, scale)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("n", SIZES)
def test_large_rows_under_small_weights(n, name):
    """Weights of 0 and far below 1: no infinity comes up between the row and its quotient."""
    g = torch.Generator().manual_seed(n)
    base = torch.randn(6, n, generator=g, dtype=torch.float64)
    for size, weight in ((1e9, 0.0), (1e18, 0.0), (1e10, 1e-38), (1e15, 1e-38), (1e-30, 1e-6)):
        x = (base * size).to(TYPES[name]).cuda()
        w = (weight * (1 + 0.2 * torch.randn(n, generator=g, dtype=torch.float64))).to(TYPES[name]).cuda()
        q, scale, s = Q.rms_norm_quantized(x, w)
        assert torch.isfinite(q.float()).all() and torch.isfinite(scale).all(), (size, weight)
        check(s, w, q, scale)
    # one large value under a weight of 0, the others small
    x = (base * 1e-20).to(TYPES[name]).cuda()
    w = torch.full((n,), 1e-15, dtype=TYPES[name], device="cuda")
    x[:, n // 3], w[n // 3] = 1e18, 0
    q, scale, s = Q.rms_norm_quantized(x, w)
    check(s, w, q, scale)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("n", SIZES)
def test_products_far_from_one(n, name):
    """Products s w that float32 does not hold, or not in all bits, where y and its scale are ordinary."""
    g = torch.Generator().manual_seed(n)
    base = torch.randn(6, n, generator=g, dtype=torch.float64)
    for size, weight in ((1e10, 1e-40), (1e10, 1e30), (1e-30, 1e-10), (1e-20, 1e-20), (1e-20, 1e25)):
        x = (base * size).to(TYPES[name]).cuda()
        w = (weight * (1 + 0.2 * torch.randn(n, generator=g, dtype=torch.float64))).to(TYPES[name]).cuda()
        q, scale, s = Q.rms_norm_quantized(x, w)
        assert torch.isfinite(q.float()).all() and torch.isfinite(scale).all(), (size, weight)
        check(s, w, q, scale)


@pytest.mark.parametrize("n", SIZES)
def test_scales_below_the_normal_range(n):
    """Rows of 1e-39 and 1e-41 keep what bits their scale has."""
    x = torch.randn(4, n, generator=torch.Generator().manual_seed(n), dtype=torch.float64)
    x = (x * torch.tensor([[1e-37], [1e-39], [1e-41], [1e-30]])).float().cuda()
    q, scale, s = Q.rms_norm_quantized(x)
    check(s, None, q, scale)


@pytest.mark.parametrize("n", SIZES)
def test_rows_of_zeros_without_eps(n):
    """1 / 0 does not reach the scale, and the rows beside them are as ever."""
    x = torch.randn(5, n, generator=torch.Generator().manual_seed(n)).cuda()
    x[1] = x[4] = 0
    for w in (None, torch.ones(n, device="cuda")):
        q, scale, s = Q.rms_norm_quantized(x, w, eps=0.0)
        assert not scale[[1, 4]].any() and not q[[1, 4]].float().any()
        rest = [0, 2, 3]
        check(s[rest], w, q[rest], scale[rest], 0.0)


@pytest.mark.parametrize("n", SIZES)
def test_infinities_under_a_weight_of_zero(n):
    """The scale of a row that holds an infinity is NaN, whatever weight stands at it."""
    g = torch.Generator().manual_seed(n)
    x, w = torch.randn(4, n, generator=g).cuda(), torch.ones(n, device="cuda")
    want = Q.rms_norm_quantized(x, w)[1]
    w[n // 2] = 0
    clean = Q.rms_norm_quantized(x, w)
    x[2, n // 2] = float("inf")
    q, scale, _ = Q.rms_norm_quantized(x, w)
    assert torch.isnan(scale[2]) and torch.isfinite(want).all()
    keep = [0, 1, 3]
    assert torch.equal(scale[keep], clean[1][keep]) and torch.equal(q[keep].float(), clean[0][keep].float())
    assert torch.isnan(Q.rms_norm_quantized(x, torch.zeros_like(w))[1][2])


@pytest.mark.parametrize("name,rows,n", [("bf16", 200000, 24), ("f32", 70000, 100), ("bf16", 20000, 700), ("f16", 20000, 900), ("bf16", 9000, 3000),
                                         ("f32", 9000, 3000), ("bf16", 9000, 6000), ("bf16", 4500, 12000), ("bf16", 600, 40000)])
def test_ordinary_rows_among_others(name, rows, n):
    """More rows than are in work at once: rows of zeros, tiny ones, such with an infinity or
    NaN and ordinary ones, in any order, each as it is alone."""
    g = torch.Generator(device="cuda").manual_seed(n)
    x = torch.randn(rows, n, generator=g, device="cuda")
    kind = torch.randint(6, (rows,), generator=g, device="cuda")
    small = 6e-8 if name == "f16" else 1e-38
    x = (x * torch.where(kind == 1, small, 1.0)[:, None] * (kind != 2)[:, None]).to(TYPES[name])
    bad = torch.nonzero(kind >= 4)[:, 0]
    at = torch.randint(n, (len(bad),), generator=g, device="cuda")
    x[bad, at] = torch.where(kind[bad] == 4, float("inf"), float("nan")).to(x.dtype)
    w = (1 + 0.2 * torch.randn(n, generator=g, device="cuda")).to(TYPES[name])
    w[::7] = 0
    eps = 1e-12
    res = torch.zeros_like(x) if n % 200 == 100 or n == 6000 else None
    q, scale, s = Q.rms_norm_quantized(x, w, res, eps)
    assert torch.isnan(scale[bad]).all()
    good = torch.nonzero(kind < 4)[:, 0]
    for part in good.split(2000):
        check(s[part], w, q[part], scale[part], eps)
    assert not scale[kind == 2].any() and not q[kind == 2].float().any()
    again = Q.rms_norm_quantized(x, w, res, eps)
    assert torch.equal(again[0].view(torch.uint8), q.view(torch.uint8)) and torch.equal(again[1][good], scale[good])
