"""Performance cases of the operators around a quantum layer: the norm in front
of its encoding and the orthogonalised update of matrix-shaped weights.

A case names one pass by plain values. ``op`` is

* ``norm``: layer norm over the last axis, forward only (inference): ``rows``
  rows of ``features``, read from a buffer whose rows are ``pad`` longer;
* ``norm_train``: the same, then its backward: gradients of x, weight and bias;
* ``orthogonalize``: ``batch`` matrices of ``rows`` x ``cols``;
* ``muon``: one optimiser step over matrices of the listed ``shapes``: momentum,
  orthogonalised update, weights (momentum and weights change in place).

``dtype`` is that of x and y, or of the matrices; ``weights`` that of the norm's
weight and bias. The momentum is float32.
"""

from __future__ import annotations

import math

import torch

own = False

DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
EPS_NORM = 1e-5
EPS_ORTHO = 1e-7
STEPS = 5
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
LR, MOMENTUM, DECAY = 0.02, 0.95, 0.1


def _norm(name, op, rows, features, dtype="float32", weights="float32", pad=0):
    return {"name": name, "op": op, "rows": rows, "features": features, "dtype": dtype, "weights": weights, "pad": pad}


def _ortho(name, batch, rows, cols, dtype="float32"):
    return {"name": name, "op": "orthogonalize", "batch": batch, "rows": rows, "cols": cols, "dtype": dtype}


def _muon(name, shapes, dtype="float32"):
    return {"name": name, "op": "muon", "shapes": shapes, "dtype": dtype}


def listed():
    return [
        # inference: 256 samples of the 10 features that a 10-qubit layer encodes
        _norm("norm 256x10", "norm", 256, 10),
        # training: a batch of 1024 samples in front of a 16-qubit layer
        _norm("norm train 1024x16", "norm_train", 1024, 16),
        # inference in half precision over some columns of a wider feature matrix, odd sizes
        _norm("norm 1037x1001 f16 strided", "norm", 1037, 1001, "float16", "float16", 7),
        # a few very long rows: whole images flattened to features
        _norm("norm train 5x50000", "norm_train", 5, 50000),
        # an ordinary layer of a network in mixed precision
        _norm("norm train 8192x1024 bf16", "norm_train", 8192, 1024, "bfloat16"),
        # the largest: a wide layer over many rows
        _norm("norm train 16384x8192 bf16", "norm_train", 16384, 8192, "bfloat16", "bfloat16"),
        # the weights of a quantum layer of 24 qubits: 20 layers of 72 angles
        _muon("muon 20x72", "20x72"),
        # a hybrid network's matrices, one step over all of them
        _muon("muon 8 matrices", "64x256,256x64,6x30,10x64,120x84,512x512,777x513,1024x256"),
        # a stack of the 256 -> 64 layers in front of quantum nodes
        _ortho("orthogonalize 16x64x256", 16, 64, 256),
        # an odd tall matrix in half precision
        _ortho("orthogonalize 1000x777 bf16", 1, 1000, 777, "bfloat16"),
        # a wide layer in single precision
        _ortho("orthogonalize 2048x8192", 1, 2048, 8192),
        # the largest: a big square layer in bfloat16
        _muon("muon 4096x4096 bf16", "4096x4096", "bfloat16"),
    ]


# Bounds of a drawn case: elements of a norm's input, multiply-adds of the
# orthogonalisation, and elements of its matrices.
MOST_NORM = 16384 * 8192
MOST_FLOPS = 1.3e12
MOST_MATRIX = 4096 * 4096


def _log(rng, low, high):
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 0.5)))))))


def draw(rng):
    op = rng.choice(("norm", "norm_train", "orthogonalize", "muon"))
    dtype = rng.choice(tuple(DTYPES))
    if op.startswith("norm"):
        features = _log(rng, 4, 65536)
        rows = _log(rng, 1, max(1, min(131072, MOST_NORM // features // (4 if dtype == "float32" else 2))))
        return {"op": op, "rows": rows, "features": features, "dtype": dtype,
                "weights": rng.choice(("float32", dtype)), "pad": rng.choice((0, 0, 1, 8))}
    while True:
        if op == "orthogonalize":
            c = {"op": op, "batch": _log(rng, 1, 64), "rows": _log(rng, 2, 4096), "cols": _log(rng, 2, 8192),
                 "dtype": dtype}
        else:
            shapes = [(_log(rng, 2, 2048), _log(rng, 2, 2048)) for _ in range(rng.randint(1, 12))]
            c = {"op": op, "shapes": ",".join("%dx%d" % s for s in shapes), "dtype": dtype}
        if work(c)["flops"] <= MOST_FLOPS and sum(b * m * n for b, m, n in _matrices(c)) <= MOST_MATRIX:
            return c


def _matrices(case):
    """The (batch, rows, cols) of a case's matrices."""
    if case["op"] == "orthogonalize":
        return [(case["batch"], case["rows"], case["cols"])]
    return [(1, *map(int, s.split("x"))) for s in case["shapes"].split(",")]


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _gradient(shape, dtype, gen):
    """A weight's gradient: rows and columns of decaying scale, so that its
    singular values cover some orders of magnitude."""
    g = torch.randn(shape, generator=gen, device="cuda")
    for axis in (-1, -2):
        n = shape[axis]
        s = torch.arange(1, n + 1, device="cuda", dtype=torch.float32).rsqrt()[torch.randperm(n, generator=gen, device="cuda")]
        g = g * (s if axis == -1 else s[:, None])
    return (0.03 * g).to(dtype)


def prepare(case, seed):
    gen, dtype, op = _generator(seed), DTYPES[case["dtype"]], case["op"]
    if op == "orthogonalize":
        shape = (case["rows"], case["cols"])
        return {"op": op, "g": _gradient(shape if case["batch"] == 1 else (case["batch"], *shape), dtype, gen)}
    if op == "muon":
        shapes = [(m, n) for _, m, n in _matrices(case)]
        return {"op": op,
                "params": [(torch.randn(s, generator=gen, device="cuda") / math.sqrt(s[1])).to(dtype) for s in shapes],
                "grads": [_gradient(s, dtype, gen) for s in shapes],
                "momenta": [_gradient(s, torch.float32, gen) for s in shapes]}
    rows, n, weights = case["rows"], case["features"], DTYPES[case["weights"]]
    # features of different scales and offsets
    scale = 0.5 + 2 * torch.rand(n, generator=gen, device="cuda")
    offset = torch.randn(n, generator=gen, device="cuda")
    wide = torch.empty((rows, n + case["pad"]), device="cuda", dtype=dtype).zero_()
    wide[:, :n] = torch.randn((rows, n), generator=gen, device="cuda") * scale + offset
    return {"op": op, "x": wide[:, :n],
            "weight": (1 + 0.2 * torch.randn(n, generator=gen, device="cuda")).to(weights),
            "bias": (0.2 * torch.randn(n, generator=gen, device="cuda")).to(weights),
            "grad": torch.randn((rows, n), generator=gen, device="cuda").to(dtype) if op == "norm_train" else None}


def run(state):
    return (_own if own else _plain)(state)


def _own(s):
    import paper_2301_03251_amd as Q

    if s["op"] == "norm":
        return Q.layer_norm(s["x"], s["weight"], s["bias"], EPS_NORM)
    if s["op"] == "norm_train":
        y, mean, rstd = Q.layer_norm_forward(s["x"], s["weight"], s["bias"], EPS_NORM)
        gx, gw, gb = Q.layer_norm_backward(s["grad"], s["x"], mean, rstd, s["weight"])
        return {"y": y, "grad_x": gx, "grad_weight": gw, "grad_bias": gb}
    if s["op"] == "orthogonalize":
        return Q.orthogonalize(s["g"])
    Q.muon_step(s["params"], s["grads"], s["momenta"], lr=LR, momentum=MOMENTUM, nesterov=True, weight_decay=DECAY)
    return {"params": s["params"], "momenta": s["momenta"]}


def _orthogonal(g):
    """The plain form of the orthogonalisation of a float32 matrix or a batch of them."""
    a, b, c = COEFFICIENTS
    x = g / (g.square().sum((-2, -1), keepdim=True).sqrt() + EPS_ORTHO)
    tall = x.shape[-2] > x.shape[-1]
    if tall:
        x = x.mT.contiguous()
    for _ in range(STEPS):
        gram = x @ x.mT
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.mT.contiguous() if tall else x


def _plain(s):
    if s["op"] == "orthogonalize":
        return _orthogonal(s["g"].float()).to(s["g"].dtype)
    if s["op"] == "muon":
        for p, g, m in zip(s["params"], s["grads"], s["momenta"]):
            g = g.float()
            m.mul_(MOMENTUM).add_(g)
            update = _orthogonal(g + MOMENTUM * m)
            rows, cols = p.shape
            p.copy_((1 - LR * DECAY) * p.float() - LR * math.sqrt(max(1.0, rows / cols)) * update)
        return {"params": s["params"], "momenta": s["momenta"]}
    x, weight, bias = s["x"].float(), s["weight"].float(), s["bias"].float()
    centred = x - x.mean(-1, keepdim=True)
    rstd = (centred.square().mean(-1, keepdim=True) + EPS_NORM).rsqrt()
    hat = centred * rstd
    y = (hat * weight + bias).to(s["x"].dtype)
    if s["op"] == "norm":
        return y
    grad = s["grad"].float()
    h = grad * weight
    gx = rstd * (h - h.mean(-1, keepdim=True) - hat * (h * hat).mean(-1, keepdim=True))
    return {"y": y, "grad_x": gx.to(y.dtype), "grad_weight": (grad * hat).sum(0).to(s["weight"].dtype),
            "grad_bias": grad.sum(0).to(s["bias"].dtype)}


def _exact_orthogonal(u):
    """The singular values of u through the polynomial p(t) = a t + b t^3 + c t^5,
    STEPS times: every step is u's Gram matrix S through a polynomial that
    commutes with it, so their product is applied to u once."""
    a, b, c = COEFFICIENTS
    u = u / (torch.linalg.matrix_norm(u, keepdim=True) + EPS_ORTHO)
    if u.shape[-2] > u.shape[-1]:
        return _exact_turned(u.transpose(-2, -1).contiguous(), a, b, c).transpose(-2, -1).contiguous()
    return _exact_turned(u, a, b, c)


def _exact_turned(u, a, b, c):
    eye = torch.eye(u.shape[-2], dtype=torch.float64, device=u.device)
    s = torch.matmul(u, u.transpose(-2, -1).contiguous())
    total = eye
    for _ in range(STEPS):
        q = a * eye + torch.matmul(s, b * eye + c * s)
        total = torch.matmul(q, total)
        s = torch.matmul(torch.matmul(q, s), q)
    return torch.matmul(total, u)


def exact(case, seed):
    s = prepare(case, seed)
    if s["op"] == "orthogonalize":
        return _exact_orthogonal(s["g"].double())
    if s["op"] == "muon":
        params, momenta = [], []
        for p, g, m in zip(s["params"], s["grads"], s["momenta"]):
            g = g.double()
            momenta.append(torch.add(g, m.double(), alpha=MOMENTUM))
            update = _exact_orthogonal(torch.add(g, momenta[-1], alpha=MOMENTUM))
            grow = max(1.0, p.shape[0] / p.shape[1]) ** 0.5
            params.append(torch.sub(p.double(), p.double() * (DECAY * LR) + update * (grow * LR)))
        return {"params": params, "momenta": momenta}
    x, weight, bias = s["x"].double(), s["weight"].double(), s["bias"].double()
    n = x.shape[1]
    var, mean = torch.var_mean(x, dim=1, correction=0)
    rstd = 1 / torch.sqrt(var + EPS_NORM)
    hat = torch.addcmul(torch.zeros_like(x), x - mean[:, None], rstd[:, None])
    y = torch.addcmul(bias, hat, weight)
    if s["op"] == "norm":
        return y
    # dx = J^T (g w), J = rstd (1 - 1 1^T / n - hat hat^T / n)
    v = s["grad"].double() * weight
    along = torch.stack((torch.full_like(v, n ** -0.5), hat * n ** -0.5))
    gx = v - (along * (along * v).sum(2, keepdim=True)).sum(0)
    return {"y": y, "grad_x": gx * rstd[:, None], "grad_weight": torch.einsum("rf,rf->f", s["grad"].double(), hat),
            "grad_bias": torch.einsum("rf->f", s["grad"].double())}


def work(case):
    size = DTYPES[case["dtype"]].itemsize
    if case["op"].startswith("norm"):
        rows, n, w = case["rows"], case["features"], DTYPES[case["weights"]].itemsize
        if case["op"] == "norm":
            return {"bytes": 2 * rows * n * size + 2 * n * w, "flops": 8 * rows * n}
        return {"bytes": 4 * rows * n * size + 4 * n * w, "flops": 24 * rows * n}
    flops = moved = 0
    for batch, m, n in _matrices(case):
        small, large = min(m, n), max(m, n)
        # the Gram matrix and its square are symmetric: half of their products
        flops += batch * STEPS * (3 * small * small * large + small ** 3)
        moved += batch * m * n * (2 * size if case["op"] == "orthogonalize" else 3 * size + 8)
    return {"bytes": moved, "flops": flops}
