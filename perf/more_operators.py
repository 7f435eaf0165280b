"""Performance cases of the operators of a network that reads sequences of tokens
in front of a quantum layer: embedding lookup, dropout, root-mean-square norm with
the residual's addition, and a gated linear recurrence.

A case names one pass by plain values. ``op`` is

* ``embed``: rows of a table of ``vocabulary`` x ``features`` for ``tokens``
  tokens, times a scale; ``embed_train``: the same, then the table's gradient;
* ``dropout``: a mask drawn from a counter, applied to ``rows`` x ``features``;
  ``dropout_train``: the same, then the gradient with the mask drawn again;
* ``rms``: the residual's addition and the norm of the sum, forward only;
  ``rms_train``: the same, then its backward; ``rms_quantized``: with an output
  in 8 bits (e4m3) and one scale a row;
* ``scan``: h_t = a_t h_{t-1} + (1 - a_t) x_t with a = sigmoid(gate) over
  ``steps`` steps of ``batch`` sequences, forward only; ``scan_train``: the same,
  then its backward; ``scan_step``: one step, the state changes in place.

``dtype`` is that of the arrays; ``weights`` that of the norm's weight.
"""

from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
EPS = 1e-6
MOST_8BIT = 448.0  # the largest value of e4m3
SEED, OFFSET = 0x1234567890ABCDEF, 77
# Philox 4x32 (Salmon, Moraes, Dror, Shaw 2011): multipliers and key increments
PHILOX_M = (0xD2511F53, 0xCD9E8D57)
PHILOX_W = (0x9E3779B9, 0xBB67AE85)
WORD = 0xFFFFFFFF


def _embed(name, op, tokens, vocabulary, features, dtype="float32", padded=0.0, scale=1.0):
    return {"name": name, "op": op, "tokens": tokens, "vocabulary": vocabulary, "features": features, "dtype": dtype,
            "padded": padded, "scale": scale}


def _dropout(name, op, rows, features, p, dtype="float32"):
    return {"name": name, "op": op, "rows": rows, "features": features, "p": p, "dtype": dtype}


def _rms(name, op, rows, features, dtype="float32", weights="float32", residual=True, pad=0):
    return {"name": name, "op": op, "rows": rows, "features": features, "dtype": dtype, "weights": weights,
            "residual": residual, "pad": pad}


def _scan(name, op, batch, steps, features, dtype="float32", packed=False, halves=False, initial=False):
    return {"name": name, "op": op, "batch": batch, "steps": steps, "features": features, "dtype": dtype,
            "packed": packed, "halves": halves, "initial": initial}


def listed():
    return [
        # serving: the next token of 32 sequences
        _embed("embed 32 of 32000x1024 bf16", "embed", 32, 32000, 1024, "bfloat16"),
        # training a small hybrid network: 32 padded sequences of 128 tokens
        _embed("embed train 4096 of 1000x64", "embed_train", 4096, 1000, 64, padded=0.3, scale=8.0),
        # training a large table: frequent tokens have thousands of rows of gradient
        _embed("embed train 131072 of 50000x1024 bf16", "embed_train", 131072, 50000, 1024, "bfloat16", scale=32.0),
        # training: the features of 256 samples in front of a quantum layer
        _dropout("dropout train 256x64", "dropout_train", 256, 64, 0.1),
        # training: the largest activations, in mixed precision
        _dropout("dropout train 131072x1024 bf16", "dropout_train", 131072, 1024, 0.1, "bfloat16"),
        # serving: one token of 32 sequences on its way to a product in 8 bits
        _rms("rms quantized 32x4096 bf16", "rms_quantized", 32, 4096, "bfloat16", "bfloat16"),
        # training in half precision over some columns of a wider array, odd sizes
        _rms("rms train 1037x1001 f16 strided", "rms_train", 1037, 1001, "float16", "float16", pad=7),
        # training: an ordinary layer in mixed precision
        _rms("rms train 8192x1024 bf16", "rms_train", 8192, 1024, "bfloat16"),
        # a whole prompt through a wide layer, in 8 bits
        _rms("rms quantized 16384x8192 bf16", "rms_quantized", 16384, 8192, "bfloat16", "bfloat16"),
        # serving: the next token of 256 sequences
        _scan("scan step 256x1024 bf16", "scan_step", 256, 1, 1024, "bfloat16", halves=True, initial=True),
        # training: few features over a long axis with packed sequences
        _scan("scan train 1x65536x64 packed", "scan_train", 1, 65536, 64, packed=True),
        # training: an ordinary layer, x and gate the halves of one projection
        _scan("scan train 8x4096x2048 bf16", "scan_train", 8, 4096, 2048, "bfloat16", halves=True, initial=True),
    ]


def _log(rng, low, high):
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 0.5)))))))


def draw(rng):
    """A case of the listed ones' ranges that moves no more than the largest of its kind."""
    kind = rng.choice(("embed", "dropout", "rms", "scan"))
    most = max(work(c)["bytes"] for c in listed() if c["op"].startswith(kind))
    while True:
        c = _drawn(kind, rng)
        if work(c)["bytes"] <= most:
            return c


def _drawn(kind, rng):
    dtype = rng.choice(tuple(DTYPES))
    if kind == "embed":
        c = _embed("", rng.choice(("embed", "embed_train")), _log(rng, 1, 262144), _log(rng, 2, 262144), _log(rng, 4, 8192),
                   dtype, rng.choice((0.0, 0.25)), rng.choice((1.0, 11.5)))
    elif kind == "dropout":
        c = _dropout("", rng.choice(("dropout", "dropout_train")), _log(rng, 1, 131072), _log(rng, 4, 65536),
                     rng.choice((0.05, 0.1, 0.5)), dtype)
    elif kind == "rms":
        c = _rms("", rng.choice(("rms", "rms_train", "rms_quantized")), _log(rng, 1, 131072), _log(rng, 4, 65536), dtype,
                 rng.choice(("float32", dtype)), rng.random() < 0.7, rng.choice((0, 0, 1, 8)))
    else:
        op = rng.choice(("scan", "scan_train", "scan_train", "scan_step"))
        packed = op != "scan_step" and rng.random() < 0.4
        c = _scan("", op, _log(rng, 1, 512), 1 if op == "scan_step" else _log(rng, 1, 65536), _log(rng, 4, 4096), dtype,
                  packed, rng.random() < 0.5, op == "scan_step" or rng.random() < 0.5)
    del c["name"]
    return c


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(shape, gen, dtype=torch.float32):
    return torch.randn(shape, generator=gen, device="cuda").to(dtype)


def _uniform(n, gen):
    return torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)


def _rows(rows, n, pad, gen, dtype):
    """Rows of features of different scales, as the first columns of a wider array."""
    wide = torch.empty((rows, n + pad), device="cuda", dtype=dtype).zero_()
    wide[:, :n] = _normal((rows, n), gen) * (0.5 + 2 * torch.rand(n, generator=gen, device="cuda"))
    return wide[:, :n]


def prepare(case, seed):
    gen, dtype, op = _generator(seed), DTYPES[case["dtype"]], case["op"]
    s = {"op": op}
    if op.startswith("embed"):
        n, vocabulary, features = case["tokens"], case["vocabulary"], case["features"]
        # the k-th most frequent token is met about 1 / k times as often as the first
        rank = (float(vocabulary) ** _uniform(n, gen)).long() - 1
        names = torch.randperm(vocabulary, generator=gen, device="cuda")
        tokens = names[rank.clamp_(0, vocabulary - 1)]
        s["padding"] = None
        if case["padded"]:
            s["padding"] = 0
            tokens = torch.where(_uniform(n, gen) < case["padded"], torch.zeros_like(tokens), tokens)
        s.update(tokens=tokens, weight=(0.02 * _normal((vocabulary, features), gen)).to(dtype), scale=case["scale"])
        if op == "embed_train":
            s["grad"] = _normal((n, features), gen, dtype)
        return s
    if op.startswith("dropout"):
        shape = (case["rows"], case["features"])
        # the pair that a layer keeps on the card: its seed, and how often it was called
        s.update(p=case["p"], x=_normal(shape, gen, dtype), seed=(SEED, OFFSET + int(seed)),
                 key=torch.tensor([SEED, OFFSET + int(seed)], device="cuda"))
        if op == "dropout_train":
            s["grad"] = _normal(shape, gen, dtype)
        return s
    if op.startswith("rms"):
        rows, n = case["rows"], case["features"]
        s.update(x=_rows(rows, n, case["pad"], gen, dtype), residual=_normal((rows, n), gen, dtype) if case["residual"] else None,
                 weight=(1 + 0.2 * _normal(n, gen)).to(DTYPES[case["weights"]]))
        if op == "rms_train":
            s["grad"] = _normal((rows, n), gen, dtype)
            s["grad_summed"] = _normal((rows, n), gen, dtype) if case["residual"] else None
        return s
    batch, steps, features = case["batch"], case["steps"], case["features"]
    shape = (batch, steps, 2 * features) if case["halves"] else (2, batch, steps, features)
    both = torch.empty(shape, device="cuda", dtype=dtype)
    x, gate = both.chunk(2, -1) if case["halves"] else both.unbind(0)
    x.copy_(_normal(x.shape, gen))
    # gates that remember from a step to some thousand
    gate.copy_(2 + 2 * _normal(gate.shape, gen))
    s.update(x=x, gate=gate, initial=_normal((batch, features), gen) if case["initial"] else None, starts=None)
    if case["packed"]:
        # sequences of 1 to a few thousand steps, one behind the other
        s["starts"] = _uniform((batch, steps), gen) < torch.exp(-8 * _uniform((batch, 1), gen)).clamp(max=0.5)
    if op == "scan_train":
        s["grad"] = _normal((batch, steps, features), gen, dtype)
    if op == "scan_step":
        s.update(x=x[:, 0], gate=gate[:, 0], state=s.pop("initial"))
    return s


def run(state):
    return (_own if own else _plain)(state)


def _own(s):
    import paper_2301_03251_amd as Q

    op = s["op"]
    if op.startswith("embed"):
        y = Q.embedding_forward(s["tokens"], s["weight"], s["scale"], s["padding"])
        if op == "embed":
            return y
        return {"y": y, "grad_weight": Q.embedding_backward(s["grad"], s["tokens"], s["weight"].shape[0], s["scale"],
                                                            s["padding"])}
    if op.startswith("dropout"):
        y = Q.dropout_forward(s["x"], s["p"], s["key"])
        if op == "dropout":
            return y
        return {"y": y, "grad_x": Q.dropout_forward(s["grad"], s["p"], s["key"])}
    if op == "rms_quantized":
        q, scale, summed = Q.rms_norm_quantized(s["x"], s["weight"], s["residual"], EPS)
        return {"q": q, "scale": scale, "summed": summed}
    if op.startswith("rms"):
        y, summed, rstd = Q.rms_norm_forward(s["x"], s["weight"], s["residual"], EPS, stats=op == "rms_train")
        out = {"y": y, "summed": summed}
        if op == "rms_train":
            out["grad_x"], out["grad_weight"] = Q.rms_norm_backward(s["grad"], summed, rstd, s["weight"], s["grad_summed"])
        return out
    if op == "scan_step":
        return {"h": Q.gated_scan_step(s["x"], s["gate"], s["state"]), "state": s["state"]}
    h, last, states = Q.gated_scan_forward(s["x"], s["gate"], s["initial"], s["starts"], states=op == "scan_train")
    out = {"h": h, "last": last}
    if op == "scan_train":
        out["grad_x"], out["grad_gate"], grad = Q.gated_scan_backward(s["grad"], s["x"], s["gate"], states, s["starts"],
                                                                      want_initial=s["initial"] is not None)
        if grad is not None:
            out["grad_initial"] = grad
    return out


def _words(count, seed, offset):
    """The words of ``count`` counters (i, offset) as [count, 4], in int64: the
    product of two words keeps its 64 bits there, whatever its sign."""
    i = torch.arange(count, device="cuda")
    c0, c1 = i & WORD, i >> 32
    c2, c3 = torch.full_like(i, offset & WORD), torch.full_like(i, offset >> 32)
    k0, k1 = seed & WORD, seed >> 32
    for _ in range(10):
        p0, p1 = c0 * PHILOX_M[0], c2 * PHILOX_M[1]
        c0, c1, c2, c3 = ((p1 >> 32) & WORD) ^ c1 ^ k0, p1 & WORD, ((p0 >> 32) & WORD) ^ c3 ^ k1, p0 & WORD
        k0, k1 = (k0 + PHILOX_W[0]) & WORD, (k1 + PHILOX_W[1]) & WORD
    return torch.stack((c0, c1, c2, c3), 1)


def _scan_pairs(a, b):
    """h_t = a_t h_{t-1} + b_t along axis 1 from h = 0, by doubling the reach of pairs (a, b)."""
    a, b, reach = a.clone(), b.clone(), 1
    while reach < b.shape[1]:
        b[:, reach:] = torch.addcmul(b[:, reach:], a[:, reach:], b[:, :-reach])
        a[:, reach:] = a[:, reach:] * a[:, :-reach]
        reach *= 2
    return b


def _plain(s):
    op = s["op"]
    if op.startswith("embed"):
        tokens, weight, scale = s["tokens"], s["weight"], s["scale"]
        y = weight[tokens].float() * scale
        if s["padding"] is not None:
            y = torch.where((tokens == s["padding"])[:, None], torch.zeros_like(y), y)
        if op == "embed":
            return y.to(weight.dtype)
        grad = s["grad"].float() * scale
        if s["padding"] is not None:
            grad = torch.where((tokens == s["padding"])[:, None], torch.zeros_like(grad), grad)
        total = torch.zeros(weight.shape, dtype=torch.float32, device=weight.device).index_add_(0, tokens, grad)
        return {"y": y.to(weight.dtype), "grad_weight": total.to(weight.dtype)}
    if op.startswith("dropout"):
        x, p = s["x"], s["p"]
        words = _words((x.numel() + 3) // 4, *s["seed"]).view(-1)[:x.numel()].view(x.shape)
        keep = words >= round(p * 2.0 ** 32)
        y = torch.where(keep, x.float() * (1 / (1 - p)), torch.zeros_like(x, dtype=torch.float32)).to(x.dtype)
        if op == "dropout":
            return y
        grad = torch.where(keep, s["grad"].float() * (1 / (1 - p)), torch.zeros_like(x, dtype=torch.float32)).to(x.dtype)
        return {"y": y, "grad_x": grad}
    if op.startswith("rms"):
        x, dtype, weight = s["x"], s["x"].dtype, s["weight"].float()
        summed = x if s["residual"] is None else (x.float() + s["residual"].float()).to(dtype)
        v = summed.float()
        rstd = (v.square().mean(-1, keepdim=True) + EPS).rsqrt()
        hat = v * rstd
        y = hat * weight
        if op == "rms_quantized":
            scale = y.abs().amax(-1, keepdim=True) / MOST_8BIT
            return {"q": (y / scale).to(torch.float8_e4m3fn), "scale": scale[:, 0], "summed": summed}
        out = {"y": y.to(dtype), "summed": summed}
        if op == "rms_train":
            grad = s["grad"].float()
            g = grad * weight
            gx = rstd * (g - hat * (g * hat).mean(-1, keepdim=True))
            if s["grad_summed"] is not None:
                gx = gx + s["grad_summed"].float()
            out.update(grad_x=gx.to(dtype), grad_weight=(grad * hat).sum(0).to(s["weight"].dtype))
        return out
    x, gate, dtype = s["x"].float(), s["gate"].float(), s["x"].dtype
    a, rest = torch.sigmoid(gate), torch.sigmoid(-gate)
    if op == "scan_step":
        h = a * s["state"] + rest * x
        s["state"].copy_(h)
        return {"h": h.to(dtype), "state": s["state"]}
    carry = a if s["starts"] is None else torch.where(s["starts"][:, :, None], torch.zeros_like(a), a)
    b = rest * x
    if s["initial"] is not None:
        b[:, 0] += carry[:, 0] * s["initial"]
    h = _scan_pairs(carry, b)
    out = {"h": h.to(dtype), "last": h[:, -1].clone()}
    if op == "scan_train":
        # total gradients of h: d_t = grad_t + a_{t+1} d_{t+1}
        later = torch.zeros_like(carry)
        later[:, :-1] = carry[:, 1:]
        d = _scan_pairs(later.flip(1), s["grad"].float().flip(1)).flip(1)
        before = torch.zeros_like(h)
        before[:, 1:] = h[:, :-1]
        if s["initial"] is not None:
            before[:, 0] = s["initial"]
        if s["starts"] is not None:
            before = torch.where(s["starts"][:, :, None], torch.zeros_like(before), before)
        out.update(grad_x=(rest * d).to(dtype), grad_gate=(d * (before - x) * a * rest).to(dtype))
        if s["initial"] is not None:
            out["grad_initial"] = carry[:, 0] * d[:, 0]
    return out


def _exact_keep(n, seed, offset, p):
    """The mask of n values, on the host in unsigned integers."""
    i = np.arange((n + 3) // 4, dtype=np.uint64)
    half = np.uint64(32)
    ctr = [i & np.uint64(WORD), i >> half, np.full_like(i, offset & WORD), np.full_like(i, offset >> 32)]
    key = [seed & WORD, seed >> 32]
    for r in range(10):
        left, right = ctr[0] * np.uint64(PHILOX_M[0]), ctr[2] * np.uint64(PHILOX_M[1])
        ctr = [(right >> half) ^ ctr[1] ^ np.uint64((key[0] + r * PHILOX_W[0]) % 2 ** 32), right & np.uint64(WORD),
               (left >> half) ^ ctr[3] ^ np.uint64((key[1] + r * PHILOX_W[1]) % 2 ** 32), left & np.uint64(WORD)]
    words = np.stack(ctr, -1).reshape(-1)[:n]
    return torch.from_numpy(words.astype(np.int64) >= int(round(p * 4294967296.0))).cuda()


def _exact_scan(s):
    x, gate = s["x"].double(), s["gate"].double()
    a = 1 / (1 + torch.exp(-gate))
    if s["op"] == "scan_step":
        h = x + a * (s["state"].double() - x)
        return {"h": h, "state": h}
    steps, starts = x.shape[1], s["starts"]
    zero = torch.zeros_like(x[:, 0])
    h, before = torch.empty_like(x), torch.empty_like(x)
    held = zero if s["initial"] is None else s["initial"].double()
    going = None if starts is None else (~starts).double()
    for t in range(steps):
        if going is not None:
            held = held * going[:, t, None]
        before[:, t] = held
        held = torch.lerp(x[:, t], held, a[:, t])
        h[:, t] = held
    out = {"h": h, "last": held}
    if s["op"] == "scan_train":
        grad, d = s["grad"].double(), torch.empty_like(x)
        behind = zero
        for t in range(steps - 1, -1, -1):
            d[:, t] = grad[:, t] + behind
            behind = a[:, t] * d[:, t]
            if going is not None:
                behind = behind * going[:, t, None]
        out.update(grad_x=d * (1 - a), grad_gate=d * (before - x) * (a - a * a))
        if s["initial"] is not None:
            out["grad_initial"] = behind
    return out


def exact(case, seed):
    s = prepare(case, seed)
    op = s["op"]
    if op.startswith("embed"):
        kept = torch.ones(len(s["tokens"]), dtype=torch.float64, device="cuda")
        if s["padding"] is not None:
            kept = (s["tokens"] != s["padding"]).double()
        factor = (kept * s["scale"])[:, None]
        y = torch.index_select(s["weight"].double(), 0, s["tokens"]) * factor
        if op == "embed":
            return y
        # sums of equal tokens from differences of running sums over the sorted ones
        order = torch.argsort(s["tokens"], stable=True)
        counts = torch.bincount(s["tokens"], minlength=case["vocabulary"])
        ends = torch.cumsum(counts, 0)
        total = torch.empty((case["vocabulary"], case["features"]), dtype=torch.float64, device="cuda")
        for first in range(0, case["features"], 64):
            part = s["grad"][:, first:first + 64].double() * factor
            running = torch.cat((torch.zeros_like(part[:1]), torch.cumsum(part[order], 0)))
            total[:, first:first + 64] = running[ends] - running[ends - counts]
        return {"y": y, "grad_weight": total}
    if op.startswith("dropout"):
        if s["x"].numel() > 1 << 25:
            return None
        keep = _exact_keep(s["x"].numel(), *s["seed"], s["p"]).view(s["x"].shape).double()
        y = s["x"].double() * keep / (1 - s["p"])
        return y if op == "dropout" else {"y": y, "grad_x": s["grad"].double() * keep / (1 - s["p"])}
    if op.startswith("rms"):
        dtype, weight, n = s["x"].dtype, s["weight"].double(), case["features"]
        v = s["x"].double()
        if s["residual"] is not None:
            v = (v + s["residual"].double()).to(dtype).double()
        rms = torch.sqrt(torch.linalg.vector_norm(v, dim=-1, keepdim=True) ** 2 / n + EPS)
        y = v * weight / rms
        if op == "rms_quantized":
            scale = torch.linalg.vector_norm(y, ord=math.inf, dim=-1) / MOST_8BIT
            return {"q": y / scale[:, None], "scale": scale, "summed": v}
        out = {"y": y, "summed": v}
        if op == "rms_train":
            g = s["grad"].double()
            # J = (1 - v v^T / (n rms^2)) / rms
            along = torch.sum(g * weight * v, -1, keepdim=True) / (n * rms ** 2)
            gx = (g * weight - along * v) / rms
            out.update(grad_x=gx if s["grad_summed"] is None else gx + s["grad_summed"].double(),
                       grad_weight=torch.sum(g * v / rms, 0))
        return out
    return _exact_scan(s)


def work(case):
    size, op = DTYPES[case["dtype"]].itemsize, case["op"]
    if op.startswith("embed"):
        n, rows, features = case["tokens"], case["vocabulary"], case["features"]
        moved, flops = 8 * n + (min(n, rows) + n) * features * size, n * features
        if op == "embed_train":
            moved, flops = moved + (n + rows) * features * size, flops + 2 * n * features
        return {"bytes": moved, "flops": flops}
    if op.startswith("dropout"):
        n = case["rows"] * case["features"]
        # ten rounds of two products for four values
        passes = 2 if op == "dropout_train" else 1
        return {"bytes": passes * 2 * n * size, "flops": passes * 12 * n}
    if op.startswith("rms"):
        n, w = case["rows"] * case["features"], DTYPES[case["weights"]].itemsize * case["features"]
        extra = 2 if case["residual"] else 0  # the residual and the sum
        if op == "rms_quantized":
            return {"bytes": n * (size * (1 + extra) + 1) + w + 4 * case["rows"], "flops": 6 * n}
        if op == "rms":
            return {"bytes": n * size * (2 + extra) + w, "flops": 5 * n}
        return {"bytes": n * size * (4 + extra + (1 if case["residual"] else 0)) + 2 * w, "flops": 16 * n}
    n, state = case["batch"] * case["steps"] * case["features"], case["batch"] * case["features"] * 4
    if op == "scan_train":
        return {"bytes": 6 * n * size + (3 if case["initial"] else 1) * state, "flops": 25 * n}
    return {"bytes": 3 * n * size + (2 if case["initial"] else 1) * state, "flops": 10 * n}
