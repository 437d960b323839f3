"""The operators around a training step's products, as cases that can be timed and compared.

Three kinds: the norms before and after a block with its gate, residual scale and residual sum, and
their gradients; the scaled embedding lookup and its gradient; the norm of all gradients and their
clipping.  ``own = False`` computes them in their plain form (elementary torch operations in 32
bits, rounded once at the end), ``own = True`` through the package's public calls.

Shapes are those of the GPT-shaped workload (hidden 1024, 2048 or 4096, four times hidden between
the two products of a block, vocabulary 50304, batches of 1 to 16 sequences of 512 to 2048 tokens)
and odd ones around them.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS = 1e-5
ALPHA = 0.5  # the residual branch's constant factor
EMBED = 1.5  # the lookup's factor
MAX_NORM = 1.0
RESCALE = 1.25  # a mean over all tokens turned into one over the tokens that are kept

MOST_TN = 32768 * 4096
MOST_VN = 50304 * 4096
MOST_CLIP_BYTES = 2 * (24 * 8 * 2048 * 2048 + 2 * 50304 * 2048)


def _norm(name, op, t, n, dtype, block, post, gate, scaled, pre, pad):
    """`block`: there is a block's output to add (else the norm of the residual stream alone)."""
    c = {"op": op, "t": t, "n": n, "dtype": dtype, "block": block, "post": post, "gate": gate, "scaled": scaled, "pre": pre, "pad": pad}
    return {"name": name, **c} if name else c


def _emb(name, op, t, v, n, dtype, padded, add, wide, pad):
    """`padded`: the share of tokens that are padding; `add`: the gradient is added to one that is there; `wide`: it is in 32 bits."""
    c = {"op": op, "t": t, "v": v, "n": n, "dtype": dtype, "padded": padded, "add": add, "wide": wide, "pad": pad}
    return {"name": name, **c} if name else c


def _clip(name, layers, hidden, vocab, dtype, gap):
    """`gap`: elements between one gradient and the next."""
    c = {"op": "clip", "layers": layers, "hidden": hidden, "vocab": vocab, "dtype": dtype, "gap": gap}
    return {"name": name, **c} if name else c


def listed():
    return [
        # One token between two blocks of a sampler: the residual sum and the next block's norm, where latency counts.
        _norm("norm, one token", "norm", 1, 2048, "bf16", True, "none", "none", False, "rms", 0),
        # Between two blocks of the widest model, 16 sequences of 2048: norms on both sides, a gate and a scale a channel.
        _norm("norm, largest", "norm", 32768, 4096, "bf16", True, "rms", "sigmoid", True, "rms", 0),
        # A ragged batch of a pruned model of odd width, rows padded, with means and biases.
        _norm("norm, ragged", "norm", 1003, 2047, "f16", True, "layer", "none", True, "layer", 5),
        # Gradients between two blocks, 8 sequences of 1024.
        _norm("norm backward, block", "norm_backward", 8192, 2048, "bf16", True, "rms", "silu", True, "rms", 0),
        # Gradients of a ragged batch kept in 32 bits.
        _norm("norm backward, ragged", "norm_backward", 1003, 1021, "f32", True, "layer", "sigmoid", False, "layer", 3),
        # The sampled token's row: the first call of a sampler's step.
        _emb("embedding, one token", "embedding", 1, 50304, 1024, "bf16", 0.0, False, False, 0),
        # A whole batch, 16 sequences of 2048, a tenth of it padding.
        _emb("embedding, largest", "embedding", 32768, 50304, 4096, "bf16", 0.1, False, False, 0),
        # A few tokens of a toy policy with an odd vocabulary and width, in 32 bits, rows padded.
        _emb("embedding backward, small", "embedding_backward", 37, 1021, 515, "f32", 0.0, False, True, 3),
        # The gradient of a whole batch, 16 sequences of 2048: frequent tokens have thousands of rows.
        _emb("embedding backward, batch", "embedding_backward", 32768, 50304, 2048, "bf16", 0.1, False, False, 0),
        # A micro-batch's gradient added to the 32-bit sum that it shares with the head's.
        _emb("embedding backward, added", "embedding_backward", 8192, 50304, 1024, "bf16", 0.0, True, True, 0),
        # All gradients of a small policy: 27 tensors.
        _clip("clip, small", 4, 256, 1024, "bf16", 0),
        # All gradients of 24 layers at hidden 2048: 147 tensors.
        _clip("clip, largest", 24, 2048, 50304, "bf16", 0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size spread over its logarithm: a multiple of 64 half of the time where it can be, any number otherwise."""
    s = _log(rng, lo, hi)
    return s // 64 * 64 if s >= 64 and rng.random() < 0.5 else s


def draw(rng):
    op = rng.choice(["norm", "norm_backward", "embedding", "embedding_backward", "clip"])
    dtype, pad = rng.choice(["bf16", "bf16", "f16", "f32"]), rng.choice([0, 0, 8, 3])
    size = 2 if dtype == "f32" else 1
    if op in ("norm", "norm_backward"):
        while True:
            t, n = _log(rng, 1, 32768), _size(rng, 32, 16384)
            if t * n * size * (2 if op == "norm_backward" else 1) <= MOST_TN:
                break
        block = rng.random() < 0.85
        post, gate = rng.choice(["none", "rms", "layer"]), rng.choice(["none", "plain", "sigmoid", "silu"])
        pre = rng.choice(["none", "rms", "rms", "layer"]) if block else rng.choice(["rms", "layer"])
        return _norm(None, op, t, n, dtype, block, post if block else "none", gate if block else "none", block and rng.random() < 0.5, pre, pad)
    if op in ("embedding", "embedding_backward"):
        while True:
            t, v, n = _log(rng, 1, 32768), _log(rng, 33, 200000), _size(rng, 32, 8192)
            if t * n * size <= MOST_TN and v * n * size <= MOST_VN:
                break
        back = op == "embedding_backward"
        return _emb(None, op, t, v, n, dtype, rng.choice([0.0, 0.1, 0.5]), back and rng.random() < 0.4, back and rng.random() < 0.5, pad)
    while True:
        layers, hidden, vocab = _log(rng, 1, 40), _size(rng, 16, 4096), _log(rng, 33, 50304)
        if 2 * size * (8 * layers * hidden * hidden + 2 * vocab * hidden) <= MOST_CLIP_BYTES:
            break
    return _clip(None, layers, hidden, vocab, dtype, rng.choice([0, 0, 8, 3]))


# ------------------------------------------------------------------ inputs


def _rows(g, rows, cols, dtype, scale, pad):
    """A [rows, cols] matrix of normal values whose rows are `pad` elements apart."""
    x = torch.randn(rows, cols + pad, generator=g, device="cuda", dtype=torch.float32 if rows * cols < 1 << 24 else dtype)
    return x.mul_(scale).to(dtype)[:, :cols]


def _shapes(c):
    """The gradients of a residual MLP policy: matrices in the case's type, vectors in 32 bits."""
    h, v = c["hidden"], c["vocab"]
    matrices, vectors = [(v, h)], []
    for _ in range(c["layers"]):
        matrices += [(4 * h, h), (h, 4 * h)]
        vectors += [(h,), (4 * h,), (h,), (h,)]
    return matrices + [(v, h)], vectors + [(h,)]


def _views(flat, shapes, gap):
    at, got = 0, []
    for s in shapes:
        got.append(flat[at:at + math.prod(s)].view(s))
        at += math.prod(s) + gap
    return got


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    c, op = dict(case), case["op"]
    dt = DTYPES[c["dtype"]]
    vector = lambda n, mean, spread: mean + spread * torch.randn(n, generator=g, device="cuda")
    if op in ("norm", "norm_backward"):
        t, n, pad, block = c["t"], c["n"], c["pad"], c["block"]
        c["r"] = _rows(g, t, n, dt, 2.0, pad)  # norm_backward: as the forward pass wrote it
        c["h"] = _rows(g, t, n, dt, 0.7, pad) if block else None
        c["g"] = _rows(g, t, n, dt, 1.0, pad) if c["gate"] != "none" else None
        c["s"] = vector(n, 0.5, 0.1) if c["scaled"] else None
        c["w1"] = vector(n, 1.0, 0.1) if c["post"] != "none" else None
        c["b1"] = vector(n, 0.0, 0.1) if c["post"] == "layer" else None
        c["w2"] = vector(n, 1.0, 0.1) if c["pre"] != "none" else None
        c["b2"] = vector(n, 0.0, 0.1) if c["pre"] == "layer" else None
        if op == "norm_backward":
            c["dy"] = _rows(g, t, n, dt, 0.01, pad) if c["pre"] != "none" else None
            c["dout"] = _rows(g, t, n, dt, 0.01, pad) if block else None
            # what the forward pass kept of its norms
            c["stats"] = torch.cat([_statistics(c["h"], c["post"], t), _statistics(c["r"], c["pre"], t)])
    elif op in ("embedding", "embedding_backward"):
        t, v, n, pad = c["t"], c["v"], c["n"], c["pad"]
        # frequent tokens first: the chance of token i goes with 1 / (i + 1)
        u = torch.rand(t, generator=g, device="cuda", dtype=torch.float64)
        ids = (torch.exp(u * math.log(v + 1)) - 1).long().clamp_(0, v - 1)
        c["none"] = v - 1 if c["padded"] else None
        if c["padded"]:
            ids[torch.rand(t, generator=g, device="cuda") < c["padded"]] = v - 1
        c["ids"] = ids
        if op == "embedding":
            c["table"] = _rows(g, v, n, dt, 1.0, pad)
        else:
            c["dy"] = _rows(g, t, n, dt, 0.01, pad)
            wide = torch.float32 if c["wide"] else dt
            c["sum"] = _rows(g, v, n, wide, 0.01, pad) if c["add"] else None
    else:
        matrices, vectors = _shapes(c)
        total = lambda shapes: sum(math.prod(s) + c["gap"] for s in shapes)
        # a bucket of each type, its gradients one after another
        c["flat"] = [_rows(g, 1, total(matrices), dt, 1e-3, 0)[0], _rows(g, 1, total(vectors), torch.float32, 1e-3, 0)[0]]
        c["grads"] = _views(c["flat"][0], matrices, c["gap"]) + _views(c["flat"][1], vectors, c["gap"])
    return c


def _statistics(x, kind, t):
    """Mean and reciprocal deviation of each row, [2, t]."""
    out = torch.zeros(2, t, device="cuda")
    if kind != "none":
        d = x.double()
        if kind == "layer":
            out[0] = d.mean(1)
            d = d - d.mean(1, keepdim=True)
        out[1] = (d.square().mean(1) + EPS) ** -0.5
    return out


# ------------------------------------------------------------------ one pass


def run(state):
    c, op = state, state["op"]
    if own:
        import paper_2510_21048_amd as xm

        gate = "none" if c.get("gate") == "plain" else c.get("gate")
        if op == "norm":
            return xm.residual_norm_forward(c["r"], c["h"], c["g"], c["s"], ALPHA, post=c["post"], post_weight=c["w1"], post_bias=c["b1"],
                                            pre=c["pre"], pre_weight=c["w2"], pre_bias=c["b2"], gate_activation=gate, eps=EPS, save_stats=True)
        if op == "norm_backward":
            return xm.residual_norm_backward(c["dy"], c["dout"], c["r"], c["stats"], c["h"], c["g"], c["s"], ALPHA, post=c["post"],
                                             post_weight=c["w1"], post_bias=c["b1"], pre=c["pre"], pre_weight=c["w2"], pre_bias=c["b2"],
                                             gate_activation=gate)
        if op == "embedding":
            return xm.embedding_forward(c["table"], c["ids"], EMBED, c["none"])
        if op == "embedding_backward":
            return xm.embedding_backward(c["dy"], c["ids"], c["v"], EMBED, c["none"], into=c["sum"],
                                         dtype=torch.float32 if c["wide"] else c["dy"].dtype)
        return xm.clip_grad_norm(c["grads"], MAX_NORM, RESCALE), c["flat"]
    if op == "norm":
        return _plain_norm(c)
    if op == "norm_backward":
        return _plain_norm_backward(c)
    if op == "embedding":
        y = c["table"][c["ids"]].float() * EMBED
        if c["none"] is not None:
            y[c["ids"] == c["none"]] = 0.0
        return y.to(c["table"].dtype)
    if op == "embedding_backward":
        return _plain_embedding_backward(c)
    return _plain_clip(c["grads"]), c["flat"]


def _gate(g, kind):
    if kind == "sigmoid":
        return 1 / (1 + torch.exp(-g))
    if kind == "silu":
        return g / (1 + torch.exp(-g))
    return g


def _gate_slope(g, kind):
    if kind == "plain":
        return torch.ones_like(g)
    s = 1 / (1 + torch.exp(-g))
    return s * (1 - s) if kind == "sigmoid" else s * (1 + g * (1 - s))


def _plain_statistics(x, kind):
    if kind == "none":
        return torch.zeros(2, len(x), device=x.device)
    mean = x.mean(1) if kind == "layer" else torch.zeros(len(x), device=x.device)
    return torch.stack([mean, 1 / torch.sqrt((x - mean[:, None]).square().mean(1) + EPS)])


def _hat(x, stats, kind):
    return x if kind == "none" else (x - stats[0][:, None]) * stats[1][:, None]


def _affine(x, w, b):
    x = x if w is None else x * w
    return x if b is None else x + b


def _plain_norm(c):
    r, dt = c["r"].float(), c["r"].dtype
    first = torch.zeros(2, len(r), device=r.device)
    if c["h"] is not None:
        h = c["h"].float()
        first = _plain_statistics(h, c["post"])
        v = _affine(_hat(h, first, c["post"]), c["w1"], c["b1"])
        if c["g"] is not None:
            v = v * _gate(c["g"].float(), c["gate"])
        r = r + ALPHA * (v if c["s"] is None else v * c["s"])
    second = _plain_statistics(r, c["pre"])
    y = None if c["pre"] == "none" else _affine(_hat(r, second, c["pre"]), c["w2"], c["b2"]).to(dt)
    return r.to(dt), y, torch.cat([first, second])


def _through_norm(d, hat, stats, kind):
    if kind == "none":
        return d
    out = d - hat * (d * hat).mean(1, keepdim=True)
    if kind == "layer":
        out = out - d.mean(1, keepdim=True)
    return stats[1][:, None] * out


def _plain_norm_backward(c):
    r, dt, st = c["r"].float(), c["r"].dtype, c["stats"]
    d = torch.zeros_like(r) if c["dout"] is None else c["dout"].float()
    dw2 = db2 = None
    if c["dy"] is not None:
        dy, hat = c["dy"].float(), _hat(r, st[2:], c["pre"])
        dw2, db2 = (dy * hat).sum(0), None if c["b2"] is None else dy.sum(0)
        d = d + _through_norm(dy * c["w2"], hat, st[2:], c["pre"])
    if c["h"] is None:
        return d.to(dt), None, None, None, None, None, dw2, db2
    hat = _hat(c["h"].float(), st[:2], c["post"])
    u = _affine(hat, c["w1"], c["b1"])
    p = d * ALPHA
    a = None if c["g"] is None else _gate(c["g"].float(), c["gate"])
    v = u if a is None else u * a
    ds = None if c["s"] is None else (p * v).sum(0)
    p = p if c["s"] is None else p * c["s"]
    dg = None if a is None else (p * u * _gate_slope(c["g"].float(), c["gate"])).to(dt)
    p = p if a is None else p * a
    dw1 = None if c["w1"] is None else (p * hat).sum(0)
    db1 = None if c["b1"] is None else p.sum(0)
    dh = _through_norm(p if c["w1"] is None else p * c["w1"], hat, st[:2], c["post"])
    return d.to(dt), dh.to(dt), dg, ds, dw1, db1, dw2, db2


def _plain_embedding_backward(c):
    ids, dy = c["ids"], c["dy"].float() * EMBED
    if c["none"] is not None:
        dy = dy * (ids != c["none"])[:, None]
    wide = torch.float32 if c["wide"] else c["dy"].dtype
    if c["sum"] is not None:
        total = c["sum"].float().index_add_(0, ids, dy) if not c["wide"] else c["sum"].index_add_(0, ids, dy)
        return c["sum"].copy_(total)
    return torch.zeros(c["v"], c["n"], device=ids.device).index_add_(0, ids, dy).to(wide)


def _plain_clip(grads):
    norm = RESCALE * torch.sqrt(torch.stack([g.float().square().sum() for g in grads]).sum())
    factor = RESCALE * torch.clamp(MAX_NORM / (norm + 1e-6), max=1.0)
    [g.copy_(g.float() * factor) for g in grads]
    return torch.stack([norm, factor])


# ------------------------------------------------------------------ what a pass cannot do without


def work(case):
    c, op = case, case["op"]
    size = 4 if c["dtype"] == "f32" else 2
    if op == "clip":
        matrices, vectors = _shapes(c)
        m, v = (sum(math.prod(s) for s in shapes) for shapes in (matrices, vectors))
        return {"bytes": 2 * (size * m + 4 * v), "flops": 3 * (m + v)}
    t, n = c["t"], c["n"]
    if op in ("norm", "norm_backward"):
        block, gate, pre = c["block"], c["gate"] != "none", c["pre"] != "none"
        weights = (c["post"] != "none") + (c["post"] == "layer") + pre + (c["pre"] == "layer") + c["scaled"]
        if op == "norm":
            return {"bytes": size * t * n * (1 + 2 * block + gate + pre) + 4 * n * weights + 16 * t, "flops": t * n * (12 if block else 5)}
        return {"bytes": size * t * n * (2 + 3 * block + 2 * gate + pre) + 8 * n * weights + 16 * t, "flops": t * n * (36 if block else 10)}
    if op == "embedding":
        return {"bytes": 2 * size * t * n + 8 * t, "flops": t * n}
    out = 4 if c["wide"] else size
    if c["add"]:  # the rows of the batch's tokens, as many as this distribution names
        rows = sum(1 - math.exp(-t * math.log((i + 2) / (i + 1)) / math.log(c["v"] + 1)) for i in range(c["v"]))
        return {"bytes": size * t * n + 2 * out * rows * n + 8 * t, "flops": t * n}
    return {"bytes": size * t * n + out * c["v"] * n + 8 * t, "flops": t * n}


# ------------------------------------------------------------------ in 64 bits


def exact(case, seed):
    """The operators' definitions in 64 bits, each written another way than the plain form: the gates through the logistic
    function, norms through torch's variance and vector norm, gradients by differentiation of the forward definition, the lookup's
    gradient token by token in sorted order, the norm of all gradients as one vector's."""
    s = prepare(case, seed)
    op = case["op"]
    up = lambda x: None if x is None else x.double()
    if op == "norm":
        out, y, stats = _exact_forward(*(up(s[k]) for k in ("r", "h", "g", "s", "w1", "b1", "w2", "b2")), case)
        return out, y, stats
    if op == "norm_backward":
        return _exact_backward(case, s, up)
    if op == "embedding":
        on = torch.ones_like(s["ids"]) if s["none"] is None else (s["ids"] != s["none"]).long()
        return torch.index_select(s["table"].double(), 0, s["ids"]) * (EMBED * on.double())[:, None]
    if op == "embedding_backward":
        total = torch.zeros(case["v"], case["n"], dtype=torch.float64, device="cuda")
        ids, order = torch.sort(s["ids"])
        counts = torch.bincount(ids, minlength=case["v"])
        ends = torch.cumsum(counts, 0)
        for row in torch.nonzero(counts).flatten().tolist() if case["t"] <= 4096 else []:
            total[row] = EMBED * s["dy"][order[ends[row] - counts[row]:ends[row]]].double().sum(0)
        if case["t"] > 4096:  # as differences of running sums, a slab of columns at a time
            for at in range(0, case["n"], 256):
                run_ = torch.zeros(case["t"] + 1, min(256, case["n"] - at), dtype=torch.float64, device="cuda")
                torch.cumsum(s["dy"][order, at:at + 256].double(), 0, out=run_[1:])
                total[:, at:at + 256] = EMBED * (run_[ends] - run_[ends - counts])
        if s["none"] is not None:
            total[s["none"]] = 0.0
        return total if s["sum"] is None else total + s["sum"].double()
    norm = RESCALE * torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(x, dtype=torch.float64) for x in s["grads"]]))
    factor = RESCALE * min(1.0, MAX_NORM / (float(norm) + 1e-6))
    flat = [x.double() for x in s["flat"]]
    [v.mul_(factor) for x, shapes in zip(flat, _shapes(case)) for v in _views(x, shapes, case["gap"])]
    return torch.stack([norm, torch.full_like(norm, factor)]), flat


def _exact_moments(x, kind):
    if kind == "none":
        return torch.zeros(2, len(x), dtype=x.dtype, device=x.device)
    if kind == "layer":
        var, mean = torch.var_mean(x, 1, correction=0)
    else:
        mean = torch.zeros(len(x), dtype=x.dtype, device=x.device)
        var = torch.linalg.vector_norm(x, dim=1) ** 2 / x.shape[1]
    return torch.stack([mean, torch.rsqrt(var + EPS)])


def _exact_norm(x, kind, w, b):
    if kind == "none":
        return x
    mean, rho = _exact_moments(x, kind)
    x = torch.sub(x, mean[:, None]) / (1 / rho)[:, None]
    return torch.addcmul(torch.zeros_like(x) if b is None else b.expand_as(x), x, w.expand_as(x))


def _exact_branch(h, g, s, w1, b1, case):
    v = _exact_norm(h, case["post"], w1, b1)
    if g is not None:
        v = v * {"plain": lambda: g, "sigmoid": lambda: torch.sigmoid(g), "silu": lambda: g * torch.sigmoid(g)}[case["gate"]]()
    return ALPHA * v * (1.0 if s is None else s)


def _exact_forward(r, h, g, s, w1, b1, w2, b2, case):
    first = torch.zeros(2, len(r), dtype=r.dtype, device=r.device)
    if h is not None:
        first = _exact_moments(h, case["post"])
        r = r + _exact_branch(h, g, s, w1, b1, case)
    y = None if case["pre"] == "none" else _exact_norm(r, case["pre"], w2, b2)
    return r, y, torch.cat([first, _exact_moments(r, case["pre"])])


def _exact_backward(case, s, up):
    """By torch's differentiation of the forward definition."""
    leaf = {k: up(s[k]) for k in ("r", "h", "g", "s", "w1", "b1", "w2", "b2")}
    on = {k: v.requires_grad_(True) for k, v in leaf.items() if v is not None}
    d = torch.zeros_like(leaf["r"]) if s["dout"] is None else s["dout"].double()
    got = {}
    if s["dy"] is not None:
        wanted = [k for k in ("r", "w2", "b2") if k in on]
        y = _exact_norm(leaf["r"], case["pre"], leaf["w2"], leaf["b2"])
        got.update(zip(wanted, torch.autograd.grad(y, [on[k] for k in wanted], s["dy"].double())))
        d = d + got["r"]
    if leaf["h"] is not None:
        wanted = [k for k in ("h", "g", "s", "w1", "b1") if k in on]
        v = _exact_branch(leaf["h"], leaf["g"], leaf["s"], leaf["w1"], leaf["b1"], case)
        got.update(zip(wanted, torch.autograd.grad(v, [on[k] for k in wanted], d)))
    return (d.detach(), *(got.get(k) for k in ("h", "g", "s", "w1", "b1", "w2", "b2")))
