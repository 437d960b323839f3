"""The operators of include/ops/xmem_step.h in 64 bits on the CPU, and how far 32-bit sums and one rounding may be from them.

E = 2^-24 is the most that one rounding to float32 moves a value, relative; HALF_ULP that of an output's type.  A sum whose chains
of additions are at most K long is off by at most K E times the sum of its terms' magnitudes: a row's threads add up at most 32
terms one after another (or n / 1024 pieces of 8) and meet in 6 + 16 additions; a vector's gradient adds up a group's rows (at
most t / 256, where a row is short enough for 256 groups), then a sixteenth of the groups, then sixteen sums."""
from __future__ import annotations

import torch

from ops_reference import E, HALF_ULP, LEAST

ROW = 64  # K of a row's sums, without what a long row adds
# exp2 and the reciprocal are off by a unit (2 E) each, the argument's rounding by |g| E and the scaling by log2(e) as much
GATE = lambda g: (2 * g.abs() + 16) * E


def row_k(n):
    return ROW + n / 1024


def column_k(t):
    return ROW + t / 256


def gate(g, kind):
    """a(g), a'(g) and the bounds of their errors."""
    if kind == "none":
        z = torch.zeros_like(g)
        return g, torch.ones_like(g), z, z
    q = torch.sigmoid(g)
    # 1 / (1 + e) is 0 where e = exp(-g) passes 2^128 and q is subnormal: q is off by at most 2^-126 there, and what q is multiplied
    # with carries that on: g q, q (1 - q) by at most 2^-126, q (1 + g (1 - q)) by at most 2^-126 (1 + |g|)
    least = 2.0 ** -126
    if kind == "sigmoid":
        return q, q * (1 - q), GATE(g) * q + least, GATE(g) * 2 * q + least  # 1 - q is off by q's error
    far = least * (1 + g.abs())
    return g * q, q * (1 + g * (1 - q)), GATE(g) * (g * q).abs() + far, 2 * GATE(g) * q * (1 + g.abs()) + far


def moments(x, ex, kind, eps):
    """mu, rho of x's rows (known within ex) and the bounds of their errors."""
    t, n = x.shape
    if kind == "none":
        z = torch.zeros(t, 1, dtype=x.dtype)
        return z, z, z, z
    k = row_k(n) * E
    mu, emu = torch.zeros(t, 1, dtype=x.dtype), torch.zeros(t, 1, dtype=x.dtype)
    if kind == "layer":
        mu = x.mean(1, keepdim=True)
        emu = k * x.abs().mean(1, keepdim=True) + ex.mean(1, keepdim=True) + 2 * E * mu.abs()
    d, ed = x - mu, ex + emu + E * (x - mu).abs()
    var = d.square().mean(1, keepdim=True)
    evar = (k + 4 * E) * var + (2 * d.abs() * ed + ed * ed).mean(1, keepdim=True) + 2 * E * eps
    rho = (var + eps) ** -0.5
    return mu, rho, emu, rho * (0.5 * evar / (var + eps) + 8 * E + (evar / (var + eps)) ** 2)


def affine(hat, ehat, w, b):
    if w is not None:
        ehat, hat = ehat * w.double().abs() + E * (hat * w).abs(), hat * w.double()
    if b is not None:
        hat = hat + b.double()
        ehat = ehat + E * hat.abs()
    return hat, ehat


def hat(x, ex, mu, rho, emu, erho):
    d = x - mu
    ed = ex + emu + E * d.abs()
    return d * rho, ed * (rho + erho) + d.abs() * erho + E * (d * rho).abs()


def forward(r, h, g, s, alpha, post, w1, b1, pre, w2, b2, act, eps):
    """(out, y, stats) and the bounds of their errors, for r, h, g of one type."""
    u, least = HALF_ULP[r.dtype], LEAST[r.dtype]
    x, z = r.double(), torch.zeros(1, dtype=torch.float64)
    ex = torch.zeros_like(x)
    first = moments(x, ex, "none", eps)
    if h is not None:
        v, zero = h.double(), torch.zeros_like(x)
        ev = zero
        first = moments(v, zero, post, eps)
        if post != "none":
            v, ev = affine(*hat(v, zero, *first), w1, b1)
        f = alpha * (1.0 if s is None else s.double())
        ev, v = (ev + 3 * E * v.abs()) * abs(f), v * f
        if g is not None:
            a, _, ea, _ = gate(g.double(), act)
            ev = ev * a.abs() + v.abs() * ea + ev * ea + E * (v * a).abs()
            v = v * a
        x = x + v
        ex = ev + E * x.abs()
    second = moments(x, ex, pre, eps)
    y = ey = None
    if pre != "none":
        y, e = affine(*hat(x, ex, *second), w2, b2)
        ey = 1.01 * e + u * y.abs() + least
    stats = torch.cat([first[0], first[1], second[0], second[1]], 1).T
    es = torch.cat([first[2], first[3], second[2], second[3]], 1).T
    return (x, y, stats), (1.01 * ex + u * x.abs() + least, ey, 1.01 * es + E * stats.abs() + 1e-44)


def backward(dy, dout, out, stats, h, g, s, alpha, post, w1, b1, pre, w2, act):
    """(dr, dh, dgate, ds, dw1, db1, dw2, db2) and their bounds; stats (float32) and out are given, so exact.  None where there is no
    such input; the vectors' gradients are there whether or not the vector is."""
    first = dout if dy is None else dy
    u, least, (t, n) = HALF_ULP[first.dtype], LEAST[first.dtype], first.shape
    kr, kc = row_k(n) * E, column_k(t) * E
    mu1, rho1, mu2, rho2 = (q[:, None] for q in stats.double())
    d = torch.zeros(t, n, dtype=torch.float64) if dout is None else dout.double()
    ed = torch.zeros_like(d)
    column = lambda v, ev: (v.sum(0), 1.01 * (ev.sum(0) + kc * v.abs().sum(0)) + 1e-44)
    dw2 = db2 = (None, None)

    def through(v, ev, x, mu, rho, kind):
        """rho (v - mean v - xhat mean(v xhat)) and its bound."""
        xh = (x - mu) * rho
        exh = 4 * E * xh.abs()
        m1, m2 = (v * xh).mean(1, keepdim=True), v.mean(1, keepdim=True)
        em1 = (ev * xh.abs() + v.abs() * exh).mean(1, keepdim=True) + (kr + 4 * E) * (v * xh).abs().mean(1, keepdim=True)
        em2 = ev.mean(1, keepdim=True) + (kr + 2 * E) * v.abs().mean(1, keepdim=True)
        if kind != "layer":
            m2, em2 = torch.zeros_like(m2), torch.zeros_like(em2)
        size = v.abs() + m2.abs() + (xh * m1).abs()
        return rho * (v - m2 - xh * m1), rho * (ev + em2 + exh * m1.abs() + xh.abs() * em1 + exh * em1 + 6 * E * size)

    if dy is not None:
        y = dy.double()
        xh = (out.double() - mu2) * rho2
        dw2, db2 = column(y * xh, 5 * E * (y * xh).abs()), column(y, torch.zeros_like(y))
        e = y if w2 is None else y * w2.double()
        add, eadd = through(e, E * e.abs(), out.double(), mu2, rho2, pre)
        d = d + add
        ed = eadd + E * d.abs() + E * add.abs()
    dr, bdr = d, 1.01 * ed + u * d.abs() + least
    if h is None:
        none = (None, None)
        got = [(dr, bdr), none, none, none, none, none, dw2, db2]
        return [v for v, _ in got], [b for _, b in got]
    x = h.double()
    if post != "none":
        xh = (x - mu1) * rho1
        exh = 4 * E * xh.abs()
    else:
        xh, exh = x, torch.zeros_like(x)
    f = torch.full((n,), float(alpha), dtype=torch.float64) * (1.0 if s is None else s.double())
    w, b = (torch.ones(n, dtype=torch.float64) if w1 is None else w1.double()), (torch.zeros(n, dtype=torch.float64) if b1 is None else b1.double())
    inner, einner = xh * w + b, exh * w.abs() + 3 * E * ((xh * w).abs() + b.abs())
    through_gate, egate, dg = d, ed, (None, None)
    if g is not None:
        a, slope, ea, eslope = gate(g.double(), act)
        p = d * f
        v = p * inner * slope
        ev = (ed * f.abs() + 3 * E * p.abs()) * (inner * slope).abs() + p.abs() * (einner * slope.abs() + inner.abs() * eslope) + 4 * E * v.abs()
        dg = (v, 1.02 * ev + u * v.abs() + least)
        through_gate, egate = d * a, ed * a.abs() + d.abs() * ea + E * (d * a).abs()
    ta, ea_ = column(through_gate * xh, egate * xh.abs() + through_gate.abs() * exh + 2 * E * (through_gate * xh).abs())
    tb, eb_ = column(through_gate, egate)
    dw1, db1 = (f * ta, f.abs() * (ea_ + 4 * E * ta.abs())), (f * tb, f.abs() * (eb_ + 4 * E * tb.abs()))
    al = abs(float(alpha))
    ds = (alpha * (w * ta + b * tb), al * (w.abs() * (ea_ + 4 * E * ta.abs()) + b.abs() * (eb_ + 4 * E * tb.abs())))
    q = through_gate * f * w
    eq = egate * (f * w).abs() + 4 * E * q.abs()
    dh, edh = through(q, eq, x, mu1, rho1, post) if post != "none" else (q, eq)
    got = [(dr, bdr), (dh, 1.02 * edh + u * dh.abs() + least), dg, ds, dw1, db1, dw2, db2]
    return [v for v, _ in got], [b for _, b in got]


def table_grad(dy, ids, vocab, scale, padding, into, out_dtype):
    """The table's gradient and its bound: a row's chain is at most as long as its token's rows, and one more scaling and sum."""
    keep = (ids >= 0) & (ids < vocab)
    if padding is not None:
        keep &= ids != padding
    d, i = dy.double()[keep], ids[keep]
    n = dy.shape[1]
    sums, mags = (torch.zeros(vocab, n, dtype=torch.float64).index_add_(0, i, v) for v in (d, d.abs()))
    counts = torch.bincount(i, minlength=vocab).double()[:, None]
    total, size = scale * sums, abs(scale) * mags
    if into is not None:
        total, size = total + into.double(), size + into.double().abs()
    return total, HALF_ULP[out_dtype] * total.abs() + (counts + 4) * E * size + (LEAST[out_dtype] if out_dtype != torch.float32 else 1e-44)
