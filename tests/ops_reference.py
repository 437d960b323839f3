"""The training operators in 64 bits on the CPU, and how far 32-bit sums and one rounding may be from them.

u = 2^-8 (bfloat16) or 2^-11 (float16) is the most that one rounding moves a value, relative; e = 2^-24 is float32's."""
from __future__ import annotations

import math

import torch

E = 2.0 ** -24
HALF_ULP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
LEAST = {torch.bfloat16: 1e-40, torch.float16: 2.0 ** -25, torch.float32: 1e-44}  # half of the least subnormal
ROOT = math.sqrt(2 / math.pi)


def gate_argument(z, act):
    return 2 * ROOT * (z + 0.044715 * z ** 3) if act == "gelu" else z


def activate(z, act):
    if act == "none":
        return z
    if act == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    return z * torch.sigmoid(gate_argument(z, act))


def slope(z, act):
    if act == "none":
        return torch.ones_like(z)
    if act == "relu":
        return (z > 0).double()
    v = gate_argument(z, act)
    s = torch.sigmoid(v)
    dv = 2 * ROOT * (1 + 3 * 0.044715 * z ** 2) if act == "gelu" else 1.0
    return s + z * s * (1 - s) * dv


def forward(x, w, b, r, act):
    """(y, z) and the bounds of their errors for x, w, r of one 16-bit type."""
    u, least, k = HALF_ULP[x.dtype], LEAST[x.dtype], x.shape[1]
    xd, wd = x.double(), w.double()
    z, mag = xd @ wd.T, xd.abs() @ wd.abs().T
    if b is not None:
        z, mag = z + b.double(), mag + b.double().abs()
    ez = (k + 8) * E * mag                      # a sum of k products in any order
    y = activate(z, act)
    ey = 1.13 * ez + (gate_argument(z, act).abs() + 8) * 2 * E * y.abs() if act in ("gelu", "silu") else ez
    if r is not None:
        y = y + r.double()
    return y, z, u * y.abs() + 2 * ey + least + 2 * E * y.abs(), u * z.abs() + 2 * ez + least


def backward(dy, x, w, z, act):
    """(dx, dw, db) and the bounds of their errors; dz is rounded for the products, not for db."""
    u, least = HALF_ULP[dy.dtype], LEAST[dy.dtype]
    s = slope(z.double(), act)
    dz = dy.double() * s
    # the slope: two terms, each with the gate's relative error
    zz = z.double()
    es = torch.zeros_like(s) if act in ("none", "relu") else (gate_argument(zz, act).abs() + 8) * 4 * E * (s.abs() + 2 * torch.exp(-zz.abs() / 2))
    edz = dy.double().abs() * es + 2 * E * dz.abs()
    rounded = (u * dz.abs() + least if act != "none" else 0) + edz
    xd, wd = x.double(), w.double()
    m, n = dz.shape
    dx, dw = dz @ wd, dz.T @ xd
    bx = rounded @ wd.abs() + (n + 8) * E * (dz.abs() @ wd.abs())
    bw = rounded.T @ xd.abs() + (m + 8) * E * (dz.abs().T @ xd.abs())
    bb = edz.sum(0) + (m + 8) * E * dz.abs().sum(0)
    return (dx, dw, dz.sum(0)), (u * dx.abs() + 1.01 * bx + least, u * dw.abs() + 1.01 * bw + least, 2 * bb + 1e-44)


def policy(x, y, wt, old, adv, ref, low, high, beta, scale=1.0):
    """(stats, logp, dlogits) in 64 bits, for rows of weight other than 0 whose logits are sound."""
    x, wt, old, adv = x.double(), wt.double(), old.double(), adv.double()
    t = torch.arange(len(y))
    on = wt != 0
    lp = torch.where(on, x[t, y] - torch.logsumexp(x, 1), 0.0)
    rho = torch.exp(lp - old)
    free, held = rho * adv, torch.clamp(rho, 1 - low, 1 + high) * adv
    pg = -torch.minimum(free, held)
    grad = torch.where(held < free, 0.0, -free)
    kl = torch.zeros_like(pg)
    if ref is not None:
        d = ref.double() - lp
        kl = torch.exp(d) - d - 1
        grad = grad + beta * (1 - torch.exp(d))
    grad = torch.where(on, grad * wt, 0.0) * scale
    p = torch.softmax(x, 1)
    dx = -grad[:, None] * p
    dx[t, y] += grad
    dx[~on] = 0.0
    sums = [torch.where(on, wt * v, 0.0).sum() for v in (pg, kl, (held < free).double())]
    b = beta if ref is not None else 0.0
    return torch.stack([sums[0] + b * sums[1], *sums]), lp, dx


def logp_bound(x):
    """Absolute error of a log-probability from 32-bit exponentials and sums: each term's relative error goes with its
    distance from the row's maximum; the terms are summed in runs of v / 512 and then as a tree."""
    x = x.double()
    far = torch.where(torch.isfinite(x), (x - x.amax(1, keepdim=True)).abs(), 0.0).amax(1)
    return (40 + x.shape[1] / 512 + 4 * far) * 2 * E


def muon(g, m, mu, nesterov, steps, scale):
    g, m = g.double(), m.double()
    m = mu * m + g
    u = g + mu * m if nesterov else m
    tall = u.shape[-2] > u.shape[-1]
    x = u.mT if tall else u
    x = x / (torch.linalg.matrix_norm(x, keepdim=True) + 1e-7)
    for _ in range(steps):
        p = x @ x.mT
        x = 3.4445 * x + (-4.7750 * p + 2.0315 * (p @ p)) @ x
    return m, (x.mT if tall else x) * scale
