"""The Newton-Schulz update with the roundings that the kernels make, on the CPU: products of half-precision operands, with the
diagonals of P and Q kept apart in 32 bits and X in two halves until the last two steps.  Either can be left out, to see that a
bound tells the difference; so can a piece of the result, as a tile written to the wrong place would leave it."""
from __future__ import annotations

import torch

KX, KP = 256.0, 1024.0
NS = (3.4445, -4.7750, 2.0315)


def half(x):
    return x.float().half().double()


def update(grad, momentum, mu=0.95, nesterov=True, steps=5, scale=1.0, diagonals=True, halves=True):
    """The update in bfloat16 (as doubles): sums are in 64 bits where the kernels' are in 32."""
    g, m = grad.double(), momentum.double()
    m = mu * m + g
    u = g + mu * m if nesterov else m
    tall = u.shape[-2] > u.shape[-1]
    x = u.mT if tall else u
    x = x / (torch.linalg.matrix_norm(x, keepdim=True) + 1e-7) * KX
    hi = half(x)
    lo = half(x - hi) if halves else torch.zeros_like(x)
    eye = torch.eye(x.shape[-2], dtype=x.dtype, device=x.device)
    for i in range(steps):
        if not (i == 0 or i < steps - 2):
            lo = torch.zeros_like(lo)
        p = hi @ hi.mT * (KP / KX ** 2)
        if diagonals:
            d = torch.diagonal(p, dim1=-2, dim2=-1) / KP
            e = half(p * (1 - eye))
            ee = e @ e
            dq = NS[1] * d + NS[2] * (torch.diagonal(ee, dim1=-2, dim2=-1) / KP ** 2 + d * d)
            q = half((NS[1] * e + NS[2] * (ee / KP + (d[..., :, None] + d[..., None, :]) * e)) * (1 - eye))
            x = (NS[0] + dq)[..., None] * (hi + lo) + q @ hi / KP
        else:
            e = half(p)
            x = NS[0] * (hi + lo) + half(NS[1] * e + NS[2] * (e @ e) / KP) @ hi / KP
        hi = half(x)
        lo = half(x - hi) if halves and i + 1 < steps - 2 else torch.zeros_like(x)
    out = x if steps else hi + lo
    return ((out.mT if tall else out) * (scale / KX)).float().bfloat16().double()


def norm_bound(rows, cols):
    """Of |error| / |update| after up to five steps on matrices of normal values: the result's rounding leaves 1.66e-3 (relative
    roundings between 2^-9 and 2^-8, uniform), the products 0.3e-3 to 0.8e-3 with the diagonals apart and 0.9e-3 to 1.7e-3 without.
    The root of the sum of squares with 0.82e-3, where averages are over many values; with 1.2e-3 where they are not."""
    return 1.85e-3 if min(rows, cols) >= 256 else 2.05e-3


# Of an element's error past its rounding, in units of the update's root mean square: ten of the 0.8e-3 above.
ELEMENT = 8e-3
# The same where a few directions hold nearly all of a gradient.  With the second halves: 1.7e-3 to 2.2e-3, elements 1e-2 at most;
# without them 4.6e-3 to 2e-2, elements 5e-2 and more.
WEAK_NORM, WEAK_ELEMENT = 3e-3, 2.5e-2


def errors(got, want):
    """(largest |error| / |update| of a matrix, largest error of an element past half a unit of bfloat16 in root mean squares)."""
    off = (got.double() - want).abs()
    rms = want.square().mean((-2, -1), keepdim=True).sqrt()
    norm = off.flatten(-2).norm(dim=-1) / want.flatten(-2).norm(dim=-1)
    past = ((off - 2.0 ** -8 * want.abs()) / rms).nan_to_num(nan=float("inf"))
    return float(norm.max()), float(past.max())


def strong(count, rows, cols, directions, seed):
    """A gradient of a few strong directions over weak noise."""
    g = torch.Generator().manual_seed(seed)
    few = torch.randn(count, rows, directions, generator=g) @ torch.randn(count, directions, cols, generator=g)
    return few + 0.05 * torch.randn(count, rows, cols, generator=g)
