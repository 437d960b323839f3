"""Norm gradients of a batch in which a row lies far out, so that its mean times its reciprocal deviation passes 32 bits while the
row's own normed values are 0: a row that a workgroup takes but the batch does not have is not multiplied with it, nor is what lies
behind a row's end."""
import pytest
import torch

import paper_2510_21048_amd as xm
import step_reference as ref
from test_gpu_ops import BF, FF, HF, log, within
from test_gpu_step_norm import NAMES

pytestmark = pytest.mark.gpu

EPS = 1e-30  # of a row of equal values: rho is 1e15
FAR = {BF: 2.0 ** 84, HF: 32768.0, FF: 2.0 ** 84}  # 2^84 1e15 passes 2^128; in float16 nothing does, and all is as elsewhere


def gradients(t, n, dtype, seed):
    """Row 0 of h and of the sum is FAR everywhere; its sum of n is exact, and so is its mean."""
    g = torch.Generator().manual_seed(seed)
    new = lambda *s: torch.randn(*s, generator=g)
    r, h, gate, dy, dout = (new(t, n).to(dtype) for _ in range(5))
    r[0], h[0] = FAR[dtype], FAR[dtype]
    s, w1, b1, w2, b2 = (new(n) for _ in range(5))
    c = dict(r=r, h=h, gate=gate, dy=dy, dout=dout, s=s, w1=w1, b1=b1, w2=w2, b2=b2)
    v = {k: x.cuda() for k, x in c.items()}
    log(f"[step] residual_norm_backward {t} x {n} {dtype}, a far row")
    # the norms' statistics as the forward pass gives them: of h, and of r alone
    first = xm.residual_norm_forward(v["h"], pre="layer", pre_weight=v["w1"], eps=EPS, save_stats=True)[2]
    second = xm.residual_norm_forward(v["r"], pre="layer", pre_weight=v["w2"], eps=EPS, save_stats=True)[2]
    stats = torch.cat([first[2:], second[2:]])
    got = xm.residual_norm_backward(v["dy"], v["dout"], v["r"], stats, v["h"], v["gate"], v["s"], 0.7, post="layer", post_weight=v["w1"],
                                    post_bias=v["b1"], pre="layer", pre_weight=v["w2"], pre_bias=v["b2"], gate_activation="sigmoid")
    torch.cuda.synchronize()
    assert float(stats[0, 0]) == FAR[dtype] == float(stats[2, 0])
    want, bound = ref.backward(c["dy"], c["dout"], c["r"], stats.cpu(), c["h"], c["gate"], c["s"], 0.7, "layer", c["w1"], c["b1"], "layer",
                               c["w2"], "sigmoid")
    return got, want, bound


def check(t, n, dtype, seed):
    """Row 0 of the gradients [t, n] is left out: there a mean's rounding is multiplied with 1e15."""
    got, want, bound = gradients(t, n, dtype, seed)
    for name, a, b, e in zip(NAMES, got, want, bound):
        first = 1 if a.dim() == 2 else 0
        if not first:
            assert bool(a.isfinite().all()), name
        a, b, e = a[first:].double().cpu(), b[first:], e[first:]
        # A row of one element is its own mean, so each has rho 1e15: a rounding of its e (2^-24, of values near 1) times that is 6e7, past
        # float16's 65504.  Where the bound passes what the type holds, infinity is within it.
        a = torch.where(a.isinf() & (b.abs() + e > torch.finfo(dtype).max), b, a)
        within(a, b, e, f"{name} {t} x {n} {dtype}")


@pytest.mark.parametrize("dtype", [BF, HF, FF])
@pytest.mark.parametrize("n", [8, 16, 72, 130, 264, 515, 1032, 2050])
def test_rows_that_are_not_there(n, dtype):
    """Widths of which a workgroup takes several rows, and batches that do not fill it."""
    for t in (2, 3, 65):
        check(t, n, dtype, n + t)


@pytest.mark.parametrize("dtype", [BF, HF, FF])
@pytest.mark.parametrize("n", [1, 2, 3, 5, 7, 16391, 32775])
def test_elements_behind_a_row(n, dtype):
    """Rows shorter than a piece, and long ones that end inside one."""
    for t in (1, 2, 5):
        check(t, n, dtype, n + t)
