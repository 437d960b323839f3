"""The norm of many gradients and their clipping on the GPU against 64 bits."""
import math

import pytest
import torch

import paper_2510_21048_amd as xm
from ops_reference import E, HALF_ULP, LEAST
from test_gpu_ops import BF, FF, HF, log, within

pytestmark = pytest.mark.gpu


def check(grads, max_norm, scale):
    """The norm is a 64-bit sum rounded once (and the factor, from it); a gradient is multiplied by the rounded factor and rounded."""
    c = [g.double().cpu() for g in grads]
    norm = scale * math.sqrt(sum(float(x.square().sum()) for x in c))
    factor = scale * min(1.0, max_norm / (norm + 1e-6))
    stats = xm.clip_grad_norm(grads, max_norm, scale)
    torch.cuda.synchronize()
    got = stats.double().cpu().tolist()
    assert stats.dtype == FF and abs(got[0] - norm) <= 1.001 * E * norm + 1e-44 and abs(got[1] - factor) <= 1.001 * E * factor + 1e-44, (got, norm, factor)
    for i, (g, x) in enumerate(zip(grads, c)):
        want = x * got[1]
        within(g, want, HALF_ULP[g.dtype] * want.abs() * 1.001 + 2 * E * want.abs() + LEAST[g.dtype], f"gradient {i} {tuple(g.shape)}")
    return stats


def new(g, *shape, dtype=FF, size=1.0):
    return (size * torch.randn(*shape, generator=g)).to(dtype).cuda()


@pytest.mark.parametrize("dtype", [BF, HF, FF])
def test_one_gradient(dtype):
    g = torch.Generator().manual_seed(1)
    for n in (1, 2, 3, 7, 8, 9, 255, 2047, 2048, 2049, 8191, 8192, 8193, 100003, 3000000):
        log(f"[step] clip_grad_norm {n} {dtype}")
        check([new(g, n, dtype=dtype)], 0.5, 1.0)


# none clipped, all clipped, scaled up and down, to 0, the norm alone
CASES = [(1e9, 1.0), (1.0, 1.0), (1.0, 3.0), (math.inf, 0.125), (1e9, 0.5), (0.0, 1.0), (math.inf, 1.0), (1.0, 0.0)]


@pytest.mark.parametrize("max_norm,scale", CASES)
@pytest.mark.parametrize("count", [2, 64, 65, 127, 128, 129, 300])
def test_many_gradients(count, max_norm, scale):
    """Of every type and size, some empty, None or transposed, more than one launch takes."""
    g = torch.Generator().manual_seed(count)
    grads = []
    for i in range(count):
        dtype = (BF, HF, FF)[i % 3]
        shape = [(i + 1,), (0,), (3, i + 1), (1,), (33, 70), (2, 3, i + 5), (5000,)][i % 7]
        grads.append(new(g, *shape, dtype=dtype, size=(1.0, 1e-3, 100.0)[i % 2]))
    grads[-1] = new(g, 40, 24).mT
    log(f"[step] clip_grad_norm of {count}, limit {max_norm}, scale {scale}")
    kept = [x.clone() for x in grads]
    stats = check(grads, max_norm, scale)
    if float(stats[1]) == 1.0:
        assert all(torch.equal(a, b) for a, b in zip(grads, kept))
    with_none = [None, *kept, None]
    assert torch.equal(xm.clip_grad_norm(with_none, max_norm, scale), stats)
    assert all(torch.equal(a, b) for a, b in zip(grads, kept))  # the same inputs, the same bits


def test_gradients_between_16_byte_boundaries():
    """Neighbours in one buffer at every offset: what lies between them stays."""
    g = torch.Generator().manual_seed(5)
    for dtype in (BF, HF, FF):
        for gap in (1, 3, 5):
            flat = new(g, 70000, dtype=dtype)
            before, at, grads = flat.clone(), 1, []
            free = torch.ones(70000, dtype=torch.bool)
            for n in (1, 2, 5, 16, 31, 4099, 9000, 17, 33000):
                grads.append(flat[at:at + n])
                free[at:at + n] = False
                at += n + gap
            log(f"[step] clip_grad_norm of views {dtype} gap={gap}")
            check(grads, 1.0, 1.0)
            assert torch.equal(flat[free.cuda()], before[free.cuda()])


def test_values_far_out():
    """Squares past 32 bits, and far below them."""
    g = torch.Generator().manual_seed(6)
    for size in (1e25, 1e-25):
        check([new(g, 5000, size=size), new(g, 77, dtype=BF, size=size)], size, 1.0)
    stats = xm.clip_grad_norm([torch.zeros(100, device="cuda")], 1.0)
    assert stats.cpu().tolist() == [0.0, 1.0]
    # an infinite norm: finite gradients become 0, infinite ones NaN; NaN makes all NaN
    for bad, want in ((math.inf, (0.0, math.nan)), (math.nan, (math.nan, math.nan))):
        a, b = torch.ones(50, device="cuda"), torch.ones(50, dtype=BF, device="cuda")
        b[7] = bad
        stats = xm.clip_grad_norm([a, b], 1.0)
        torch.cuda.synchronize()
        assert (math.isnan(float(stats[0])) if math.isnan(bad) else float(stats[0]) == bad)
        assert bool((a.isnan() if math.isnan(want[0]) else a == 0).all()) and bool(b[7].isnan())
        alone = torch.full((4,), bad, device="cuda")
        assert not math.isfinite(float(xm.clip_grad_norm([alone], math.inf)[0])) and bool((alone == bad).all() if bad == math.inf else alone.isnan().all())


def test_same_gradient_twice_is_refused():
    a, b = torch.ones(100, device="cuda"), torch.ones(100, device="cuda")
    for bad in ([a, b, a], [a, a[10:20]], [b[50:], a, b[:51]]):
        with pytest.raises(xm.XmemError):
            xm.clip_grad_norm(bad, 1.0)
    torch.cuda.synchronize()
    assert bool((a == 1).all()) and bool((b == 1).all())
    assert abs(float(xm.clip_grad_norm([a, a], math.inf)[0]) - math.sqrt(200)) < 1e-5  # the norm alone takes them


def test_large_gradient_past_32_bits():
    """More than 2^32 bytes of one gradient, its ends looked at."""
    n = (1 << 31) + 12345
    a = torch.ones(n, dtype=BF, device="cuda")
    log("[step] clip_grad_norm of 2^31 + 12345 elements")
    stats = xm.clip_grad_norm([a[:17], a[17:]], 1.0)
    torch.cuda.synchronize()
    norm = math.sqrt(n)
    assert abs(float(stats[0]) - norm) <= 1e-7 * norm
    want = float(torch.tensor(1.0 / norm).to(BF))
    assert all(float(x) == want for x in (a[0], a[16], a[17], a[n // 2], a[-1])) and bool((a.view(torch.int16)[::4097] == a.view(torch.int16)[0]).all())
