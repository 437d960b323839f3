"""The Newton-Schulz update element by element on the GPU, within bounds that a lesser number format or a misplaced piece does not
meet (tests/test_muon_roundings.py shows that on the CPU)."""
import pytest
import torch

import muon_roundings as mr
import ops_reference as ref
import paper_2510_21048_amd as xm
from test_gpu_ops import BF, FF, HF, MUON, log

pytestmark = pytest.mark.gpu


def check(grad, mom, what, norm_bound, element_bound, steps=5):
    m = mom.clone()
    log(f"[ops] muon {what} {tuple(grad.shape)} {grad.dtype} steps={steps}")
    up = xm.muon_update(grad, m, steps=steps)
    torch.cuda.synchronize()
    wm, want = ref.muon(grad, mom, 0.95, True, steps, 1.0)
    # two operations in 32 bits
    assert bool(((m.double() - wm).abs() <= 4 * ref.E * (mom.double().abs() + grad.double().abs())).all()), what
    norm, element = mr.errors(up, want)
    print(f"    norm {norm:.2e} element {element:.2e}", flush=True)
    assert element < element_bound and (norm_bound is None or norm < norm_bound), (what, norm, element)


# small ones, and large tiles, whole and cut, mirrored blocks, k split
SIZES = MUON + [(2, 136, 2048), (60, 520, 1040), (60, 1040, 520), (1, 3000, 2500), (1, 2057, 2120), (2, 72, 9000), (2, 9000, 40)]


@pytest.mark.parametrize("count,r,c", SIZES)
@pytest.mark.parametrize("dtype", [BF, HF, FF])
def test_normal_matrices(count, r, c, dtype):
    g = torch.Generator(device="cuda").manual_seed(r + c)
    grad = (1e-3 * torch.randn(count, r, c, generator=g, device="cuda")).to(dtype)
    mom = 1e-2 * torch.randn(count, r, c, generator=g, device="cuda")
    for steps in (5, 3):
        # a norm over few values is not an average
        check(grad, mom, "normal", mr.norm_bound(r, c) if r * c >= 2000 else None, mr.ELEMENT, steps)


@pytest.mark.parametrize("directions", [1, 2, 8, 16])
@pytest.mark.parametrize("count,r,c", [(2, 256, 300), (1, 300, 256), (1, 200, 700), (3, 1030, 385)])
def test_weak_directions(count, r, c, directions):
    grad = mr.strong(count, r, c, directions, r + directions).cuda()
    check(grad, torch.zeros_like(grad), f"{directions} strong directions", mr.WEAK_NORM, mr.WEAK_ELEMENT)
