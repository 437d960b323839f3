"""The bounds of the Newton-Schulz tests tell the kernels' number formats from lesser ones: a simulation of the roundings is within
them, and past them once a mechanism is left out or a piece of the result is wrong (no GPU needed)."""
import pytest
import torch

import muon_roundings as mr
import ops_reference as ref


@pytest.mark.parametrize("rows,cols", [(33, 65), (64, 64), (130, 127), (100, 517), (520, 300), (520, 1040)])
def test_normal_matrices(rows, cols):
    g = torch.Generator().manual_seed(rows)
    grad, mom = 1e-3 * torch.randn(1, rows, cols, generator=g), 1e-2 * torch.randn(1, rows, cols, generator=g)
    want = ref.muon(grad, mom, 0.95, True, 5, 1.0)[1]
    got = mr.update(grad, mom)
    norm, element = mr.errors(got, want)
    assert norm < mr.norm_bound(rows, cols) and element < mr.ELEMENT, (norm, element)
    assert mr.errors(mr.update(grad, mom, diagonals=False), want)[0] > mr.norm_bound(rows, cols)
    for wrong in (lambda u: u[..., 8:16, 24:32].zero_(), lambda u: u[..., -1, -8:].mul_(-1), lambda u: u[..., :8, :8].copy_(u[..., :8, :8].mT.clone())):
        moved = got.clone()
        wrong(moved)
        assert mr.errors(moved, want)[1] > mr.ELEMENT


@pytest.mark.parametrize("directions", [1, 2, 8, 16])
@pytest.mark.parametrize("rows,cols", [(256, 300), (300, 256), (200, 700)])
def test_weak_directions(rows, cols, directions):
    grad = mr.strong(1, rows, cols, directions, rows + directions)
    none = torch.zeros_like(grad)
    want = ref.muon(grad, none, 0.95, True, 5, 1.0)[1]
    norm, element = mr.errors(mr.update(grad, none), want)
    assert norm < mr.WEAK_NORM and element < mr.WEAK_ELEMENT, (norm, element)
    norm, element = mr.errors(mr.update(grad, none, halves=False), want)
    assert norm > mr.WEAK_NORM and element > mr.WEAK_ELEMENT, (norm, element)
