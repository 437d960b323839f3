"""The memory of the calls of include/ops/xmem_step.h on the host (no GPU needed): their workspaces' sizes."""
import pytest

import paper_2510_21048_amd as xm
from test_step_abi import EWORKSPACE, table_grad


@pytest.mark.parametrize("vocab,width", [(100, 64), (900, 515), (1021, 1024), (50304, 1024), (50304, 5), (200000, 64)])
def test_embedding_backward_workspace_never_shrinks(vocab, width):
    """A buffer that holds the largest batch holds every smaller one."""
    size, last = xm.xmem_embedding_backward_workspace_bytes, 0
    for t in [*range(0, 40000), *range(40000, 1 << 20, 997), 1 << 24, (1 << 31) - 1]:
        now = size(t, vocab, width)
        assert now >= last, (t, last, now)
        last = now


def test_norm_backward_workspace_never_shrinks():
    for width in (1, 7, 64, 1021, 4096, 16384, 40000):
        for dtype in (xm.XMEM_BF16, xm.XMEM_F32):
            sizes = [xm.xmem_residual_norm_backward_workspace_bytes(t, width, dtype) for t in [*range(0, 40000), *range(40000, 1 << 20, 997)]]
            assert sizes == sorted(sizes)


def test_embedding_backward_workspace():
    """A grouped table's: one byte less, none, or one that begins between 256-byte boundaries."""
    for t in (300, 16383, 16384, 20000):
        need = xm.xmem_embedding_backward_workspace_bytes(t, 50304, 64)
        assert need > 0
        for over in (dict(size=need - 1), dict(ws=None), dict(ws=(1 << 20) + 8)):
            assert table_grad(t=t, vocab=50304, **over) == EWORKSPACE
            assert table_grad(t=t, vocab=50304, add=1, **over) == EWORKSPACE
