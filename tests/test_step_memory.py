"""The memory of the calls of include/ops/xmem_step.h on the host (no GPU needed): their workspaces' sizes, and what they refuse to
overwrite."""
import pytest
import torch

import paper_2510_21048_amd as xm
from paper_2510_21048_amd.ops_step import _apart
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


def test_what_is_overwritten_is_apart_from_every_input():
    """Matrices, vectors, statistics and tokens, each before, on and behind what a call overwrites."""
    flat = torch.zeros(1000)
    over = flat[100:484].view(8, 48)[:, :24]  # rows of 24 elements, 48 apart; the last ends at 460
    row = lambda at, n: flat[at:at + n]
    for free in (row(0, 100), row(460, 100), row(0, 0), row(110, 0)):
        _apart(over, "over", x=free)
        _apart(over, "over", x=free, y=None)
    for bad in (row(0, 101), row(459, 1), row(100, 24), row(123, 1), row(123, 2), row(147, 2), row(148, 1), row(436 - 24, 25), row(0, 1000)):
        with pytest.raises(xm.XmemError, match="vector: shares memory with over"):
            _apart(over, "over", matrix=row(0, 100).view(4, 25), vector=bad)
    stats, ids = row(60, 400).view(torch.int32), flat[0:102].view(torch.int64)
    for bad in (stats, stats.view(4, 100), ids, ids[50:]):
        with pytest.raises(xm.XmemError, match="shares memory"):
            _apart(over, "over", x=bad)
    _apart(over, "over", ids=ids[:50], stats=row(460, 400).view(4, 100))
    # matrices as before: halves of one, and neighbours
    both = flat[:960].view(10, 96)
    for a, b, apart in ((both[:, :48], both[:, 48:], True), (both[:, 48:], both[:, :48], True), (both[:5], both[5:], True), (both[:, :48], both[:, 47:95], False),
                        (both[:, :48], both[1:, :48], False), (both[:, 48:], both[:9, 47:95], False), (both, both, False), (both[:6], both[5:], False)):
        if apart:
            _apart(a, "over", x=b)
        else:
            with pytest.raises(xm.XmemError, match="shares memory"):
                _apart(a, "over", x=b)


def test_what_lies_between_two_rows_is_apart():
    """One row, a vector or a whole small matrix in the gap between two rows of what is overwritten, up to both of its ends."""
    flat = torch.zeros(1000)
    over = flat[100:484].view(8, 48)[:, :24]
    row = lambda at, n: flat[at:at + n]
    for free in (row(124, 24), row(124, 1), row(147, 1), row(412, 24), row(130, 6), row(124, 24).view(1, 24), row(172, 24).view(4, 6),
                 flat[124:].as_strided((1, 24), (1000, 1))):
        _apart(over, "over", x=free)
        _apart(free, "free", x=over)
    for bad in (row(123, 25), row(123, 1), row(124, 25), row(148, 1), row(412, 25), row(172, 25).view(5, 5)):
        for a, b in ((over, bad), (bad, over)):
            with pytest.raises(xm.XmemError, match="shares memory"):
                _apart(a, "over", x=b)
