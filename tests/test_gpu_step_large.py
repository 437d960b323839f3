"""Sizes from which the step's operators take another way: outputs past the caches, and more workgroups than a launch has."""
import pytest
import torch

import paper_2510_21048_amd as xm
from test_gpu_ops import BF, FF, HF, log
from test_gpu_step_norm import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t,n,dtype,pre", [(8200, 16381, BF, "none"), (4200, 16381, HF, "rms"), (66000, 1021, BF, "layer"), (34000, 997, FF, "rms"),
                                           (700000, 100, BF, "rms")])
def test_outputs_past_the_caches(t, n, dtype, pre):
    """256 MiB of outputs and more, rows that end inside a piece: the bits of the same rows in smaller calls, in place too."""
    g = torch.Generator(device="cuda").manual_seed(t)
    r, h = (torch.randn(t, n, generator=g, device="cuda").to(dtype) for _ in range(2))
    w = torch.randn(n, generator=g, device="cuda")
    assert (1 + (pre != "none")) * r.nbytes >= 1 << 28
    how = dict(scale=w, alpha=0.3, post="rms", post_weight=w, pre=pre, pre_weight=None if pre == "none" else w, save_stats=True)
    log(f"[step] residual_norm_forward {t} x {n} {dtype} pre={pre}")
    out, y, stats = xm.residual_norm_forward(r, h, **how)
    few = 3000 if t < 100000 else 50000  # rows whose outputs stay below the limit, and that take the same threads
    for at in range(0, t, few):
        end = min(at + few, t)
        at = max(0, end - few)
        a, b, c = xm.residual_norm_forward(r[at:end], h[at:end], **how)
        assert torch.equal(out[at:end], a) and torch.equal(stats[:, at:end], c) and (y is None or torch.equal(y[at:end], b))
    mine = r.clone()
    got = xm.residual_norm_forward(mine, h, in_place=True, **how)
    assert got[0] is mine and torch.equal(mine, out) and torch.equal(got[2], stats) and (y is None or torch.equal(got[1], y))


@pytest.mark.parametrize("n", [1, 3])
def test_more_rows_than_a_launch(n):
    """2^21 workgroups of 1024 threads are a launch of rows shorter than a piece."""
    g = torch.Generator().manual_seed(n)
    check(g, (1 << 21) + 5, n, FF if n == 3 else BF, 0, "rms", "silu", True, "rms", True)


@pytest.mark.parametrize("vocab,n,dtype,o", [(5, 8, BF, FF), (200000, 8, HF, FF), (7, 3, BF, FF), (50304, 16, FF, FF)])
def test_more_runs_than_a_launch(vocab, n, dtype, o):
    """2^19 runs of 16 entries are a launch of the table gradient's sums: rows that begin in one and go on in the next.  Gradients of small
    whole numbers, so that every sum of 32 bits is exact."""
    t = (1 << 23) + 1007
    g = torch.Generator().manual_seed(vocab)
    dy, ids = torch.randint(-1, 2, (t, n), generator=g), torch.randint(0, vocab, (t,), generator=g)
    ids[::5] = vocab // 2  # a frequent token
    want = torch.zeros(vocab, n, dtype=torch.float64).index_add_(0, ids, dy.double())
    d, i = dy.to(dtype).cuda(), ids.cuda()
    log(f"[step] embedding_backward {t} tokens of {vocab}, width {n}, {dtype}")
    got = xm.embedding_backward(d, i, vocab, 2.0, dtype=o)
    torch.cuda.synchronize()
    assert torch.equal(got.double().cpu(), 2 * want)
    into = torch.ones(vocab, n, dtype=o, device="cuda")
    xm.embedding_backward(d, i, vocab, 2.0, into=into)
    torch.cuda.synchronize()
    assert torch.equal(into.double().cpu(), 2 * want + 1)
