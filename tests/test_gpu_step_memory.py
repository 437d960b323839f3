"""What the step's operators do with a caller's workspace."""
import pytest
import torch

import paper_2510_21048_amd as xm
from test_gpu_ops import BF, FF, log

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("add", [False, True])
def test_one_workspace_for_every_smaller_batch(add):
    """Of the size of the largest batch: ragged ones on either side of where runs change take it, and give the bits that their own gives."""
    vocab, n, most = 5000, 72, 20000
    g = torch.Generator().manual_seed(17)
    dy, ids = torch.randn(most, n, generator=g).to(BF).cuda(), torch.randint(0, vocab, (most,), generator=g).cuda()
    hold = torch.empty(xm.xmem_embedding_backward_workspace_bytes(most, vocab, n) + 4096, dtype=torch.uint8, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    for t in (most, 16385, 16384, 16383, 9000, 2049, 300):
        need = hold.numel() - 4096
        hold.fill_(255)
        got = torch.ones(vocab, n, device="cuda")
        log(f"[step] embedding_backward {t} tokens, workspace of {most}, add={add}")
        assert xm.xmem_embedding_backward(dy, n, ids, t, vocab, n, xm.XMEM_BF16, 0.5, xm.XMEM_NO_PADDING, add, xm.XMEM_F32, got, n, hold, need, stream) == 0
        torch.cuda.synchronize()
        assert bool((hold[need:] == 255).all())
        want = xm.embedding_backward(dy[:t], ids[:t], vocab, 0.5, into=torch.ones(vocab, n, device="cuda") if add else None, dtype=FF)
        assert torch.equal(got, want)


def test_vectors_and_tokens_in_what_is_overwritten_are_refused():
    """Scale, weights, biases, statistics or tokens that lie in what a call overwrites: refused before anything is written."""
    n = 24
    flat = torch.randn(2000, device="cuda")
    over, before = flat[200:680].view(10, 48)[:, :n], flat.clone()
    other, w = torch.randn(10, n, device="cuda"), torch.randn(n, device="cuda")
    stats, ids = torch.ones(4, 10, device="cuda"), torch.arange(10, device="cuda")
    inside, behind = flat[248:272], flat[700:724]
    forward = lambda **how: xm.residual_norm_forward(over, other, in_place=True, **dict(dict(post="layer", pre="layer"), **how))
    backward = lambda **how: xm.residual_norm_backward(other, over, other, how.pop("stats", stats), other, in_place=True,
                                                       **dict(dict(post="layer", pre="layer"), **how))
    for name in ("scale", "post_weight", "post_bias", "pre_weight", "pre_bias"):
        for call in (forward, backward):
            with pytest.raises(xm.XmemError, match=name + ": shares memory"):
                call(**{name: inside})
            assert torch.equal(flat, before)
            call(**{name: w})
            flat.copy_(before)
            call(**{name: behind})
            flat.copy_(before)
    with pytest.raises(xm.XmemError, match="stats: shares memory"):
        backward(stats=flat[170:210].view(4, 10))
    mine = flat[600:620].view(torch.int64)
    with pytest.raises(xm.XmemError, match="ids: shares memory"):
        xm.embedding_backward(other, mine, 10, into=over)
    torch.cuda.synchronize()
    assert torch.equal(flat, before)
    xm.embedding_backward(other, ids, 10, into=over)
    torch.cuda.synchronize()
    assert torch.equal(over, before[200:680].view(10, 48)[:, :n] + other)


def test_one_row_between_the_rows_that_are_overwritten_is_taken():
    """A single token's row of dy, and vectors, between the rows of what a call overwrites: the bits of copies elsewhere."""
    n = 24
    flat = torch.randn(500, device="cuda")
    over, between, before = flat[:480].view(10, 48)[:, :n], flat[24:48], flat.clone()
    one = torch.tensor([3], device="cuda")
    want = xm.embedding_backward(between.clone().view(1, n), one, 10, into=over.clone())
    got = xm.embedding_backward(between.view(1, n), one, 10, into=over)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(between, before[24:48])
    flat.copy_(before)
    h = torch.randn(10, n, device="cuda")
    want = xm.residual_norm_forward(over.clone(), h, scale=between.clone())
    got = xm.residual_norm_forward(over, h, scale=between, in_place=True)
    torch.cuda.synchronize()
    assert got[0] is over and torch.equal(over, want[0]) and torch.equal(got[1], want[1]) and torch.equal(between, before[24:48])


def test_a_workspace_on_an_operand_is_refused():
    """One that lies on an input or on what is overwritten: refused before anything is written, and taken beside them."""
    g = torch.Generator().manual_seed(23)
    t, n, vocab = 300, 72, 20000  # a table whose gradient needs a workspace
    hold = torch.randn(1 << 21, generator=g).cuda()
    before, raw = hold.clone(), hold.view(torch.uint8)
    x, h, dy = hold[:t * n].view(t, n), hold[30000:30000 + t * n].view(t, n), hold[60000:60000 + t * n].view(t, n)
    ids = torch.randint(0, vocab, (t,), generator=g).cuda()
    out, _, stats = xm.residual_norm_forward(x, h, save_stats=True, pre_weight=hold[90000:90000 + n])
    w, into, grads = hold[90000:90000 + n], hold[100000:100000 + vocab * n].view(vocab, n), [hold[:17], hold[500000:500100]]
    calls = {"norms": (lambda ws: xm.residual_norm_backward(dy, None, out, stats, h, pre_weight=w, workspace=ws), (60000, 90000, 30000)),
             "in place": (lambda ws: xm.residual_norm_backward(dy, x, out, stats, h, pre_weight=w, in_place=True, workspace=ws), (0, 60000, 90000)),
             "table": (lambda ws: xm.embedding_backward(dy, ids, vocab, into=into, workspace=ws), (60000, 100000, 400000)),
             "clip": (lambda ws: xm.clip_grad_norm(grads, 1.0, workspace=ws), (0, 500000))}
    assert xm.xmem_embedding_backward_workspace_bytes(t, vocab, n) > 0
    torch.cuda.synchronize()
    for name, (call, at) in calls.items():
        for a in at:
            a = a // 64 * 64  # a 256-byte boundary
            with pytest.raises(xm.XmemError):
                call(raw[4 * a:4 * a + (1 << 20)])
            torch.cuda.synchronize()
            assert torch.equal(hold, before), name
        log(f"[step] {name} with a workspace beside its operands")
        call(torch.empty(1 << 22, dtype=torch.uint8, device="cuda"))
        torch.cuda.synchronize()
        hold.copy_(before)
