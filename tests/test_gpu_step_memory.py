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
