"""The embedding gradient's rows without a token: 0 whatever the factor is, in tables that every row searches and in grouped ones."""
import math

import pytest
import torch

import paper_2510_21048_amd as xm
from test_gpu_ops import BF, FF, HF, log

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, HF, FF])
@pytest.mark.parametrize("t,vocab,n", [(6, 40, 5), (20, 70, 24), (300, 900, 515), (0, 40, 24), (20, 50304, 24), (300, 50304, 5), (3000, 900, 24), (0, 50304, 24)])
def test_rows_without_a_token_are_zero(t, vocab, n, dtype):
    """A factor of infinity or NaN has nothing to multiply there, and a negative one makes no negative zeros: all bits are 0."""
    g = torch.Generator().manual_seed(t + vocab)
    ids = torch.randint(0, vocab // 2, (t,), generator=g)
    dy = (torch.rand(t, n, generator=g) + 0.5).to(dtype).cuda()
    empty = torch.ones(vocab, dtype=torch.bool)
    empty[ids] = False
    empty[1] = True  # padding
    for scale in (math.inf, -math.inf, math.nan, -1.5):
        for o in {dtype, FF}:
            log(f"[step] embedding_backward {t} tokens of {vocab}, width {n}, {dtype} -> {o}, scale {scale}")
            got = xm.embedding_backward(dy, ids.cuda(), vocab, scale, 1, dtype=o)
            torch.cuda.synchronize()
            bits = got.view(torch.int32 if o == FF else torch.int16).cpu()
            assert bool((bits[empty] == 0).all())
            named = got.cpu()[~empty]
            assert bool((named.isnan() if math.isnan(scale) else named == scale).all()) if scale != -1.5 else bool((named < 0).all())
