"""The training operators where a size, a stream, a limit or a value is at an edge; bounds as in test_gpu_ops.py."""
import math

import pytest
import torch

import ops_reference as ref
import paper_2510_21048_amd as xm
from test_gpu_ops import BF, HF, log, rows, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("size", [(64, 64, 65), (128, 129, 68), (512, 64, 1025), (64, 1025, 129), (256, 132, 71), (1024, 192, 67)],
                         ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", [BF, HF])
def test_linear_backward_last_tile_of_few_rows(size, dtype):
    """Operands with their rows contiguous whose last tile holds fewer than eight of them, summed over whole k tiles."""
    m, n, k = size
    g = torch.Generator().manual_seed(m + n + k)
    dy, dyc = rows(g, m, n, dtype, 0)
    x, xc = rows(g, m, k, dtype, 0)
    w, wc = rows(g, n, k, dtype, 0, 1 / math.sqrt(n))
    log(f"[ops] linear_backward {size} {dtype}")
    got = xm.linear_backward(dy, x, w)
    torch.cuda.synchronize()
    want, bound = ref.backward(dyc, xc, wc, dyc, "none")
    for name, a, v, b in zip(("dx", "dw", "db"), got, want, bound):
        within(a, v, b, f"{name} {size}")
