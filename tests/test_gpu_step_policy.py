"""The example step with normed blocks: it runs, its memory is what the estimate says, and its gradients are the loss's."""
import math

import pytest
import torch

from test_gpu_policy_step import example
from test_gpu_step_norm import definition

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hidden,layers,vocab,tokens", [(256, 4, 1024, 512), (136, 2, 1021, 77)])
def test_normed_step_runs_and_its_peak_is_estimated(hidden, layers, vocab, tokens):
    got = example().train(hidden, layers, vocab, tokens, steps=3, normed=True)
    print(got, flush=True)
    assert all(math.isfinite(x) for x in got["loss"])
    # every tensor of the step is in the trace; the device's allocator hands out blocks up to 1 MiB too large unsplit
    assert got["estimated"][0] <= got["measured"][0] <= 1.05 * got["estimated"][0] + 2**20
    assert got["estimated"][1] >= got["estimated"][0]


def test_normed_gradients():
    """Against autograd in 64 bits.  Some 16 roundings to bfloat16 a block, forward and back, and 4 at the ends, each at most 2^-8 of a
    tensor's norm and in unrelated directions, doubled by the norms' gradients: 2 sqrt(36) 2^-8 = 4.7e-2 of a gradient's norm."""
    ex = example()
    hidden, layers, vocab, tokens = 136, 2, 203, 150
    net = ex.NormedPolicy(hidden, layers, vocab, tokens, seed=3)
    g = torch.Generator(device="cuda").manual_seed(4)
    net.down.mul_(10)  # so that the blocks matter
    for v in net.vectors():
        v.add_(0.1 * torch.randn(v.shape, generator=g, device="cuda"))
    ids, y = (torch.randint(0, vocab, (tokens,), generator=g, device="cuda") for _ in range(2))
    adv, weights = torch.randn(tokens, generator=g, device="cuda"), torch.full((tokens,), 1.0 / tokens, device="cuda")
    old = net.logp(ids, y)  # ratios of 1: none is clipped
    stats, _, grads = net.gradients(ids, y, weights, old, adv, old - 0.1, ex.Ledger())
    torch.cuda.synchronize()
    names = ["table", "up", "down", "head", "scale", "post", "pre", "first", "up_b", "down_b"]
    p = {k: getattr(net, k).double().cpu().requires_grad_() for k in names}
    b = lambda **k: {**dict.fromkeys(("r", "h", "g", "s", "w1", "b1", "w2", "b2")), **k}
    x = p["table"][ids.cpu()]
    a = definition(b(r=x, w2=p["first"]), 1.0, "none", "rms", "none")[1]
    for i in range(layers):
        o = torch.nn.functional.gelu(a @ p["up"][i].T + p["up_b"][i], approximate="tanh") @ p["down"][i].T + p["down_b"][i]
        x, a, _ = definition(b(r=x, h=o, s=p["scale"][i], w1=p["post"][i], w2=p["pre"][i]), 1.0, "rms", "rms", "none")
    lp = torch.log_softmax(a @ p["head"].T, 1)[torch.arange(tokens), y.cpu()]
    # the ratio and the KL term at the old log-probabilities as they were given
    rho, d = torch.exp(lp - old.double().cpu()), (old.double().cpu() - 0.1) - lp
    loss = (-rho * adv.double().cpu() + 0.02 * (torch.exp(d) - d - 1)).mean()
    want = torch.autograd.grad(loss, [p[k] for k in names])
    for k, got, w in zip(names, grads, want):
        far = float((got.double().cpu() - w).norm() / w.norm())
        print(f"[step] gradient of {k}: {far:.2e}", flush=True)
        assert far <= 2 * 6 * 2.0 ** -8, (k, far)
