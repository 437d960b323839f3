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


def calls():
    """Each operator as a call of a stream, on inputs made beforehand on the current one, with sizes that need a workspace."""
    g = torch.Generator().manual_seed(77)
    new = lambda *s: torch.randn(*s, generator=g).to(BF).cuda()
    x, w, dy, z = new(512, 4096), new(256, 4096), new(512, 256), new(512, 256)
    logits, tokens = new(300, 999), torch.randint(0, 999, (300,), generator=g).cuda()
    f = [torch.randn(300, generator=g).cuda() for _ in range(4)]
    weights, old, refp = f[0].abs(), f[1] - 7, f[3] - 7
    grad, mom = new(2, 512, 300), torch.randn(2, 512, 300, generator=g).cuda()
    return {
        "xmem_linear_forward": lambda s: xm.linear_forward(x[:128], w, activation="gelu", save_z=True, stream=s),
        "xmem_linear_backward": lambda s: xm.linear_backward(dy, x, w, z, "silu", stream=s),
        "xmem_policy_loss": lambda s: xm.policy_loss(logits, tokens, weights, old, f[2], refp, kl_coef=0.1, stream=s),
        "xmem_muon_update": lambda s: (xm.muon_update(grad, mom.clone() if s is None else mom, stream=s),),
    }


@pytest.mark.parametrize("name", ["xmem_linear_forward", "xmem_linear_backward", "xmem_policy_loss", "xmem_muon_update"])
def test_workspace_of_a_given_stream_stays_its_own(name, monkeypatch):
    """What a call on another stream took is not handed to the current one while the call may still run."""
    from paper_2510_21048_amd import ops
    seen = []
    real = getattr(ops, name)

    def spy(*args):
        seen.extend((t.data_ptr(), t.untyped_storage().nbytes()) for t in args if isinstance(t, torch.Tensor) and t.dtype == torch.uint8)
        return real(*args)

    monkeypatch.setattr(ops, name, spy)
    call = calls()[name]
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    log(f"[ops] {name} on a stream of its own")
    call(s.cuda_stream)
    assert len(seen) == 1
    at, size = seen[0]
    for _ in range(3):
        taken = torch.empty(size, dtype=torch.uint8, device="cuda")
        assert taken.data_ptr() + size <= at or at + size <= taken.data_ptr()
    torch.cuda.synchronize()


@pytest.mark.parametrize("name", ["xmem_linear_forward", "xmem_linear_backward", "xmem_policy_loss", "xmem_muon_update"])
def test_given_stream_beside_the_current_one(name):
    """The same bits on a stream that runs late while the current one takes and writes blocks of the same sizes, before and after."""
    call = calls()[name]
    want = call(None)
    torch.cuda.synchronize()
    sizes = [t.nbytes for t in want if t is not None] + [1 << 16, 1 << 20, 1 << 22]
    s = torch.cuda.Stream()

    def flood():
        for size in sizes:
            for _ in range(3):
                torch.empty(size, dtype=torch.uint8, device="cuda").fill_(255)

    flood()
    s.wait_stream(torch.cuda.current_stream())
    torch.cuda._sleep(20_000_000)  # the blocks are written late ...
    flood()
    with torch.cuda.stream(s):
        torch.cuda._sleep(10_000_000)
    log(f"[ops] {name} beside writes")
    got = call(s.cuda_stream)  # ... and the call runs late
    flood()
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert (a is None) == (b is None) and (a is None or torch.equal(a, b))


def test_no_call_drops_a_gradient():
    """Whichever input requires a gradient, each call says so instead of returning results without one."""
    g = torch.Generator().manual_seed(4)
    new = lambda *s: torch.randn(*s, generator=g).to(BF).cuda()
    x, w, r, dy = new(8, 16), new(24, 16), new(8, 24), new(8, 24)
    b, y = torch.randn(24, generator=g).cuda(), torch.randint(0, 24, (8,), generator=g).cuda()
    f = [torch.randn(8, generator=g).cuda() for _ in range(4)]
    for call, args in ((lambda *a: xm.linear_forward(*a), [x, w, b, r]), (lambda *a: xm.linear_backward(*a, "silu"), [dy, x, w, r]),
                       (lambda lg, *a: xm.policy_loss(lg, y, *a), [dy, *f]), (lambda lg, a: xm.token_logp(lg, y, a), [dy, f[0]]),
                       (lambda *a: xm.muon_update(*a), [dy, torch.zeros(8, 24, device="cuda")])):
        call(*args)
        for i in range(len(args)):
            mine = [a.clone().requires_grad_() if i == j else a for j, a in enumerate(args)]
            with pytest.raises(xm.XmemError, match="gradient"):
                call(*mine)
            with torch.no_grad():
                call(*mine)
    torch.cuda.synchronize()


def test_overwritten_inputs_are_seen_by_autograd():
    """A graph that saved the logits, or the momentum, before a call overwrote them raises instead of using the new values."""
    g = torch.Generator().manual_seed(5)
    y = torch.randint(0, 24, (8,), generator=g).cuda()
    f = [torch.randn(8, generator=g).cuda() for _ in range(3)]
    for write, kept in ((lambda t: xm.policy_loss(t, y, *f, in_place=True), False), (lambda t: xm.policy_loss(t, y, *f), True),
                        (lambda t: xm.muon_update(torch.ones(8, 24, device="cuda"), t), False)):
        leaf = torch.randn(8, 24, generator=g).cuda().requires_grad_()
        logits = leaf * 2
        out = logits.square().sum()  # saves logits
        write(logits.detach())
        if kept:
            out.backward()
            assert torch.equal(leaf.grad, 8 * leaf.detach())
        else:
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                out.backward()
    with torch.inference_mode():
        xm.muon_update(torch.ones(8, 24, device="cuda"), torch.zeros(8, 24, device="cuda"))
    torch.cuda.synchronize()


def test_policy_of_more_rows_than_a_launch():
    """2^26 rows and a few: four a workgroup of 256 threads, which is a grid of 2^32 threads, past what one launch may have."""
    t = 2 ** 26 + 5
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(t, 2, generator=g, device="cuda", dtype=HF)
    y = torch.randint(0, 2, (t,), generator=g, device="cuda")
    log("[ops] policy_loss of 2^26 + 5 rows")
    want = torch.nn.functional.logsigmoid((x[:, 0].float() - x[:, 1].float()) * (1 - 2 * y))
    adv = torch.randn(t, generator=g, device="cuda")
    stats, lp, dx = xm.policy_loss(x, y, None, want, adv)
    torch.cuda.synchronize()
    # each value: a few roundings of 32 bits of numbers below 16
    assert float((lp - want).abs().max()) < 16 * 8 * ref.E
    # the ratio is 1 to 1e-5: the loss is minus the mean advantage, and dx = -adv / t (1[j = y] - p_j)
    assert abs(float(stats[0]) + float(adv.double().mean())) < 1e-5 and float(stats[3]) == 0.0
    hit = torch.stack([y == 0, y == 1], 1).float()
    slope = -adv[:, None] / t * (hit - torch.softmax(x.float(), 1))
    # half a unit of float16's subnormals (all of dx are), and 1e-4 of the value
    assert float((dx.float() - slope).abs().max()) <= 2.0 ** -25 + 1e-4 * float(slope.abs().max())


def test_linear_of_more_tiles_than_a_launch():
    """2^30 - 1 rows of one element: tiles of 128 rows in 512 threads are a grid of 2^32 threads, past what one launch may have."""
    m = 2 ** 30 - 1
    x = torch.randn(m, 1, device="cuda", dtype=BF)
    w = torch.randn(1, 1, device="cuda", dtype=BF)
    log("[ops] linear_forward of 2^30 - 1 rows")
    y = xm.linear_forward(x, w)[0]
    torch.cuda.synchronize()
    assert torch.equal(y, x * w)


def test_linear_gradients_of_more_columns_than_a_launch():
    """2^28 columns: their sums take 64 a workgroup of 1024 threads, a grid of 2^32 threads, past what one launch may have."""
    n = 2 ** 28 + 7
    log("[ops] linear_backward of 2^28 + 7 columns")
    dy, x, w = (torch.zeros(*size, device="cuda", dtype=BF) for size in ((0, n), (0, 1), (n, 1)))
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    held = torch.full((n,), math.nan, device="cuda")  # what the memory that db gets holds
    at = held.data_ptr()
    del held
    db = xm.linear_backward(dy, x, w, need_dx=False, need_dw=False)[2]
    torch.cuda.synchronize()
    assert db.data_ptr() == at and db.shape == (n,) and bool((db == 0).all())


@pytest.mark.parametrize("v", [33, 600, 4100, 60000, 140000])
def test_policy_terms_of_weight_nothing(v):
    """What is multiplied by 0 adds 0, however large: a ratio past 32 bits times an advantage of 0, and a KL term past 32 bits
    whose coefficient is 0 (it is still reported)."""
    from test_gpu_ops import policy_check, policy_inputs
    x, y, wt, old, adv, refp = policy_inputs(6, v, torch.float32, 40 + v)
    wt[:] = 0.25
    lp = (x.double()[torch.arange(6), y] - torch.logsumexp(x.double(), 1)).float()
    old[1], adv[1] = lp[1] - 100, 0.0  # exp(100) is past 32 bits
    old[2], adv[2] = -math.inf, 0.0
    log(f"[ops] policy_loss, terms of weight 0, v={v}")
    # 64 bits hold exp(100) 0 = 0; exp(inf) 0 counts as the same
    finite = old.clone()
    finite[2] = lp[2]
    got = xm.policy_loss(x.cuda(), *[a.cuda() for a in (y, wt, old, adv)], clip_low=0.2, clip_high=0.28)
    policy_check(got, x, y, wt, finite, adv, None, 0.0)
    far = refp.clone()
    far[3] = lp[3] + 100
    stats, lp2, dx = xm.policy_loss(x.cuda(), *[a.cuda() for a in (y, wt, old, adv, far)], clip_low=0.2, clip_high=0.28, kl_coef=0.0)
    assert torch.equal(stats[:2], got[0][:2]) and float(stats[2]) == math.inf and torch.equal(stats[3], got[0][3])
    assert torch.equal(lp2, got[1]) and torch.equal(dx, got[2])
    # NaN is none of these
    old[1] = math.nan
    stats, _, dx = xm.policy_loss(x.cuda(), *[a.cuda() for a in (y, wt, old, adv)], clip_low=0.2, clip_high=0.28)
    assert bool(stats[0].isnan()) and bool(dx[1].isnan().all()) and not bool(dx[2].isnan().any())


def test_operators_in_a_graph():
    """A captured step of every operator, replayed on new inputs with eager work and synchronizations between: each replay is the
    eager result, bit for bit."""
    g = torch.Generator(device="cuda").manual_seed(9)
    new = lambda *s: torch.randn(*s, generator=g, device="cuda")
    x, w, dy = new(200, 1000).to(BF), (new(300, 1000) / 30).to(BF), new(200, 300).to(BF)
    y, f = torch.randint(0, 300, (200,), generator=g, device="cuda"), [new(200) for _ in range(3)]
    mom = new(300, 1000)

    def step(m):
        out, z = xm.linear_forward(x, w, activation="gelu", save_z=True)
        dx, dw, db = xm.linear_backward(dy, x, w, z, "gelu")
        stats, lp, dlogits = xm.policy_loss(out, y, None, f[0] - 6, f[1], f[2] - 6, kl_coef=0.1)
        return out, z, dx, dw, db, stats, lp, dlogits, xm.muon_update(dw, m), xm.token_logp(out, y), m

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(mom.clone())
    torch.cuda.current_stream().wait_stream(side)
    graph, held = torch.cuda.CUDAGraph(), mom.clone()
    with torch.cuda.graph(graph):
        got = step(held)
    for i in range(4):
        x.copy_(new(200, 1000))
        dy.copy_(new(200, 300))
        held.copy_(mom)
        want = step(mom.clone())
        torch.cuda.synchronize()
        log(f"[ops] graph replay {i}")
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert torch.equal(a, b)
