"""The operators of include/ops/xmem_step.h on streams, in graphs, beside autograd and together, as a step uses them."""
import math

import pytest
import torch

import paper_2510_21048_amd as xm
from test_gpu_ops import BF, FF, HF, log
from test_gpu_step_norm import definition

pytestmark = pytest.mark.gpu


def calls():
    """Each operator as a call of a stream, on inputs made beforehand on the current one, with sizes that need a workspace."""
    g = torch.Generator().manual_seed(78)
    new = lambda *s, dtype=BF: torch.randn(*s, generator=g).to(dtype).cuda()
    r, h, gate, dy, dout = (new(300, 520) for _ in range(5))
    w, s = new(520, dtype=FF), new(520, dtype=FF)
    how = dict(post="layer", post_weight=w, post_bias=s, pre="rms", pre_weight=w, gate_activation="silu")
    out, _, stats = xm.residual_norm_forward(r, h, gate, s, 0.5, save_stats=True, **how)
    table, ids, big = new(5000, 264), torch.randint(0, 5000, (3000,), generator=g).cuda(), new(3000, 264)
    grads = [new(700, 33), new(5001, dtype=FF), new(40000, dtype=HF)]
    copies = [[x.clone() for x in grads] for _ in range(2)]

    def clip(mine, s_):
        return (xm.clip_grad_norm(mine, 1.0, stream=s_), *mine)

    return {
        "residual_norm_forward": lambda s_: xm.residual_norm_forward(r, h, gate, s, 0.5, save_stats=True, stream=s_, **how),
        "residual_norm_backward": lambda s_: xm.residual_norm_backward(dy, dout, out, stats, h, gate, s, 0.5, stream=s_, **how),
        "embedding_forward": lambda s_: (xm.embedding_forward(table, ids, 2.0, stream=s_),),
        "embedding_backward": lambda s_: (xm.embedding_backward(big, ids, 5000, stream=s_),),
        # each call takes copies of its own: a clipped gradient's norm is the limit only up to its roundings
        "clip_grad_norm": lambda s_: clip(copies.pop(), s_),
    }


NAMES = ["residual_norm_forward", "residual_norm_backward", "embedding_forward", "embedding_backward", "clip_grad_norm"]


@pytest.mark.parametrize("name", NAMES)
def test_given_stream_beside_the_current_one(name):
    """The same bits on a stream that runs late while the current one takes and writes blocks of the same sizes, before and after."""
    call = calls()[name]
    want = call(None)
    torch.cuda.synchronize()
    sizes = [t.nbytes for t in want if t is not None and t.nbytes] + [1 << 14, 1 << 16, 1 << 20, 1 << 22]
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
    log(f"[step] {name} beside writes")
    got = call(s.cuda_stream)  # ... and the call runs late
    flood()
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert (a is None) == (b is None) and (a is None or torch.equal(a, b)), name


@pytest.mark.parametrize("name", ["residual_norm_backward", "embedding_backward", "clip_grad_norm"])
def test_callers_workspace(name, monkeypatch):
    """A workspace of just the size that is asked for, full of NaN: the same bits, and nothing behind it is written."""
    from paper_2510_21048_amd import ops_step
    call, seen = calls()[name], []
    want = call(None)
    real = ops_step._workspace

    def exact(workspace, need, device):
        hold = torch.full((need // 4 + 64,), math.nan, device=device)
        seen.append((hold, need))
        return real(hold.view(torch.uint8)[:need], need, device)

    monkeypatch.setattr(ops_step, "_workspace", exact)
    got = call(None)
    torch.cuda.synchronize()
    assert len(seen) == 1 and seen[0][1] > 0 and bool(seen[0][0][seen[0][1] // 4:].isnan().all())
    for a, b in zip(want, got):
        assert (a is None and b is None) or torch.equal(a, b)


def test_no_call_drops_a_gradient():
    """Whichever input requires a gradient, each call says so instead of returning results without one."""
    g = torch.Generator().manual_seed(4)
    new = lambda *s: torch.randn(*s, generator=g).cuda()
    x, h, gate, w = new(8, 16), new(8, 16), new(8, 16), new(16)
    stats, ids = new(4, 8).abs(), torch.randint(0, 8, (8,), generator=g).cuda()
    for call, args in ((lambda r, h, g, s, w: xm.residual_norm_forward(r, h, g, s, post="rms", post_weight=w), [x, h, gate, w, w]),
                       (lambda dy, o, st, h, g, s: xm.residual_norm_backward(dy, None, o, st, h, g, s), [x, x, stats, h, gate, w]),
                       (lambda t: xm.embedding_forward(t, ids), [x]), (lambda d, i: xm.embedding_backward(d, ids, 8, into=i), [x, h]),
                       (lambda a, b: xm.clip_grad_norm([a, b], 1.0), [x.clone(), w.clone()])):
        call(*args)
        for i in range(len(args)):
            mine = [a.clone().requires_grad_() if i == j else a.clone() for j, a in enumerate(args)]
            with pytest.raises(xm.XmemError, match="gradient"):
                call(*mine)
            with torch.no_grad():
                call(*mine)
    torch.cuda.synchronize()


def test_outputs_over_other_inputs_are_refused():
    """What a call overwrites shares no element with what else it reads; the halves of one matrix are apart."""
    g = torch.Generator().manual_seed(12)
    both, other = torch.randn(6, 48, generator=g).cuda(), torch.randn(6, 24, generator=g).cuda()
    a, b, c = both[:, :24], both[:, 24:], both[:, 16:40]
    stats, ids = torch.ones(4, 6, device="cuda"), torch.tensor([3, 1, 3], device="cuda")
    for call in (lambda x, y: xm.residual_norm_forward(x, y, in_place=True), lambda x, y: xm.residual_norm_forward(x, other, y, in_place=True),
                 lambda x, y: xm.residual_norm_backward(y, x, other, stats, in_place=True),
                 lambda x, y: xm.residual_norm_backward(other, x, y, stats, in_place=True),
                 lambda x, y: xm.residual_norm_backward(other, x, other, stats, y, in_place=True),
                 lambda x, y: xm.residual_norm_backward(other, x, other, stats, other, y, in_place=True),
                 lambda x, y: xm.embedding_backward(y[2:5], ids, 6, into=x)):
        for x, y in ((a, a), (a, c), (c, a), (c, b), (both.view(12, 24)[:6], both.view(12, 24)[2:8])):
            before = both.clone()
            with pytest.raises(xm.XmemError, match="shares memory"):
                call(x, y)
            assert torch.equal(both, before)
        for x, y in ((a, b), (b, a)):
            call(x, y)
            both.copy_(before)
    want = xm.residual_norm_forward(a.clone(), b.clone())[0]
    assert torch.equal(xm.residual_norm_forward(a, b, in_place=True)[0], want) and torch.equal(a, want) and torch.equal(b, before[:, 24:])


def test_overwritten_inputs_are_seen_by_autograd():
    """A graph that saved what a call overwrites raises instead of using the new values; one that saved what is only read does not."""
    g = torch.Generator().manual_seed(5)
    h, ids = torch.randn(8, 24, generator=g).cuda(), torch.randint(0, 8, (8,), generator=g).cuda()
    stats = torch.ones(4, 8, device="cuda")
    for write, kept in ((lambda t: xm.residual_norm_forward(t, h, in_place=True), False), (lambda t: xm.residual_norm_forward(t, h), True),
                        (lambda t: xm.residual_norm_backward(h, t, h, stats, in_place=True), False),
                        (lambda t: xm.residual_norm_backward(h, t, h, stats), True), (lambda t: xm.embedding_backward(h, ids, 8, into=t), False),
                        (lambda t: xm.embedding_backward(t, ids, 8), True), (lambda t: xm.clip_grad_norm([h.clone(), t], 1e-3), False),
                        (lambda t: xm.clip_grad_norm([t, h], math.inf), True)):
        leaf = torch.randn(8, 24, generator=g).cuda().requires_grad_()
        x = leaf * 2
        out = x.square().sum()  # saves x
        write(x.detach())
        if kept:
            out.backward()
            assert torch.equal(leaf.grad, 8 * leaf.detach())
        else:
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                out.backward()
    torch.cuda.synchronize()


class Net:
    """A policy of normed residual blocks from the package's operators: embedding, blocks of two linear layers, head, policy loss."""

    def __init__(self, hidden, layers, vocab, tokens, seed, dtype=HF):
        g = torch.Generator().manual_seed(seed)
        new = lambda *s, scale=1.0: (scale * torch.randn(*s, generator=g))
        h = hidden
        self.n = layers
        self.p = {"table": new(vocab, h).to(dtype), "head": new(vocab, h, scale=h ** -0.5).to(dtype), "w0": 1 + new(h, scale=0.1)}
        for i in range(layers):
            self.p.update({f"up{i}": new(2 * h, h, scale=h ** -0.5).to(dtype), f"down{i}": new(h, 2 * h, scale=(2 * h) ** -0.5).to(dtype),
                           f"b{i}": new(2 * h, scale=0.1), f"s{i}": 0.5 + new(h, scale=0.1), f"post{i}": 1 + new(h, scale=0.1),
                           f"pre{i}": 1 + new(h, scale=0.1), f"bias{i}": new(h, scale=0.1)})
        self.ids = torch.randint(0, vocab, (tokens,), generator=g)
        self.ids[::7] = vocab - 1  # padding
        self.y = torch.randint(0, vocab, (tokens,), generator=g)
        self.old = new(tokens, scale=0.1) - math.log(vocab)
        self.adv = new(tokens)
        self.padding, self.vocab, self.scale = vocab - 1, vocab, 1.5
        self.names = list(self.p)

    def cuda(self):
        self.p = {k: v.cuda() for k, v in self.p.items()}
        self.ids, self.y, self.old, self.adv = (v.cuda() for v in (self.ids, self.y, self.old, self.adv))
        return self

    def how(self, i):
        p = self.p
        return dict(post="rms", post_weight=p[f"post{i}"], pre="layer", pre_weight=p[f"pre{i}"], pre_bias=p[f"bias{i}"])

    def step(self, max_norm=0.5):
        """(stats of the loss, stats of the clipping, the clipped gradients by name)."""
        p, grads, kept = self.p, {}, []
        x = xm.embedding_forward(p["table"], self.ids, self.scale, self.padding)
        _, y, st0 = xm.residual_norm_forward(x, pre_weight=p["w0"], save_stats=True)
        x0 = x
        for i in range(self.n):
            mid, z = xm.linear_forward(y, p[f"up{i}"], p[f"b{i}"], activation="gelu", save_z=True)
            o = xm.linear_forward(mid, p[f"down{i}"])[0]
            x, y_next, st = xm.residual_norm_forward(x, o, None, p[f"s{i}"], 0.7, save_stats=True, **self.how(i))
            kept.append((y, mid, z, o, x, st))
            y = y_next
        logits = xm.linear_forward(y, p["head"])[0]
        loss, _, dlogits = xm.policy_loss(logits, self.y, None, self.old, self.adv, grad_scale=float(len(self.y)), in_place=True)
        dy, grads["head"], _ = xm.linear_backward(dlogits, y, p["head"], need_db=False)
        dx = None
        for i in reversed(range(self.n)):
            y, mid, z, o, x, st = kept[i]
            dx, do, _, grads[f"s{i}"], grads[f"post{i}"], _, grads[f"pre{i}"], grads[f"bias{i}"] = xm.residual_norm_backward(
                dy, dx, x, st, o, None, p[f"s{i}"], 0.7, in_place=dx is not None, **self.how(i))
            dmid, grads[f"down{i}"], _ = xm.linear_backward(do, mid, p[f"down{i}"], need_db=False)
            dy, grads[f"up{i}"], grads[f"b{i}"] = xm.linear_backward(dmid, y, p[f"up{i}"], z, "gelu")
        dx, _, _, _, _, _, grads["w0"], _ = xm.residual_norm_backward(dy, dx, x0, st0, pre_weight=p["w0"], in_place=True)
        grads["table"] = xm.embedding_backward(dx, self.ids, self.vocab, self.scale, self.padding)
        clip = xm.clip_grad_norm([grads[k] for k in self.names], max_norm, 1.0 / len(self.y))
        return loss, clip, grads

    def exact(self):
        """The loss and its gradients in 64 bits by autograd, from the definitions."""
        p = {k: v.double().cpu().requires_grad_() for k, v in self.p.items()}
        ids, y, old, adv = (v.cpu() for v in (self.ids, self.y, self.old, self.adv))
        b = lambda **k: {**dict.fromkeys(("r", "h", "g", "s", "w1", "b1", "w2", "b2")), **k}
        x = self.scale * p["table"][ids] * (ids != self.padding)[:, None]
        _, a, _ = definition(b(r=x, w2=p["w0"]), 1.0, "none", "rms", "none")
        for i in range(self.n):
            z = a @ p[f"up{i}"].T + p[f"b{i}"]
            o = torch.nn.functional.gelu(z, approximate="tanh") @ p[f"down{i}"].T
            x, a, _ = definition(b(r=x, h=o, s=p[f"s{i}"], w1=p[f"post{i}"], w2=p[f"pre{i}"], b2=p[f"bias{i}"]), 0.7, "rms", "layer", "none")
        lp = torch.log_softmax(a @ p["head"].T, 1)[torch.arange(len(y)), y]
        rho = torch.exp(lp - old.double())
        loss = -torch.minimum(rho * adv, torch.clamp(rho, 0.8, 1.2) * adv).mean()
        return loss.detach(), dict(zip(p, torch.autograd.grad(loss, list(p.values()))))


def test_a_step_of_all_operators():
    """Gradients of a whole step against 64-bit autograd.  A gradient passes at most 8 roundings to float16 a block forward (y, z, mid, o,
    out, and what they were made from) and as many back, and 4 at the ends: 36 for two blocks, each at most 2^-11 of a tensor's norm.
    The maps between them keep relative errors (norms, random matrices) or double them (the norm's gradient, a difference of two of
    its size): 2 x 36 x 2^-11 = 3.6e-2 of a gradient's norm if all of them pointed one way.  Clipped ratios would jump: none is near."""
    net = Net(96, 2, 203, 120, seed=3).cuda()
    loss, want = net.exact()
    stats, clip, grads = net.step()
    torch.cuda.synchronize()
    norm = math.sqrt(sum(float(g.square().sum()) for g in want.values()))
    bound = 2 * 36 * 2.0 ** -11
    assert abs(float(stats[0]) - float(loss)) <= bound * (1 + abs(float(loss)))
    assert abs(float(clip[0]) - norm) <= bound * norm and norm > 0.5
    factor = 0.5 / (norm + 1e-6)
    for k in net.names:
        a, b = grads[k].double().cpu(), factor * want[k]
        far = float((a - b).norm() / b.norm())
        log(f"[step] gradient of {k}: {far:.2e}")
        assert far <= 2 * bound, k  # the clipping's own norm is off by as much
    total = math.sqrt(sum(float(g.double().square().sum()) for g in grads.values()))
    assert abs(total - 0.5) < 1e-3


def test_a_captured_step():
    """A whole step in a graph, replayed on new inputs with eager work and synchronizations between: each replay is the eager result,
    bit for bit.  A second graph with the same workspaces does not disturb the first."""
    net = Net(64, 2, 1021, 700, seed=5, dtype=BF).cuda()  # enough tokens for grouped rows
    g = torch.Generator(device="cuda").manual_seed(9)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        net.step()
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = net.step()
        graphs.append((graph, got))
    for i in range(4):
        net.ids.copy_(torch.randint(0, 1021, (700,), generator=g, device="cuda"))
        net.adv.copy_(torch.randn(700, generator=g, device="cuda"))
        net.p["up0"].mul_(1.01)
        want = net.step()
        torch.cuda.synchronize()
        log(f"[step] graph replay {i}")
        graph, got = graphs[i % 2]
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
        for k in net.names:
            assert torch.equal(want[2][k], got[2][k]), k


def test_two_streams_at_once():
    """The same operators at work on two streams, each on its own data: the bits of one after the other."""
    nets = [Net(96, 1, 600, 500, seed=s, dtype=BF).cuda() for s in (11, 12)]
    want = [net.step() for net in nets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in nets]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        got = []
        for net, s in zip(nets, streams):
            with torch.cuda.stream(s):
                got.append(net.step())
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert torch.equal(a[0], b[0]) and all(torch.equal(a[2][k], b[2][k]) for k in nets[0].names)
