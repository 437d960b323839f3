"""Residual norms and their gradients on the GPU against 64-bit implementations on the CPU (tests/step_reference.py)."""
import math

import pytest
import torch

import paper_2510_21048_amd as xm
import step_reference as ref
from test_gpu_ops import BF, FF, HF, log, rows, within

pytestmark = pytest.mark.gpu

KINDS = ["none", "rms", "layer"]
GATES = [None, "none", "sigmoid", "silu"]


def inputs(g, t, n, dtype, pad, post, gate, scaled, pre, block=True, weights=True):
    """GPU tensors and their values on the CPU, by name."""
    gpu, cpu = {}, {}
    for name, wanted, size in (("r", True, 2.0), ("h", block, 1.0), ("g", block and gate is not None, 1.5), ("dy", pre != "none", 1.0),
                               ("dout", True, 1.0)):
        gpu[name], cpu[name] = rows(g, t, n, dtype, pad, size) if wanted else (None, None)
    if gpu["h"] is not None:  # a mean that is not near 0
        for to in (gpu, cpu):
            to["h"].add_(0.5)
        cpu["h"] = gpu["h"].cpu()
    for name, wanted in (("s", block and scaled), ("w1", block and post != "none" and weights), ("b1", block and post == "layer" and weights),
                         ("w2", pre != "none" and weights), ("b2", pre == "layer" and weights)):
        cpu[name] = torch.randn(n, generator=g) if wanted else None
        gpu[name] = None if cpu[name] is None else cpu[name].cuda()
    return gpu, cpu


def forward(v, alpha, post, pre, gate, **more):
    return xm.residual_norm_forward(v["r"], v["h"], v["g"], v["s"], alpha, post=post if v["h"] is not None else "none", post_weight=v["w1"],
                                    post_bias=v["b1"], pre=pre, pre_weight=v["w2"], pre_bias=v["b2"], gate_activation=gate or "none", **more)


def backward(v, out, stats, alpha, post, pre, gate, **more):
    return xm.residual_norm_backward(v["dy"], v["dout"], out, stats, v["h"], v["g"], v["s"], alpha, post=post if v["h"] is not None else "none",
                                     post_weight=v["w1"], post_bias=v["b1"], pre=pre, pre_weight=v["w2"], pre_bias=v["b2"],
                                     gate_activation=gate or "none", **more)


NAMES = ("dr", "dh", "dgate", "dscale", "dw1", "db1", "dw2", "db2")


def check(g, t, n, dtype, pad, post, gate, scaled, pre, block, alpha=0.7, eps=1e-5, weights=True):
    what = f"t={t} n={n} {dtype} pad={pad} post={post} gate={gate} scaled={scaled} pre={pre} block={block} weights={weights}"
    log(f"[step] residual_norm {what}")
    v, c = inputs(g, t, n, dtype, pad, post, gate, scaled, pre, block, weights)
    p = post if block else "none"
    out, y, stats = forward(v, alpha, post, pre, gate, eps=eps, save_stats=True)
    torch.cuda.synchronize()
    want, bound = ref.forward(c["r"], c["h"], c["g"], c["s"], alpha, p, c["w1"], c["b1"], pre, c["w2"], c["b2"], gate or "none", eps)
    within(out, want[0], bound[0], f"out {what}")
    assert (out is v["r"]) == (not block) and (y is None) == (pre == "none")
    if y is not None:
        within(y, want[1], bound[1], f"y {what}")
    within(stats, want[2], bound[2], f"stats {what}")
    got = backward(v, out, stats, alpha, post, pre, gate)
    torch.cuda.synchronize()
    want, bound = ref.backward(c["dy"], c["dout"], out.cpu(), stats.cpu(), c["h"], c["g"], c["s"], alpha, p, c["w1"], c["b1"], pre, c["w2"],
                               gate or "none")
    given = (True, block, c["g"] is not None, c["s"] is not None, c["w1"] is not None, c["b1"] is not None, c["w2"] is not None,
             c["b2"] is not None)
    for name, a, b, e, there in zip(NAMES, got, want, bound, given):
        assert (a is not None) == there, (name, what)
        if there:
            within(a, b, e, f"{name} {what}")
    return v, got


# one element, less than a piece, each width of rows and number of pieces, their neighbours, and rows that no registers hold
WIDTHS = [1, 2, 7, 8, 9, 64, 255, 512, 513, 1000, 1024, 1025, 2047, 2048, 2049, 4096, 4100, 8191, 8200, 16384, 16390, 33000]


@pytest.mark.parametrize("i,n", list(enumerate(WIDTHS)), ids=map(str, WIDTHS))
@pytest.mark.parametrize("dtype", [BF, HF, FF])
def test_residual_norm_widths(i, n, dtype):
    g = torch.Generator().manual_seed(n)
    for j in range(4):
        t = (1, 3, 6, 37)[(i + j) % 4] if n < 8000 else (1, 2)[j % 2]
        check(g, t, n, dtype, (0, 8, 3, 0)[j], KINDS[(i + j) % 3], GATES[(i + 2 * j) % 4], (i + j) % 2 == 0, KINDS[1 + (i + j + 1) % 2],
              True)


@pytest.mark.parametrize("post", KINDS)
@pytest.mark.parametrize("pre", KINDS)
@pytest.mark.parametrize("gate", GATES)
def test_residual_norm_kinds(post, pre, gate):
    """Every combination of norms and gates, with and without scale and weights."""
    g = torch.Generator().manual_seed(KINDS.index(post) + 3 * KINDS.index(pre))
    for j, (dtype, scaled, weights) in enumerate([(BF, True, True), (HF, False, False), (FF, True, False), (FF, False, True)]):
        check(g, 5, (72, 515, 1024, 130)[j], dtype, (0, 3, 0, 8)[j], post, gate, scaled, pre, True, alpha=(1.0, -0.5, 2.0, 0.25)[j],
              weights=weights)


@pytest.mark.parametrize("pre", ["rms", "layer"])
@pytest.mark.parametrize("dtype", [BF, HF, FF])
def test_norm_alone(pre, dtype):
    """Without a block: the norm of the residual stream, and its gradient with and without what comes to the sum past it."""
    g = torch.Generator().manual_seed(11)
    for t, n, pad in ((1, 1, 0), (4, 33, 3), (9, 1024, 0), (3, 5000, 5), (2, 70000, 0)):
        v, got = check(g, t, n, dtype, pad, "none", None, False, pre, False)
        stats = forward(v, 1.0, "none", pre, None, save_stats=True)[2]
        alone = xm.residual_norm_backward(v["dy"], None, v["r"], stats, pre=pre, pre_weight=v["w2"], pre_bias=v["b2"])
        want, bound = ref.backward(v["dy"].cpu(), None, v["r"].cpu(), stats.cpu(), None, None, None, 1.0, "none", None, None, pre,
                                   v["w2"].cpu(), "none")
        within(alone[0], want[0], bound[0], f"dr alone {pre} {n}")


@pytest.mark.parametrize("t,n,dtype", [(2000, 520, BF), (2050, 2056, HF), (4099, 64, HF), (1111, 2050, BF), (700, 4104, HF), (530, 1024, FF), (600, 16384, BF),
                                       (40, 16400, FF), (300, 40000, BF)])
def test_residual_norm_many_rows(t, n, dtype):
    """More rows than there are groups of them."""
    g = torch.Generator().manual_seed(t)
    check(g, t, n, dtype, 0, "layer", "silu", True, "layer", True)
    check(g, t, n, dtype, 3, "rms", "sigmoid", True, "rms", True)


def test_residual_norm_of_no_rows():
    e = torch.empty(0, 24, dtype=BF, device="cuda")
    w = torch.ones(24, device="cuda")
    out, y, stats = xm.residual_norm_forward(e, e, None, w, post="rms", post_weight=w, pre_weight=w, save_stats=True)
    assert out.shape == y.shape == (0, 24) and stats.shape == (4, 0)
    got = xm.residual_norm_backward(e, e, out, stats, e, None, w, post="rms", post_weight=w, pre_weight=w)
    torch.cuda.synchronize()
    assert got[0].shape == got[1].shape == (0, 24) and got[2] is None and got[5] is None
    assert all(bool((got[i] == 0).all()) and got[i].shape == (24,) for i in (3, 4, 6))


def test_residual_norm_in_place_and_same_bits():
    """out over residual and dr over dout, and again: the same bits."""
    for n, dtype in ((515, BF), (2048, HF), (4097, FF), (20000, BF), (40000, FF)):
        g = torch.Generator().manual_seed(n)
        v, _ = inputs(g, 9, n, dtype, 5, "layer", "silu", True, "rms")
        first = forward(v, 0.5, "layer", "rms", "silu", save_stats=True)
        grads = backward(v, first[0], first[2], 0.5, "layer", "rms", "silu")
        log(f"[step] residual_norm in place n={n} {dtype}")
        for place in (False, True):
            again = forward(v, 0.5, "layer", "rms", "silu", save_stats=True, in_place=place)
            more = backward(v, first[0], first[2], 0.5, "layer", "rms", "silu", in_place=place)
            torch.cuda.synchronize()
            for a, b in zip(first + grads, again + more):
                assert (a is None) == (b is None) and (a is None or torch.equal(a, b))
        assert again[0] is v["r"] and more[0] is v["dout"]


def test_residual_norm_in_place_without_sums_between():
    """Nothing is summed between the reads of a row and its writes: no norm of the block, and no norm after the sum.  In rows whose last
    piece begins a wavefront and shares columns with the one before it."""
    g = torch.Generator().manual_seed(31)
    for n, dtype in ((513, BF), (1025, HF), (259, FF), (2049, BF), (4097, BF), (8193, HF), (8195, FF), (70001, BF)):
        r, h, d = (torch.randn(600, n, generator=g).to(dtype).cuda() for _ in range(3))
        want = xm.residual_norm_forward(r, h, alpha=0.3, pre="none", save_stats=True)
        grads = xm.residual_norm_backward(None, d, None if dtype == BF else want[0], want[2], h, alpha=0.3, pre="none")
        log(f"[step] residual_norm in place without sums n={n} {dtype}")
        for _ in range(3):
            mine, grad = r.clone(), d.clone()
            got = xm.residual_norm_forward(mine, h, alpha=0.3, pre="none", save_stats=True, in_place=True)
            back = xm.residual_norm_backward(None, grad, None if dtype == BF else got[0], got[2], h, alpha=0.3, pre="none", in_place=True)
            torch.cuda.synchronize()
            assert got[0] is mine and torch.equal(mine, want[0]) and back[0] is grad and torch.equal(grad, grads[0])
            assert torch.equal(back[1], grads[1]) and torch.equal(grad, d)


def test_residual_norm_keeps_to_its_rows():
    """Through the C ABI with padded outputs: nothing between the rows is written, and the rows are the same."""
    g = torch.Generator().manual_seed(3)
    for t, n, pad in ((5, 30, 2), (4, 1021, 7), (3, 4099, 13), (2, 17000, 9)):
        v, _ = inputs(g, t, n, BF, 0, "rms", "sigmoid", True, "rms")
        want = forward(v, 1.0, "rms", "rms", "sigmoid", save_stats=True)
        grads = backward(v, want[0], want[2], 1.0, "rms", "rms", "sigmoid", need_vectors=False)
        assert all(q is None for q in grads[3:])
        new = lambda: torch.full((t, n + pad), 7.0, dtype=BF, device="cuda")
        out, y, dr, dh, dg = (new() for _ in range(5))
        st = torch.cuda.current_stream().cuda_stream
        stats = torch.empty(4, t, device="cuda")
        log(f"[step] residual_norm padded outputs {t}x{n}+{pad}")
        assert xm.xmem_residual_norm_forward(v["r"], n, v["h"], n, v["g"], n, v["s"], 1.0, 1, v["w1"], None, 1, v["w2"], None, 1, 1e-5, t, n, 0,
                                             out, n + pad, y, n + pad, stats, st) == 0
        assert xm.xmem_residual_norm_backward(v["dy"], n, v["dout"], n, out, n + pad, stats, v["h"], n, v["g"], n, v["s"], 1.0, 1, v["w1"], None,
                                              1, v["w2"], 1, t, n, 0, dr, n + pad, dh, n + pad, dg, n + pad, None, None, None, None, None,
                                              None, 0, st) == 0
        torch.cuda.synchronize()
        for a, b in zip((out, y, dr, dh, dg), (want[0], want[1], *grads[:3])):
            assert torch.equal(a[:, :n], b) and bool((a[:, n:] == 7).all())


def test_residual_norm_unaligned_bases():
    """Operands that begin between 16-byte boundaries."""
    g = torch.Generator().manual_seed(8)
    t, n = 6, 1024
    v, _ = inputs(g, t, n, BF, 0, "rms", "silu", True, "layer")
    want = forward(v, 1.0, "rms", "layer", "silu", save_stats=True)
    grads = backward(v, want[0], want[2], 1.0, "rms", "layer", "silu")
    for off in (1, 4):
        moved = {}
        for k, x in v.items():
            moved[k] = None if x is None else torch.empty(x.numel() + 8, dtype=x.dtype, device="cuda")[off:off + x.numel()].view(x.shape)
            if x is not None:
                moved[k].copy_(x)
        got = forward(moved, 1.0, "rms", "layer", "silu", save_stats=True)
        more = backward(moved, got[0], got[2], 1.0, "rms", "layer", "silu")
        torch.cuda.synchronize()
        for a, b in zip(want + grads, got + more):
            assert (a is None and b is None) or torch.equal(a, b)


def test_residual_norm_rows_keep_to_themselves():
    """A row with NaN or infinity is what the formula makes of it; the others do not see it.  A row of zeros, and one of equal
    values, whose deviation is 0, give what eps leaves."""
    for n, dtype in ((72, BF), (1024, FF), (5000, HF), (33000, BF)):
        g = torch.Generator().manual_seed(n)
        v, _ = inputs(g, 7, n, dtype, 0, "none", None, False, "layer")
        want = forward(v, 1.0, "none", "layer", None, save_stats=True)
        grads = backward(v, want[0], want[2], 1.0, "none", "layer", None)
        v["r"][2, n // 2] = math.nan
        v["h"][4, n - 1] = math.inf
        v["r"][5] = 0
        v["h"][5] = 0
        v["r"][6] = 3
        v["h"][6] = -1
        log(f"[step] residual_norm NaN, infinity, equal values n={n} {dtype}")
        out, y, stats = forward(v, 1.0, "none", "layer", None, save_stats=True)
        got = backward(v, out, stats, 1.0, "none", "layer", None)
        torch.cuda.synchronize()
        assert bool(y[2].isnan().all()) and bool(y[4].isnan().all()) and bool(got[0][[2, 4]].isnan().all())
        for i in (5, 6):  # (x - mean) is 0: the bias
            within(y[i], v["b2"].double().cpu(), ref.HALF_ULP[dtype] * v["b2"].double().cpu().abs() + ref.LEAST[dtype], f"y[{i}]")
        keep = [0, 1, 3]
        assert torch.equal(y[keep], want[1][keep]) and torch.equal(got[0][keep], grads[0][keep]) and torch.equal(got[1][keep], grads[1][keep])


def test_residual_norm_far_values():
    """Gates far out, and means far larger than the deviations: nothing cancels that is not in the inputs."""
    g = torch.Generator().manual_seed(5)
    for n in (256, 3000):
        v, c = inputs(g, 4, n, FF, 0, "layer", "silu", True, "layer")
        for to in (v, c):
            to["g"][0, :8] = torch.tensor([-200.0, -90.0, -50.0, 50.0, 90.0, 200.0, 0.0, -0.0])
            to["h"][1] += 3000.0
            to["h"][2] *= 1e-3
        for act in ("silu", "sigmoid"):
            out, y, stats = forward(v, 1.0, "layer", "layer", act, save_stats=True)
            got = backward(v, out, stats, 1.0, "layer", "layer", act)
            torch.cuda.synchronize()
            want, bound = ref.forward(c["r"], c["h"], c["g"], c["s"], 1.0, "layer", c["w1"], c["b1"], "layer", c["w2"], c["b2"], act, 1e-5)
            for a, b, e, name in zip((out, y, stats), want, bound, ("out", "y", "stats")):
                within(a, b, e, f"{name} {act} n={n}")
            want, bound = ref.backward(c["dy"], c["dout"], out.cpu(), stats.cpu(), c["h"], c["g"], c["s"], 1.0, "layer", c["w1"], c["b1"],
                                       "layer", c["w2"], act)
            for a, b, e, name in zip(got, want, bound, NAMES):
                within(a, b, e, f"{name} {act} n={n}")


@pytest.mark.parametrize("post,pre,act", [("rms", "layer", "silu"), ("layer", "rms", "sigmoid"), ("none", "rms", "none"), ("rms", "none", "silu")])
def test_residual_norm_gradients_against_differences(post, pre, act):
    """Every gradient against central differences, in 64 bits, of sum(dy y) + sum(dout out): step 1e-5, whose own error is near 1e-9.
    The forward pass is the definition's; float32 leaves the bounds of ref.backward, below 1e-4 here."""
    g = torch.Generator().manual_seed(21)
    t, n, alpha = 3, 10, 0.8
    v, c = inputs(g, t, n, FF, 0, post, act, True, pre)
    out, y, stats = forward(v, alpha, post, pre, act, save_stats=True)
    got = backward(v, out, stats, alpha, post, pre, act)
    names = ["r", "h", "g", "s", "w1", "b1", "w2", "b2"]
    base = {k: None if c[k] is None else c[k].double() for k in names}

    def total(b):
        o, yy, _ = definition(b, alpha, post, pre, act)
        return (c["dout"].double() * o).sum() + (0.0 if yy is None else (c["dy"].double() * yy).sum())

    for name, k, a in zip(NAMES, names, got):
        if base[k] is None:
            assert a is None
            continue
        want = torch.zeros_like(base[k])
        for i in range(want.numel()):
            for sign in (1, -1):
                moved = {q: None if x is None else x.clone() for q, x in base.items()}
                moved[k].view(-1)[i] += sign * 1e-5
                want.view(-1)[i] += sign * total(moved) / 2e-5
        within(a, want, torch.full_like(want, 1e-4), f"{name} {post} {pre} {act}")


def definition(b, alpha, post, pre, act, eps=1e-5):
    """The forward pass in 64 bits."""
    def norm(x, kind, w, bias):
        if kind == "none":
            return x
        x = x - x.mean(1, keepdim=True) if kind == "layer" else x
        x = x / (x.square().mean(1, keepdim=True) + eps).sqrt()
        x = x if w is None else x * w
        return x if bias is None else x + bias

    out = b["r"]
    if b["h"] is not None:
        u = norm(b["h"], post, b["w1"], b["b1"])
        if b["g"] is not None:
            u = u * {"none": lambda q: q, "sigmoid": torch.sigmoid, "silu": lambda q: q * torch.sigmoid(q)}[act](b["g"])
        out = out + alpha * u * (1.0 if b["s"] is None else b["s"])
    return out, None if pre == "none" else norm(out, pre, b["w2"], b["b2"]), None
