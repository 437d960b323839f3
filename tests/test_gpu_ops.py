"""The training operators on the GPU against plain 64-bit implementations on the CPU (tests/ops_reference.py), at
the sizes, strides, masks and values where they can go wrong.  Bounds are those of 32-bit sums and one rounding."""
import math

import pytest
import torch

import ops_reference as ref
import paper_2510_21048_amd as xm

pytestmark = pytest.mark.gpu

BF, HF, FF = torch.bfloat16, torch.float16, torch.float32
ACTS = ["none", "relu", "gelu", "silu"]


def log(msg):
    print(msg, flush=True)


def within(got, want, bound, what):
    got = got.double().cpu()
    assert got.shape == want.shape, what
    off = (got - want).abs()
    bad = ~(off <= bound)
    if bad.any():
        i = tuple(int(v) for v in torch.nonzero(bad)[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} values off; at {i} got {got[i]:.9g}, want "
                             f"{want[i]:.9g} within {bound[i] if torch.is_tensor(bound) and bound.dim() else bound:.3g}")


def rows(g, r, c, dtype, pad, scale=1.0):
    """A [r, c] matrix on the GPU (and its values on the CPU) whose rows are pad elements apart; what lies between is NaN."""
    v = (torch.randn(r, c, generator=g) * scale).to(dtype)
    t = torch.full((r, c + pad), math.nan, dtype=dtype, device="cuda")[:, :c]
    t.copy_(v)
    return t, v


SIZES = [(1, 1, 1), (1, 5, 8), (1, 64, 64), (2, 300, 1000), (3, 17, 64), (7, 1030, 264), (16, 16, 32), (17, 33, 65), (31, 129, 520),
         (64, 128, 64), (100, 70, 2056), (129, 127, 130), (130, 257, 72), (250, 512, 40), (300, 200, 0), (0, 5, 5), (5, 0, 5),
         (257, 520, 1024), (513, 264, 192), (1024, 768, 320), (33, 4096, 1001), (2, 7, 20011)]


@pytest.mark.parametrize("i,size", list(enumerate(SIZES)), ids=["x".join(map(str, s)) for s in SIZES])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_linear_forward(i, size, dtype):
    m, n, k = size
    for j, pad in enumerate((0, 8, 3)):
        act = ACTS[(i + j) % 4]
        has_b, has_r, save = (i + j) % 3 != 0, (i + j) % 2 == 0, (i + j) % 3 != 1
        g = torch.Generator().manual_seed(100 * i + j)
        x, xc = rows(g, m, k, dtype, pad)
        w, wc = rows(g, n, k, dtype, pad, 1 / math.sqrt(max(k, 1)))
        b = torch.randn(n, generator=g) if has_b else None
        r, rc = rows(g, m, n, dtype, pad) if has_r else (None, None)
        log(f"[ops] linear_forward {size} {dtype} {act} pad={pad} bias={has_b} residual={has_r} z={save}")
        y, z = xm.linear_forward(x, w, None if b is None else b.cuda(), r, activation=act, save_z=save)
        torch.cuda.synchronize()
        wy, wz, by, bz = ref.forward(xc, wc, b, rc, act)
        within(y, wy, by, f"y {size} {act} pad={pad}")
        assert (z is not None) == save
        if save:
            within(z, wz, bz, f"z {size} {act} pad={pad}")


@pytest.mark.parametrize("i,size", list(enumerate(SIZES)), ids=["x".join(map(str, s)) for s in SIZES])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_linear_backward(i, size, dtype):
    m, n, k = size
    for j, pad in enumerate((0, 8, 3)):
        act = ACTS[(i + j + 1) % 4]
        need = [(True, True, True), (True, False, True), (False, True, False)][(i + j) % 3]
        g = torch.Generator().manual_seed(1000 + 100 * i + j)
        dy, dyc = rows(g, m, n, dtype, pad)
        x, xc = rows(g, m, k, dtype, pad)
        w, wc = rows(g, n, k, dtype, pad, 1 / math.sqrt(max(n, 1)))
        z, zc = rows(g, m, n, dtype, pad, 1.5)
        log(f"[ops] linear_backward {size} {dtype} {act} pad={pad} need={need}")
        got = xm.linear_backward(dy, x, w, z if act != "none" else None, act, *need)
        torch.cuda.synchronize()
        want, bound = ref.backward(dyc, xc, wc, zc, act)
        for name, a, v, b, wanted in zip(("dx", "dw", "db"), got, want, bound, need):
            assert (a is not None) == wanted
            if wanted:
                within(a, v, b, f"{name} {size} {act} pad={pad}")


# Large tiles, whole and cut, in each of the three products; operands copied to aligned rows; k split over workgroups
BIG = [(4096, 4096, 96), (4000, 4104, 136), (4104, 72, 4000), (72, 4104, 4000), (2049, 2051, 1023), (1500, 1528, 1030), (200, 136, 9000),
       (64, 96, 20000), (30000, 64, 40), (5, 9001, 2048), (130, 130, 40)]


@pytest.mark.parametrize("i,size", list(enumerate(BIG)), ids=["x".join(map(str, s)) for s in BIG])
def test_linear_large_and_split(i, size):
    m, n, k = size
    for j, pad in enumerate((0, 3)):
        dtype, act = (BF, HF)[(i + j) % 2], ACTS[(i + j) % 4]
        g = torch.Generator().manual_seed(7000 + 10 * i + j)
        x, xc = rows(g, m, k, dtype, pad)
        w, wc = rows(g, n, k, dtype, pad, 1 / math.sqrt(k))
        r, rc = rows(g, m, n, dtype, pad)
        dy, dyc = rows(g, m, n, dtype, pad)
        b = torch.randn(n, generator=g)
        log(f"[ops] linear {size} {dtype} {act} pad={pad}")
        y, z = xm.linear_forward(x, w, b.cuda(), r, activation=act, save_z=True)
        torch.cuda.synchronize()
        wy, wz, by, bz = ref.forward(xc, wc, b, rc, act)
        within(y, wy, by, f"y {size} {act} pad={pad}")
        within(z, wz, bz, f"z {size} {act} pad={pad}")
        zc = z.cpu()
        got = xm.linear_backward(dy, x, w, z, act)
        torch.cuda.synchronize()
        want, bound = ref.backward(dyc, xc, wc, zc, act)
        for name, a, v, c in zip(("dx", "dw", "db"), got, want, bound):
            within(a, v, c, f"{name} {size} {act} pad={pad}")


def test_linear_unaligned_base():
    """Operands that begin between 16-byte boundaries, though their rows are a multiple of 8 apart."""
    g = torch.Generator().manual_seed(12)
    m, n, k = 200, 168, 256
    hold = [torch.randn(r * c + 8, generator=g).to(BF).cuda() for r, c in ((m, k), (n, k), (m, n))]
    for off in (1, 4):
        x, w, dy = (h[off:off + r * c].view(r, c) for h, (r, c) in zip(hold, ((m, k), (n, k), (m, n))))
        wy, _, by, _ = ref.forward(x.cpu(), w.cpu(), None, None, "none")
        within(xm.linear_forward(x, w)[0], wy, by, f"y off={off}")
        want, bound = ref.backward(dy.cpu(), x.cpu(), w.cpu(), dy.cpu(), "none")
        for name, a, v, c in zip(("dx", "dw", "db"), xm.linear_backward(dy, x, w), want, bound):
            within(a, v, c, f"{name} off={off}")


@pytest.mark.parametrize("act", ["none", "gelu", "silu"])
def test_linear_gradients_against_differences(act):
    """dx and dw against central differences of sum(dy y) in 64 bits, step 1e-4 (its own error ~1e-8): what is left is
    the rounding of the 16-bit outputs and of dz."""
    g = torch.Generator().manual_seed(5)
    m, n, k = 5, 7, 11
    x, w = (torch.randn(m, k, generator=g)).to(HF), (torch.randn(n, k, generator=g) / 3).to(HF)
    b, dy = torch.randn(n, generator=g), torch.randn(m, n, generator=g).to(HF)
    zh = xm.linear_forward(x.cuda(), w.cuda(), b.cuda(), activation=act, save_z=True)[1]
    dx, dw, db = xm.linear_backward(dy.cuda(), x.cuda(), w.cuda(), zh, act)

    def total(xd, wd, bd):
        return (dy.double() * ref.activate(xd @ wd.T + bd, act)).sum()

    for at, got in ((0, dx), (1, dw), (2, db)):
        base = [x.double(), w.double(), b.double()]
        want = torch.zeros_like(base[at])
        for i in range(want.numel()):
            for sign in (1, -1):
                moved = [v.clone() for v in base]
                moved[at].view(-1)[i] += sign * 1e-4
                want.view(-1)[i] += sign * total(*moved) / 2e-4
        # z was saved in 16 bits: 2^-11 of z (below 4 here) moves a slope whose derivative is below 1.2; dz is rounded once
        slack = 2.0 ** -11 * 4.0 * 1.2 + 1.2 * 2.0 ** -11
        mag = (dy.double().abs() @ w.double().abs()) if at == 0 else (dy.double().abs().T @ x.double().abs()) if at == 1 else dy.double().abs().sum(0)
        within(got, want, slack * mag + 2.0 ** -11 * want.abs() + 1e-6, f"{('dx', 'dw', 'db')[at]} {act}")


def test_linear_keeps_to_its_rows():
    """Through the C ABI with padded outputs: nothing between the rows is written, and the residual may be y itself."""
    g = torch.Generator().manual_seed(9)
    m, n, k = 70, 50, 24
    x, xc = rows(g, m, k, BF, 8)
    w, wc = rows(g, n, k, BF, 16)
    for pad in (1, 6, 14):
        y = torch.full((m, n + pad), 7.0, dtype=BF, device="cuda")
        rc = torch.randn(m, n, generator=g).to(BF)
        y[:, :n] = rc.cuda()
        z = torch.full((m, n + pad), 7.0, dtype=BF, device="cuda")
        assert xm.xmem_linear_forward(x, x.stride(0), w, w.stride(0), None, y, n + pad, m, n, k, xm.XMEM_BF16, 2, y, n + pad, z,
                                      n + pad, None, 0, torch.cuda.current_stream().cuda_stream) == 0
        wy, wz, by, bz = ref.forward(xc, wc, None, rc, "gelu")
        within(y[:, :n], wy, by, f"y pad={pad}")
        within(z[:, :n], wz, bz, f"z pad={pad}")
        assert bool((y[:, n:] == 7).all()) and bool((z[:, n:] == 7).all())


def test_linear_carries_nan_and_inf():
    """A row of x with NaN or infinity makes that row of y what the formula makes of it and leaves the others alone."""
    for act in ACTS:
        x, w = torch.ones(40, 72, dtype=BF, device="cuda"), torch.ones(33, 72, dtype=BF, device="cuda")
        x[3, 5], x[20, 71], x[21, 0] = math.nan, math.inf, -math.inf
        y = xm.linear_forward(x, w, activation=act)[0].float().cpu()
        assert bool(y[3].isnan().all()) and bool((y[20] == math.inf).all())
        low = {"none": -math.inf, "relu": 0.0}.get(act)
        assert bool((y[21] == low).all()) if low is not None else bool((y[21].isnan() | (y[21] == 0)).all())
        keep = [i for i in range(40) if i not in (3, 20, 21)]
        assert bool((y[keep] == y[0, 0]).all()) and float(y[0, 0]) == 72.0


def test_other_stream_and_same_bits():
    """On a stream of its own, with the inputs made on it, and again: the same bits."""
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        x = torch.randn(500, 264, device="cuda", dtype=BF)
        w = torch.randn(300, 264, device="cuda", dtype=BF)
        dy = torch.randn(500, 300, device="cuda", dtype=BF)
        first = [xm.linear_forward(x, w, activation="silu", save_z=True), None]
        first[1] = xm.linear_backward(dy, x, w, first[0][1], "silu")
        again = [xm.linear_forward(x, w, activation="silu", save_z=True), None]
        again[1] = xm.linear_backward(dy, x, w, again[0][1], "silu")
    s.synchronize()
    for a, b in zip(first[0] + first[1], again[0] + again[1]):
        assert torch.equal(a, b)
    wy = ref.forward(x.cpu(), w.cpu(), None, None, "silu")
    within(first[0][0], wy[0], wy[2], "y")


# ------------------------------------------------------------------ policy loss

POLICY = [(1, 1), (1, 2), (2, 7), (5, 64), (3, 511), (4, 512), (9, 513), (37, 1021), (6, 4096), (3, 8191), (2, 16391), (3, 50304), (2, 65537),
          (2, 131075), (300, 33)]


def policy_inputs(t, v, dtype, seed, low=0.2, high=0.28, dead=0):
    g = torch.Generator().manual_seed(seed)
    x = (2 * torch.randn(t, v, generator=g)).to(dtype)
    y = torch.randint(0, v - dead, (t,), generator=g)
    x[torch.arange(t), y] += 4
    if dead:
        x[:, v - dead:] = -math.inf
    lp = x.double()[torch.arange(t), y] - torch.logsumexp(x.double(), 1)
    moved = 0.3 * torch.randn(t, generator=g)
    for edge in (math.log(1 - low), math.log(1 + high)):  # not at the clip's edges, where there is no derivative
        moved = torch.where((moved - edge).abs() < 1e-3, torch.full_like(moved, edge + 2e-3), moved)
    old = (lp - moved).float()
    refp = (lp + 0.4 * torch.randn(t, generator=g)).float()
    adv = torch.randn(t, generator=g)
    wt = torch.where(torch.rand(t, generator=g) < 0.7, torch.rand(t, generator=g) + 0.1, 0.0)
    wt[0] = 0.5
    return x, y, wt, old, adv, refp


def policy_check(got, x, y, wt, old, adv, refp, beta, scale=1.0, low=0.2, high=0.28):
    stats, lp, dx = got
    ws, wl, wd = ref.policy(x, y, wt, old, adv, refp, low, high, beta, scale)
    on = wt != 0
    elp = torch.where(on, ref.logp_bound(x) + 2 * ref.E * wl.abs(), 0.0)
    within(lp, wl, elp, "logp")
    # how far the slope may be: through the ratio and through the reference's
    rho = torch.exp(wl - old.double())
    eg = (rho * adv.double()).abs() * (elp + 8 * ref.E * (1 + (wl - old.double()).abs() + old.double().abs()))
    ek = torch.zeros_like(eg)
    if refp is not None:
        d = refp.double() - wl
        ek = (torch.exp(d) + 1) * (elp + 8 * ref.E * (1 + d.abs() + refp.double().abs()))
        eg = eg + beta * ek
    wta = wt.double().abs()
    if dx is not None:
        p = torch.softmax(x.double(), 1)
        hit = torch.zeros_like(p)
        hit[torch.arange(len(y)), y] = 1.0
        full = scale * wta * ((rho * adv.double()).abs() + (beta * (1 + torch.exp(d)) if refp is not None else 0))
        far = torch.where(torch.isfinite(x.double()), (x.double() - x.double().amax(1, keepdim=True)).abs(), 0.0)
        rel = elp[:, None] + (far + 12) * 2 * ref.E
        bound = (scale * wta * eg)[:, None] * (p + hit) + full[:, None] * (p * rel + hit * 4 * ref.E)
        within(dx, wd, 1.01 * bound + ref.HALF_ULP[x.dtype] * wd.abs() + ref.LEAST[x.dtype], "dlogits")
        assert bool((dx[~on] == 0).all())
    es = torch.stack([(wta * (eg + beta * ek)).sum(), (wta * eg).sum(), (wta * ek).sum(), torch.zeros((), dtype=torch.float64)])
    mags = torch.stack([(wta * (rho * adv.double()).abs()).sum() + beta * ws[2].abs(), (wta * (rho * adv.double()).abs()).sum(), ws[2].abs(), wta.sum()])
    within(stats, ws, 1.01 * es + 8 * ref.E * mags + 1e-30, "stats")


@pytest.mark.parametrize("t,v", POLICY)
@pytest.mark.parametrize("dtype", [BF, HF, FF])
def test_policy_loss(t, v, dtype):
    for j, (with_ref, beta, dead, pad) in enumerate([(True, 0.05, 0, 0), (False, 0.0, 0, 3), (True, 0.3, min(5, v - 1), 8)]):
        x, y, wt, old, adv, refp = policy_inputs(t, v, dtype, 50 * t + v + j, dead=dead)
        refp = refp if with_ref else None
        d = torch.full((t, v + pad), math.nan, dtype=dtype, device="cuda")[:, :v]
        d.copy_(x)
        log(f"[ops] policy_loss t={t} v={v} {dtype} ref={with_ref} dead={dead} pad={pad}")
        args = [a.cuda() if a is not None else None for a in (y, wt, old, adv, refp)]
        got = xm.policy_loss(d, *args, clip_low=0.2, clip_high=0.28, kl_coef=beta)
        torch.cuda.synchronize()
        policy_check(got, x, y, wt, old, adv, refp, beta)
        lp = xm.token_logp(d, args[0])
        within(lp, x.double()[torch.arange(t), y] - torch.logsumexp(x.double(), 1), 1.01 * ref.logp_bound(x) + 2 * ref.E * 40, "token_logp")
        inplace = xm.policy_loss(d, *args, clip_low=0.2, clip_high=0.28, kl_coef=beta, in_place=True)
        assert inplace[2].data_ptr() == d.data_ptr()
        for a, b in zip(got, inplace):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [BF, HF, FF])
def test_policy_masked_rows_are_not_looked_at(dtype):
    """Rows of weight 0 may hold anything, a token outside the vocabulary too; rows of their own NaN stay theirs."""
    x, y, wt, old, adv, refp = policy_inputs(12, 700, dtype, 3)
    wt[:] = 0.25
    wt[[2, 5, 6, 7]] = 0.0
    bad = x.clone()
    bad[2] = math.nan
    bad[5] = math.inf
    bad[6] = -math.inf
    yb = y.clone()
    yb[7] = -100
    args = [a.cuda() for a in (yb, wt, old, adv, refp)]
    got = xm.policy_loss(bad.cuda(), *args, clip_low=0.2, clip_high=0.28, kl_coef=0.1)
    policy_check(got, x, y, wt, old, adv, refp, 0.1)
    # the same rows with a weight: NaN there, and in the sums
    args[1] = torch.full((12,), 0.25, device="cuda")
    stats, lp, dx = xm.policy_loss(bad.cuda(), *args, clip_low=0.2, clip_high=0.28, kl_coef=0.1)
    assert lp.isnan().cpu().tolist() == [i in (2, 5, 6, 7) for i in range(12)]
    assert bool(stats[0].isnan()) and bool(dx[[2, 5, 6, 7]].isnan().all()) and not bool(dx[[0, 1, 3, 4, 8]].isnan().any())


def test_policy_no_weights_and_no_tokens():
    x, y, wt, old, adv, refp = policy_inputs(33, 129, FF, 8)
    got = xm.policy_loss(x.cuda(), y.cuda(), None, old.cuda(), adv.cuda(), clip_low=0.2, clip_high=0.28)
    policy_check(got, x, y, torch.full((33,), 1 / 33), old, adv, None, 0.0)
    e = torch.empty(0, device="cuda")
    stats, lp, dx = xm.policy_loss(torch.empty(0, 9, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda"), e, e, e)
    assert stats.cpu().tolist() == [0, 0, 0, 0] and lp.numel() == 0 and dx.shape == (0, 9)


def test_policy_values_far_out():
    """Logits whose exponentials overflow 32 bits, and rows that are one certain token."""
    x = torch.zeros(4, 1000)
    x[0] = torch.linspace(-3e38, 3e38, 1000, dtype=torch.float64).float()
    x[1] = 1e4 * torch.randn(1000, generator=torch.Generator().manual_seed(1))
    x[2, 7] = 60000.0
    x[3] = -6e4
    y = torch.tensor([999, int(x[1].argmax()), 7, 3])
    lp = xm.token_logp(x.cuda(), y.cuda()).cpu()
    want = x.double()[torch.arange(4), y] - torch.logsumexp(x.double(), 1)
    assert bool(((lp.double() - want).abs() <= 1e-6 * (1 + want.abs())).all()), (lp, want)


def test_policy_gradient_against_differences():
    """dlogits against central differences of the 64-bit loss (step 1e-5, error ~1e-9), and scaled by grad_scale."""
    x, y, wt, old, adv, refp = policy_inputs(6, 9, FF, 21)
    scale = 8.0
    dx = xm.policy_loss(x.cuda(), *[a.cuda() for a in (y, wt, old, adv, refp)], clip_low=0.2, clip_high=0.28, kl_coef=0.2,
                        grad_scale=scale)[2]
    want = torch.zeros(6, 9, dtype=torch.float64)
    for i in range(6):
        for j in range(9):
            for sign in (1, -1):
                xx = x.double().clone()
                xx[i, j] += sign * 1e-5
                want[i, j] += scale * sign * ref.policy(xx, y, wt, old, adv, refp, 0.2, 0.28, 0.2)[0][0] / 2e-5
    within(dx, want, torch.full_like(want, 2e-5), "dlogits")


# ------------------------------------------------------------------ the orthogonalised update

MUON = [(1, 1, 1), (1, 1, 9), (2, 9, 1), (1, 2, 3), (3, 33, 65), (1, 64, 64), (2, 128, 128), (1, 130, 127), (2, 100, 517), (1, 517, 100),
        (1, 256, 1024), (5, 300, 260), (1, 1000, 72), (1, 385, 1030)]


@pytest.mark.parametrize("count,r,c", MUON)
@pytest.mark.parametrize("dtype", [BF, HF, FF])
def test_muon_update(count, r, c, dtype):
    """Thirty roundings to 11 bits (six a step, at most 2^-11 of a norm each, in unrelated directions) and one to 8 bits (at
    most 2^-8): sqrt(30) 2^-11 + 2^-8 = 6.6e-3, so 1e-2 of the update's norm.  Momentum is two operations in 32 bits."""
    for j, (nesterov, steps, mu, scale) in enumerate([(True, 5, 0.95, 1.5), (False, 3, 0.5, 1.0), (True, 0, 0.9, 1.0)]):
        g = torch.Generator().manual_seed(7 * r + c + j)
        grad = (1e-3 * torch.randn(count, r, c, generator=g)).to(dtype)
        mom = 1e-2 * torch.randn(count, r, c, generator=g)
        log(f"[ops] muon {count}x{r}x{c} {dtype} nesterov={nesterov} steps={steps}")
        m = mom.cuda()
        up = xm.muon_update(grad.cuda(), m, mu=mu, nesterov=nesterov, steps=steps, scale=scale)
        torch.cuda.synchronize()
        wm, wu = ref.muon(grad, mom, mu, nesterov, steps, scale)
        within(m, wm, 4 * ref.E * (mom.double().abs() + grad.double().abs()), "momentum")
        far = ((up.double().cpu() - wu).flatten(1).norm(dim=1) / wu.flatten(1).norm(dim=1)).max()
        assert up.dtype == BF and float(far) < 1e-2, (count, r, c, float(far))
        again = mom.cuda()
        assert torch.equal(up, xm.muon_update(grad.cuda(), again, mu=mu, nesterov=nesterov, steps=steps, scale=scale))
        assert torch.equal(m, again)


@pytest.mark.parametrize("count,r,c", [(60, 520, 1040), (60, 1040, 520), (1, 3000, 2500), (2, 72, 9000), (2, 9000, 40)])
def test_muon_update_large(count, r, c):
    """Large tiles, whole and cut, and few rows with many columns (k split); the reference is computed on the GPU in 64 bits."""
    g = torch.Generator(device="cuda").manual_seed(r)
    grad = (1e-3 * torch.randn(count, r, c, generator=g, device="cuda")).to(BF)
    mom = 1e-2 * torch.randn(count, r, c, generator=g, device="cuda")
    m = mom.clone()
    log(f"[ops] muon {count}x{r}x{c}")
    up = xm.muon_update(grad, m)
    wm, wu = ref.muon(grad, mom, 0.95, True, 5, 1.0)
    assert float((m.double() - wm).abs().max()) <= 4 * ref.E * float(wm.abs().max() + 1)
    far = ((up.double() - wu).flatten(1).norm(dim=1) / wu.flatten(1).norm(dim=1)).max()
    assert float(far) < 1e-2, float(far)


def test_muon_weak_directions():
    """Eight directions that hold nearly all of a gradient: the others, which the steps bring up, keep their accuracy."""
    g = torch.Generator().manual_seed(2)
    grad = torch.randn(2, 256, 8, generator=g) @ torch.randn(2, 8, 300, generator=g) + 0.05 * torch.randn(2, 256, 300, generator=g)
    up = xm.muon_update(grad.cuda(), torch.zeros(2, 256, 300, device="cuda"))
    want = ref.muon(grad, torch.zeros(2, 256, 300), 0.95, True, 5, 1.0)[1]
    assert float((up.double().cpu() - want).norm() / want.norm()) < 1e-2


def test_muon_scale_of_a_gradient():
    """Zero gradients give zero; gradients whose squares leave the range of 32 bits are divided by their norm all the same."""
    z = torch.zeros(2, 40, 24, device="cuda")
    assert bool((xm.muon_update(z, z.clone()) == 0).all())
    g = torch.randn(40, 24, generator=torch.Generator().manual_seed(4))
    for size in (1e25, 1e-3):
        up = xm.muon_update((g * size).cuda(), torch.zeros(40, 24, device="cuda"))
        want = ref.muon((g * size)[None], torch.zeros(1, 40, 24), 0.95, True, 5, 1.0)[1][0]
        assert float((up.double().cpu() - want).norm() / want.norm()) < 1e-2
    bad = g.clone()
    bad[3, 3] = math.nan
    pair = torch.stack([bad, g]).cuda()
    up = xm.muon_update(pair, torch.zeros_like(pair))
    assert bool(up[0].isnan().any()) and not bool(up[1].isnan().any())  # a matrix of a batch keeps to itself
