"""The embedding and its gradient on the GPU against 64-bit implementations on the CPU (tests/step_reference.py)."""
import math

import pytest
import torch

import paper_2510_21048_amd as xm
import step_reference as ref
from test_gpu_ops import BF, FF, HF, log, rows, within

pytestmark = pytest.mark.gpu

SIZES = [(1, 1, 1), (1, 5, 8), (3, 2, 7), (17, 40, 33), (64, 1, 64), (65, 300, 65), (37, 1021, 515), (300, 33, 1000), (1000, 257, 72),
         (500, 70000, 16), (129, 999, 2049), (9, 50304, 1024), (2100, 600, 264), (5, 11, 9000), (5000, 3, 40), (4097, 5000, 24)]


def some_ids(g, t, vocab, kind):
    """Tokens: spread evenly, few of them frequent, all one, or with padding and tokens outside of the table."""
    if kind == "even":
        return torch.randint(0, vocab, (t,), generator=g)
    if kind == "one":
        return torch.full((t,), vocab - 1)
    u = torch.rand(t, generator=g, dtype=torch.float64)
    ids = (torch.exp(u * math.log(vocab + 1)) - 1).long().clamp_(0, vocab - 1)
    if kind == "outside" and t > 2:
        ids[torch.randint(0, t, (max(1, t // 5),), generator=g)] = vocab // 2
        ids[0], ids[t // 2], ids[-1] = -1, vocab, 1 << 40
    return ids


@pytest.mark.parametrize("i,size", list(enumerate(SIZES)), ids=["x".join(map(str, s)) for s in SIZES])
@pytest.mark.parametrize("dtype", [BF, HF, FF])
def test_embedding_forward(i, size, dtype):
    t, vocab, n = size
    for j, pad in enumerate((0, 8, 3)):
        g = torch.Generator().manual_seed(100 * i + j)
        table, c = rows(g, vocab, n, dtype, pad)
        ids = some_ids(g, t, vocab, ("even", "outside", "frequent")[j])
        padding, scale = (None, vocab // 2, -1)[j], (1.0, 0.7, -32.0)[j]
        log(f"[step] embedding_forward {size} {dtype} pad={pad} padding={padding}")
        y = xm.embedding_forward(table, ids.cuda(), scale, padding)
        torch.cuda.synchronize()
        inside = (ids >= 0) & (ids < vocab)
        want = scale * c.double()[torch.where(inside, ids, 0)]
        masked = torch.zeros(t, dtype=torch.bool) if padding is None else ids == padding
        want[masked] = 0.0
        bad = ~inside & ~masked
        got = y.cpu()
        assert bool(got[bad].isnan().all())
        within(got[~bad], want[~bad], ref.HALF_ULP[dtype] * want[~bad].abs() * (1 if scale == 1.0 else 1.001) + ref.E * want[~bad].abs()
               + ref.LEAST[dtype], f"y {size} pad={pad}")
        if scale == 1.0:
            assert torch.equal(got[~bad], c[ids[~bad]])


@pytest.mark.parametrize("i,size", list(enumerate(SIZES)), ids=["x".join(map(str, s)) for s in SIZES])
@pytest.mark.parametrize("dtype", [BF, HF, FF])
def test_embedding_backward(i, size, dtype):
    t, vocab, n = size
    for j, pad in enumerate((0, 8, 3, 0)):
        g = torch.Generator().manual_seed(1000 + 100 * i + j)
        dy, c = rows(g, t, n, dtype, pad)
        kind = ("even", "outside", "frequent", "one")[j]
        ids = some_ids(g, t, vocab, kind)
        padding, scale = (None, vocab // 2, None, vocab)[j], (1.0, 0.7, -3.0, 1.5)[j]
        for wide in (False, True):
            o = FF if wide else dtype
            log(f"[step] embedding_backward {size} {dtype} -> {o} {kind} pad={pad}")
            got = xm.embedding_backward(dy, ids.cuda(), vocab, scale, padding, dtype=o)
            torch.cuda.synchronize()
            want, bound = ref.table_grad(c, ids, vocab, scale, padding, None, o)
            assert got.dtype == o
            within(got, want, bound, f"dtable {size} {kind} {o}")
            assert torch.equal(got, xm.embedding_backward(dy, ids.cuda(), vocab, scale, padding, dtype=o))
            into, ic = rows(g, vocab, n, o, pad)
            more = xm.embedding_backward(dy, ids.cuda(), vocab, scale, padding, into=into)
            torch.cuda.synchronize()
            assert more is into
            want, bound = ref.table_grad(c, ids, vocab, scale, padding, ic, o)
            within(into, want, bound, f"dtable added {size} {kind} {o}")


# frequent tokens among many, more tokens than one workgroup sorts, a vocabulary of more bits, long runs of one token
LARGE = [(20000, 50304, 136, "frequent"), (33000, 200000, 64, "even"), (40000, 7, 72, "even"), (70001, 1000, 40, "frequent"),
         (30000, 30000, 520, "one"), (9000, 1 << 21, 8, "frequent"), (150000, 50304, 16, "outside"),
         (5000, 6_000_000, 9, "frequent"), (3000, 12345, 1, "frequent"), (40000, 5, 7, "even"), (2000, 700, 3, "outside")]


@pytest.mark.parametrize("t,vocab,n,kind", LARGE)
@pytest.mark.parametrize("dtype,wide", [(BF, False), (HF, True), (FF, True)])
def test_embedding_backward_many_tokens(t, vocab, n, kind, dtype, wide):
    g = torch.Generator().manual_seed(t)
    dy, c = rows(g, t, n, dtype, 0)
    ids = some_ids(g, t, vocab, kind)
    o = FF if wide else dtype
    into, ic = rows(g, vocab, n, o, 0)
    kept = into.clone()
    log(f"[step] embedding_backward {t} tokens of {vocab}, width {n}, {kind}, {dtype} -> {o}")
    got = xm.embedding_backward(dy, ids.cuda(), vocab, 0.5, vocab // 2, dtype=o)
    again = xm.embedding_backward(dy, ids.cuda(), vocab, 0.5, vocab // 2, dtype=o)
    xm.embedding_backward(dy, ids.cuda(), vocab, 0.5, vocab // 2, into=into)
    torch.cuda.synchronize()
    want, bound = ref.table_grad(c, ids, vocab, 0.5, vocab // 2, None, o)
    within(got, want, bound, "dtable")
    assert torch.equal(got, again)
    want, bound = ref.table_grad(c, ids, vocab, 0.5, vocab // 2, ic, o)
    within(into, want, bound, "dtable added")
    untouched = torch.ones(vocab, dtype=torch.bool)
    untouched[ids[(ids >= 0) & (ids < vocab) & (ids != vocab // 2)]] = False
    u = untouched.cuda()
    assert torch.equal(into[u], kept[u]) and bool((got[u] == 0).all())


def test_embedding_backward_of_no_tokens():
    dy, ids = torch.empty(0, 24, dtype=BF, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda")
    assert bool((xm.embedding_backward(dy, ids, 50) == 0).all()) and xm.embedding_forward(torch.ones(5, 24, device="cuda"), ids).shape == (0, 24)
    into = torch.full((50, 24), 3.0, device="cuda")
    assert bool((xm.embedding_backward(dy, ids, 50, into=into) == 3).all())


@pytest.mark.parametrize("vocab,n", [(50304, 264), (300000, 5), (7, 300000)])
@pytest.mark.parametrize("o", [BF, FF])
def test_embedding_backward_of_no_tokens_clears_large_tables(vocab, n, o):
    dy, ids = torch.empty(0, n, dtype=BF, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda")
    full = torch.full((vocab, n), 3.0, dtype=o, device="cuda")  # freed, so that the outputs are likely to lie where it lay
    del full
    log(f"[step] embedding_backward of no tokens, table {vocab} x {n} {o}")
    assert bool((xm.embedding_backward(dy, ids, vocab, dtype=o) == 0).all())
    into = torch.full((vocab, n), 3.0, dtype=o, device="cuda")
    assert bool((xm.embedding_backward(dy, ids, vocab, into=into) == 3).all())


def test_embedding_backward_with_the_most_notes_and_keys():
    """A group of 1024 rows, and as many notes of tokens as a wavefront keeps: 128 KiB of LDS."""
    g = torch.Generator().manual_seed(70)
    t, vocab, n = 70000, 300000, 8
    dy, c = rows(g, t, n, BF, 0)
    ids = some_ids(g, t, vocab, "frequent")
    log("[step] embedding_backward 70000 tokens of 300000, width 8")
    got = xm.embedding_backward(dy, ids.cuda(), vocab)
    torch.cuda.synchronize()
    want, bound = ref.table_grad(c, ids, vocab, 1.0, None, None, BF)
    within(got, want, bound, "dtable")


def test_embedding_rows_keep_to_themselves():
    """What lies between rows stays; NaN and infinity of one token stay in its row, those of padding and of unnamed rows are not seen."""
    g = torch.Generator().manual_seed(6)
    for n, pad in ((30, 2), (520, 8), (1021, 3)):
        dy = torch.randn(200, n, generator=g).cuda()
        ids = torch.randint(0, 90, (200,), generator=g)
        ids[3], ids[7], ids[11], ids[12] = 90, 91, 92, -5
        dy[3], dy[7], dy[11], dy[12] = math.nan, math.inf, math.nan, math.nan
        hold = torch.full((95, n + pad), 7.0, device="cuda")
        into = hold[:, :n]
        into[94] = math.nan
        log(f"[step] embedding_backward rows of NaN n={n} pad={pad}")
        got = xm.embedding_backward(dy, ids.cuda(), 95, padding_id=92, into=into)
        torch.cuda.synchronize()
        assert bool((hold[:, n:] == 7).all()) and bool(got[90].isnan().all()) and bool((got[91] == math.inf).all())
        assert bool(got[94].isnan().all()) and bool((got[92] == 7).all()) and bool(got[:90].isfinite().all())
        table = torch.randn(95, n, generator=g).cuda()
        table[4] = math.nan
        y = xm.embedding_forward(table, torch.tensor([4, 5, 4, 6]).cuda(), padding_id=4)
        assert bool((y[[0, 2]] == 0).all()) and torch.equal(y[[1, 3]], table[[5, 6]])


def test_embedding_unaligned_bases():
    g = torch.Generator().manual_seed(7)
    hold, ids = torch.randn(100 * 256 + 8, generator=g).to(BF).cuda(), torch.randint(0, 100, (300,), generator=g).cuda()
    grads = torch.randn(300 * 256 + 8, generator=g).to(BF).cuda()
    for off in (1, 4):
        table, dy = hold[off:off + 100 * 256].view(100, 256), grads[off:off + 300 * 256].view(300, 256)
        assert torch.equal(xm.embedding_forward(table, ids), table[ids])
        want = xm.embedding_backward(dy.clone(), ids, 100)
        into = torch.zeros(100 * 256 + 8, dtype=BF, device="cuda")[off:off + 100 * 256].view(100, 256)
        assert torch.equal(xm.embedding_backward(dy, ids, 100), want) and torch.equal(xm.embedding_backward(dy, ids, 100, into=into), want)


def test_embedding_gradient_against_differences():
    """By central differences of sum(dy y) in 64 bits: the lookup is linear, so their own error is only a rounding's."""
    g = torch.Generator().manual_seed(9)
    table, dy, ids = torch.randn(6, 5, generator=g).double(), torch.randn(11, 5, generator=g), torch.randint(0, 6, (11,), generator=g)
    got = xm.embedding_backward(dy.cuda(), ids.cuda(), 6, 2.5)
    want = torch.zeros(6, 5, dtype=torch.float64)
    for i in range(30):
        for sign in (1, -1):
            moved = table.clone()
            moved.view(-1)[i] += sign * 1e-3
            want.view(-1)[i] += sign * (dy.double() * 2.5 * moved[ids]).sum() / 2e-3
    within(got, want, torch.full_like(want, 1e-5), "dtable")


def test_embedding_past_32_bits():
    """Rows that begin past 2^32 elements of their table, looked up and added to."""
    n, vocab = 2048, (1 << 21) + 40
    table = torch.empty(vocab, n, dtype=BF, device="cuda")
    ids = torch.tensor([vocab - 1, 0, 1 << 20, (1 << 21) + 3, vocab - 1], device="cuda")
    table[ids] = torch.randn(5, n, device="cuda").to(BF)
    log("[step] embedding of a table past 2^32 elements")
    assert torch.equal(xm.embedding_forward(table, ids), table[ids])
    dy = torch.randn(5, n, device="cuda").to(BF)
    want = table[ids[:4]].double()
    want += torch.stack([dy[0].double() + dy[4].double(), *dy[1:4].double()])
    xm.embedding_backward(dy, ids, vocab, into=table)
    torch.cuda.synchronize()
    off = (table[ids[:4]].double() - want).abs()
    assert bool((off <= 2.0 ** -8 * want.abs() + 1e-6).all())
