"""The memory of the calls of include/ops/xmem_step.h on the host (no GPU needed): their workspaces' sizes, and what they refuse to
overwrite."""
import ctypes
import subprocess

import pytest
import torch

import paper_2510_21048_amd as xm
from paper_2510_21048_amd.ops_step import _apart
from test_step_abi import EINVAL, EWORKSPACE, INF, ROOT, back, clip, table_grad


@pytest.mark.parametrize("vocab,width", [(100, 64), (900, 515), (1021, 1024), (50304, 1024), (50304, 5), (200000, 64)])
def test_embedding_backward_workspace_never_shrinks(vocab, width):
    """A buffer that holds the largest batch holds every smaller one."""
    size, last = xm.xmem_embedding_backward_workspace_bytes, 0
    for t in [*range(0, 40000), *range(40000, 1 << 20, 997), 1 << 24, (1 << 31) - 1]:
        now = size(t, vocab, width)
        assert now >= last, (t, last, now)
        last = now


def test_norm_backward_workspace_never_shrinks():
    for width in (1, 7, 64, 1021, 4096, 16384, 40000):
        for dtype in (xm.XMEM_BF16, xm.XMEM_F32):
            sizes = [xm.xmem_residual_norm_backward_workspace_bytes(t, width, dtype) for t in [*range(0, 40000), *range(40000, 1 << 20, 997)]]
            assert sizes == sorted(sizes)


def test_embedding_backward_workspace():
    """A grouped table's: one byte less, none, or one that begins between 256-byte boundaries."""
    for t in (300, 16383, 16384, 20000):
        need = xm.xmem_embedding_backward_workspace_bytes(t, 50304, 64)
        assert need > 0
        for over in (dict(size=need - 1), dict(ws=None), dict(ws=(1 << 20) + 8)):
            assert table_grad(t=t, vocab=50304, **over) == EWORKSPACE
            assert table_grad(t=t, vocab=50304, add=1, **over) == EWORKSPACE


def test_what_is_overwritten_is_apart_from_every_input():
    """Matrices, vectors, statistics and tokens, each before, on and behind what a call overwrites."""
    flat = torch.zeros(1000)
    over = flat[100:484].view(8, 48)[:, :24]  # rows of 24 elements, 48 apart; the last ends at 460
    row = lambda at, n: flat[at:at + n]
    for free in (row(0, 100), row(460, 100), row(0, 0), row(110, 0)):
        _apart(over, "over", x=free)
        _apart(over, "over", x=free, y=None)
    for bad in (row(0, 101), row(459, 1), row(100, 24), row(123, 1), row(123, 2), row(147, 2), row(148, 1), row(436 - 24, 25), row(0, 1000)):
        with pytest.raises(xm.XmemError, match="vector: shares memory with over"):
            _apart(over, "over", matrix=row(0, 100).view(4, 25), vector=bad)
    stats, ids = row(60, 400).view(torch.int32), flat[0:102].view(torch.int64)
    for bad in (stats, stats.view(4, 100), ids, ids[50:]):
        with pytest.raises(xm.XmemError, match="shares memory"):
            _apart(over, "over", x=bad)
    _apart(over, "over", ids=ids[:50], stats=row(460, 400).view(4, 100))
    # matrices as before: halves of one, and neighbours
    both = flat[:960].view(10, 96)
    for a, b, apart in ((both[:, :48], both[:, 48:], True), (both[:, 48:], both[:, :48], True), (both[:5], both[5:], True), (both[:, :48], both[:, 47:95], False),
                        (both[:, :48], both[1:, :48], False), (both[:, 48:], both[:9, 47:95], False), (both, both, False), (both[:6], both[5:], False)):
        if apart:
            _apart(a, "over", x=b)
        else:
            with pytest.raises(xm.XmemError, match="shares memory"):
                _apart(a, "over", x=b)


def test_what_lies_between_two_rows_is_apart():
    """One row, a vector or a whole small matrix in the gap between two rows of what is overwritten, up to both of its ends."""
    flat = torch.zeros(1000)
    over = flat[100:484].view(8, 48)[:, :24]
    row = lambda at, n: flat[at:at + n]
    for free in (row(124, 24), row(124, 1), row(147, 1), row(412, 24), row(130, 6), row(124, 24).view(1, 24), row(172, 24).view(4, 6),
                 flat[124:].as_strided((1, 24), (1000, 1))):
        _apart(over, "over", x=free)
        _apart(free, "free", x=over)
    for bad in (row(123, 25), row(123, 1), row(124, 25), row(148, 1), row(412, 25), row(172, 25).view(5, 5)):
        for a, b in ((over, bad), (bad, over)):
            with pytest.raises(xm.XmemError, match="shares memory"):
                _apart(a, "over", x=b)


MIB = 1 << 20
FAR = 1 << 40  # where nothing else lies


def test_a_workspace_on_a_norm_gradients_operands_is_refused():
    t, n, ld = 8, 64, 64
    need = xm.xmem_residual_norm_backward_workspace_bytes(t, n, xm.XMEM_BF16)
    where = ("dy", "dout", "o", "stats", "h", "gate", "s", "w1", "b1", "w2", "dr", "dh", "dg", "ds", "dw1", "db1", "dw2", "db2")
    bytes_of = lambda k: t * n * 2 if k in ("dy", "dout", "o", "h", "gate", "dr", "dh", "dg") else 16 * t if k == "stats" else 4 * n
    ws = 64 * MIB
    apart = dict(ws=ws, size=need, t=t, n=n, **{k: FAR + i * MIB for i, k in enumerate(where)})
    for k in where:
        for at in (ws, ws + need - 4, ws - bytes_of(k) + 4):
            assert back(**dict(apart, **{k: at})) == EINVAL, (k, at)
        # neighbours are no fault: what is refused then is the workspace's size, which is looked at first
        for at in (ws + need, ws - bytes_of(k)):
            assert back(**dict(apart, **{k: at, "size": need - 1})) == EWORKSPACE
    # rows far apart, the workspace on one of them, or over the end of one
    for k, d in (("dy", "lddy"), ("dout", "lddo"), ("o", "ldo"), ("h", "ldh"), ("gate", "ldg"), ("dr", "lddr"), ("dh", "lddh"), ("dg", "lddg")):
        assert back(**dict(apart, **{k: ws - 3 * MIB, d: MIB // 2})) == EINVAL
        assert back(**dict(apart, **{k: ws - 3 * MIB - 126, d: MIB // 2})) == EINVAL
        assert back(**dict(apart, **{k: ws - 2 * MIB + 256, d: MIB // 2})) == EINVAL


def test_a_workspace_on_a_table_gradients_operands_is_refused():
    t, vocab, n = 300, 50304, 64
    need, ws = xm.xmem_embedding_backward_workspace_bytes(t, vocab, n), 64 * MIB
    apart = dict(ws=ws, size=need, t=t, vocab=vocab, n=n, ldd=n, dy=FAR, ids=FAR + MIB, out=FAR + 64 * MIB)
    for add in (0, 1):
        for k, size in (("dy", t * n * 2), ("ids", 8 * t), ("out", vocab * n * 4)):
            for at in (ws, ws + need - 4, ws - size + 4, ws - size // 2):
                assert table_grad(**dict(apart, add=add, **{k: at})) == EINVAL, (k, at)
            for at in (ws + need, ws - size):
                assert table_grad(**dict(apart, add=add, size=need - 1, **{k: at})) == EWORKSPACE


def test_a_workspace_on_a_gradient_is_refused():
    need, ws = xm.xmem_clip_grad_norm_workspace_bytes(), 64 * MIB
    call = lambda at, max_norm=1.0, **over: clip(at=(FAR, at), sizes=(100, 200), ws=ws, max_norm=max_norm, **dict(dict(size=need), **over))
    for max_norm in (1.0, INF):  # the norm alone writes its workspace too
        for at in (ws, ws + need - 4, ws - 796, ws - 400):
            assert call(at, max_norm) == EINVAL
        assert clip(at=(FAR, FAR + MIB), ws=ws, size=need, max_norm=max_norm, stats=ws + 8) == EINVAL
        for at in (ws + need, ws - 800):
            assert call(at, max_norm, size=need - 1) == EWORKSPACE
    assert clip(at=(ws, FAR), sizes=(0, 200), ws=ws, size=need - 1) == EWORKSPACE


def shares(ws, size, x, rows, ld, width, element):
    """Whether a matrix has a byte of the workspace, row by row."""
    return any(ws < x + (r * ld + width) * element and x + r * ld * element < ws + size for r in range(rows))


def test_a_workspace_between_rows(tmp_path):
    """The check itself, as the host compiles it, against every row looked at."""
    src = tmp_path / "shares.cpp"
    text = (ROOT / "paper_2510_21048_amd/csrc/ops/rows.h").read_text()
    body = text[text.index("inline bool shares("):]
    body = body[:body.index("\n}\n") + 3]
    src.write_text("#include <stddef.h>\n#include <stdint.h>\n" + body + '''
extern "C" int check(uint64_t ws, uint64_t bytes, uint64_t x, int64_t rows, int64_t ld, int64_t width, int size) {
  return shares(reinterpret_cast<void*>(ws), bytes, reinterpret_cast<void*>(x), rows, ld, width, size);
}
''')
    lib = tmp_path / "shares.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", str(src), "-o", str(lib)], check=True)
    check = ctypes.CDLL(str(lib)).check
    check.argtypes = [ctypes.c_uint64] * 3 + [ctypes.c_int64] * 3 + [ctypes.c_int]
    seen = [0, 0]
    for x in (64,):
        for rows in (0, 1, 2, 4):
            for ld, width in ((1, 1), (5, 3), (6, 6), (7, 1)):
                for element in (2, 4):
                    for ws in range(40, 200):
                        for size in (1, 4, 9, 40):
                            want = shares(ws, size, x, rows, ld, width, element)
                            seen[want] += 1
                            assert bool(check(ws, size, x, rows, ld, width, element)) == want
    assert min(seen) > 1000
    # no workspace, no operand, and the largest sizes that a call takes
    assert not check(64, 0, 64, 1, 1, 1, 4) and not check(64, 8, 0, 1, 1, 1, 4)
    assert not check(64, 64, 80, 1, 0, 0, 8) and not check(64, 64, 80, 0, 8, 8, 4)  # no tokens, wherever their pointer points
    most = (1 << 31) - 1, (1 << 40) - 1
    assert check((1 << 60) + (1 << 42), 8, 1 << 60, most[0], most[1], most[0], 4) and not check((1 << 60) - 8, 8, 1 << 60, most[0], most[1], most[0], 4)
    assert not check((1 << 60) + (1 << 41), 8, 1 << 60, most[0], most[1], most[0], 4)
