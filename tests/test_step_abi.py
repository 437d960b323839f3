"""The C ABI of include/ops/xmem_step.h on the host (no GPU needed): what the header declares is exported, and every argument check
returns its code before any device work."""
import re
import subprocess
from pathlib import Path

import pytest
import torch

import paper_2510_21048_amd as xm

ROOT = Path(__file__).resolve().parents[1]
HEADER = ROOT / "include" / "ops" / "xmem_step.h"
OK, EINVAL, EWORKSPACE = 0, -1, -5
NONE, RMS, LAYER = 0, 1, 2
NAN, INF = float("nan"), float("inf")


def test_library_exports_what_the_header_declares():
    text = re.sub(r"/\*.*?\*/", "", HEADER.read_text(), flags=re.S)
    names = sorted(set(re.findall(r"^(?:int|size_t) (xmem_[a-z_]+)\(", text, flags=re.M)))
    assert names == sorted([
        "xmem_residual_norm_forward", "xmem_residual_norm_backward", "xmem_residual_norm_backward_workspace_bytes", "xmem_embedding_forward",
        "xmem_embedding_backward", "xmem_embedding_backward_workspace_bytes", "xmem_clip_grad_norm", "xmem_clip_grad_norm_workspace_bytes"])
    lib = xm.load_ops()
    for name in names:
        assert hasattr(lib, name) and hasattr(xm, name), name
    subprocess.run(["gcc", "-std=c99", "-fsyntax-only", "-x", "c", f"-I{ROOT / 'include'}", str(HEADER)], check=True)


def norm(**over):
    a = dict(r=4096, ldr=64, h=8192, ldh=64, gate=12288, ldg=64, s=64, alpha=1.0, post=RMS, w1=64, b1=64, pre=RMS, w2=64, b2=64, act=1,
             eps=1e-5, t=8, n=64, dtype=xm.XMEM_BF16, out=16384, ldo=64, y=20480, ldy=64, stats=64, stream=None)
    a.update(over)
    return xm.xmem_residual_norm_forward(*a.values())


NO_BLOCK = dict(h=None, gate=None, s=None, post=NONE, w1=None, b1=None, out=None)


@pytest.mark.parametrize("over", [
    dict(t=-1), dict(t=1 << 31), dict(n=0), dict(n=1 << 31), dict(dtype=3), dict(dtype=-1), dict(post=3), dict(pre=-1), dict(act=3), dict(act=-1),
    dict(eps=-1e-9), dict(eps=NAN), dict(ldr=63), dict(ldh=63), dict(ldg=63), dict(ldo=63), dict(ldy=63), dict(ldr=1 << 40),
    dict(post=NONE), dict(post=NONE, w1=None), dict(post=NONE, b1=None), dict(pre=NONE), dict(pre=NONE, w2=None, b2=None),
    dict(NO_BLOCK, gate=64), dict(NO_BLOCK, s=64), dict(NO_BLOCK, post=RMS), dict(NO_BLOCK, out=64),
    dict(r=None), dict(y=None), dict(out=None), dict(out=4096, ldo=128)])
def test_residual_norm_forward_refuses(over):
    assert norm(**over) == EINVAL


def test_residual_norm_forward_of_nothing():
    assert norm(t=0, r=None, out=None, y=None) == OK and norm(**NO_BLOCK, t=0) == OK
    assert norm(**dict(NO_BLOCK, pre=NONE, w2=None, b2=None, y=None, stats=None)) == OK


def back(**over):
    a = dict(dy=4096, lddy=64, dout=8192, lddo=64, o=4096, ldo=64, stats=64, h=8192, ldh=64, gate=12288, ldg=64, s=64, alpha=1.0, post=RMS,
             w1=64, b1=64, pre=RMS, w2=64, act=1, t=8, n=64, dtype=xm.XMEM_BF16, dr=16384, lddr=64, dh=16384, lddh=64, dg=16384, lddg=64,
             ds=64, dw1=64, db1=64, dw2=64, db2=64, ws=1 << 20, size=1 << 30, stream=None)
    a.update(over)
    return xm.xmem_residual_norm_backward(*a.values())


NO_BLOCK_BACK = dict(h=None, gate=None, s=None, post=NONE, w1=None, b1=None, dh=None, dg=None, ds=None, dw1=None, db1=None)
NO_PRE = dict(pre=NONE, dy=None, w2=None, dw2=None, db2=None)


@pytest.mark.parametrize("over", [
    dict(t=-1), dict(t=1 << 31), dict(n=0), dict(n=1 << 31), dict(dtype=3), dict(post=3), dict(pre=-1), dict(act=3),
    dict(lddy=63), dict(lddo=63), dict(ldo=63), dict(ldh=63), dict(ldg=63), dict(lddr=63), dict(lddh=63), dict(lddg=63), dict(lddg=1 << 40),
    dict(post=NONE), dict(post=NONE, w1=None, b1=None, dw1=None), dict(post=NONE, w1=None, b1=None, db1=None),
    dict(NO_PRE, dy=64), dict(NO_PRE, w2=64), dict(NO_PRE, dw2=64), dict(NO_PRE, db2=64), dict(NO_PRE, dout=None),
    dict(NO_BLOCK_BACK, gate=64), dict(NO_BLOCK_BACK, s=64), dict(NO_BLOCK_BACK, post=LAYER), dict(NO_BLOCK_BACK, dh=64),
    dict(NO_BLOCK_BACK, ds=64), dict(gate=None), dict(dr=None), dict(stats=None), dict(dy=None), dict(o=None), dict(dh=None),
    dict(dr=8192, lddr=128)])
def test_residual_norm_backward_refuses(over):
    assert back(**over) == EINVAL


def test_residual_norm_backward_workspace():
    need = xm.xmem_residual_norm_backward_workspace_bytes(8, 64, xm.XMEM_BF16)
    assert need > 0 and xm.xmem_residual_norm_backward_workspace_bytes(0, 64, 0) == 0
    for bad in ((-1, 64, 0), (8, 0, 0), (8, 64, 3), (1 << 31, 64, 0)):
        assert xm.xmem_residual_norm_backward_workspace_bytes(*bad) == 0
    for over in (dict(size=need - 1), dict(ws=None), dict(ws=(1 << 20) + 8)):
        assert back(**over) == EWORKSPACE
    no_sums = dict(ds=None, dw1=None, db1=None, dw2=None, db2=None)
    assert back(**no_sums, t=0, ws=None, size=0) == OK
    # a wide row's parts stay bounded, and never less than one group's
    for n in (1 << 20, 1 << 26, (1 << 31) - 1):
        assert 16 * n <= xm.xmem_residual_norm_backward_workspace_bytes(1 << 20, n, xm.XMEM_F32) <= max(1 << 28, 16 * n + 256)


def lookup(**over):
    a = dict(table=4096, ldt=64, ids=64, t=8, vocab=100, n=64, dtype=xm.XMEM_BF16, scale=1.0, padding=xm.XMEM_NO_PADDING, y=8192, ldy=64,
             stream=None)
    a.update(over)
    return xm.xmem_embedding_forward(*a.values())


@pytest.mark.parametrize("over", [
    dict(t=-1), dict(t=1 << 31), dict(vocab=0), dict(vocab=1 << 31), dict(n=0), dict(n=1 << 31), dict(dtype=3), dict(ldt=63), dict(ldy=63),
    dict(ldt=1 << 40), dict(table=None), dict(ids=None), dict(y=None)])
def test_embedding_forward_refuses(over):
    assert lookup(**over) == EINVAL


def table_grad(**over):
    a = dict(dy=4096, lddy=64, ids=64, t=8, vocab=100, n=64, dtype=xm.XMEM_BF16, scale=1.0, padding=xm.XMEM_NO_PADDING, add=0,
             out_dtype=xm.XMEM_F32, out=8192, ldd=64, ws=1 << 20, size=1 << 30, stream=None)
    a.update(over)
    return xm.xmem_embedding_backward(*a.values())


@pytest.mark.parametrize("over", [
    dict(t=-1), dict(t=1 << 31), dict(vocab=0), dict(vocab=1 << 31), dict(n=0), dict(n=1 << 31), dict(dtype=3), dict(out_dtype=xm.XMEM_F16),
    dict(dtype=xm.XMEM_F32, out_dtype=xm.XMEM_BF16), dict(lddy=63), dict(ldd=63), dict(dy=None), dict(ids=None), dict(out=None)])
def test_embedding_backward_refuses(over):
    assert table_grad(**over) == EINVAL


def test_embedding_of_nothing():
    assert lookup(t=0, table=None, ids=None, y=None) == OK
    assert table_grad(t=0, add=1, dy=None, ids=None, ws=None, size=0) == OK
    assert xm.xmem_embedding_backward_workspace_bytes(-1, 100, 64) == 0 == xm.xmem_embedding_backward_workspace_bytes(8, 0, 64)


def clip(at=(4096, 8192), sizes=(100, 200), kinds=(xm.XMEM_BF16, xm.XMEM_F32), count=None, max_norm=1.0, scale=1.0, stats=64, ws=1 << 20,
         size=1 << 20):
    return xm.xmem_clip_grad_norm(at, sizes, kinds, len(at or ()) if count is None else count, max_norm, scale, stats, ws, size, None)


@pytest.mark.parametrize("over", [
    dict(count=-1), dict(count=1 << 31), dict(at=None, count=2), dict(sizes=None), dict(kinds=None), dict(stats=None), dict(max_norm=-1.0),
    dict(max_norm=NAN), dict(scale=-1.0), dict(scale=NAN), dict(scale=INF), dict(sizes=(100, -1)), dict(sizes=(100, 1 << 48)),
    dict(kinds=(0, 3)), dict(at=(None, 8192)), dict(at=(4097, 8192)), dict(at=(4096, 8194)),
    # overlapping gradients: the same twice, and one that begins in another, in either order
    dict(at=(4096, 4096)), dict(at=(8192 + 796, 8192)), dict(at=(8192 - 198, 8192)), dict(at=(4096, 4096), scale=2.0, max_norm=INF)])
def test_clip_grad_norm_refuses(over):
    assert clip(**over) == EINVAL


def test_clip_grad_norm_workspace():
    need = xm.xmem_clip_grad_norm_workspace_bytes()
    for over in (dict(size=need - 1), dict(ws=None), dict(ws=(1 << 20) + 8)):
        assert clip(**over) == EWORKSPACE
    # neighbours do not overlap: what is refused then is the workspace
    assert clip(at=(8192 - 200, 8192), ws=None) == EWORKSPACE and clip(at=(4096, 4096), sizes=(0, 8), ws=None) == EWORKSPACE
    # the norm alone takes overlapping ones
    assert clip(at=(4096, 4096), max_norm=INF, ws=None) == EWORKSPACE


def test_python_calls_refuse_what_the_kernels_cannot_take():
    x, v, ids = torch.zeros(4, 8), torch.zeros(8), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: xm.residual_norm_forward(x),                                      # not on a GPU
                 lambda: xm.residual_norm_forward(x.double()),
                 lambda: xm.residual_norm_forward(x, pre="batch"),
                 lambda: xm.residual_norm_backward(x, None, x, torch.zeros(4, 4)),
                 lambda: xm.residual_norm_backward(None, None, x, torch.zeros(4, 4), pre="none"),
                 lambda: xm.residual_norm_backward(None, x, x, torch.zeros(4, 4)),
                 lambda: xm.embedding_forward(x, ids),
                 lambda: xm.embedding_backward(x, ids, 9),
                 lambda: xm.clip_grad_norm([x, v], 1.0),
                 lambda: xm.clip_grad_norm([], 1.0),
                 lambda: xm.clip_grad_norm([None], 1.0),
                 lambda: xm.clip_grad_norm([ids], 1.0)):
        with pytest.raises(xm.XmemError):
            call()
