"""The training operators' C ABI on the host (no GPU needed): what the header declares is exported, and every
argument check returns its code before any device work."""
import re
import subprocess
from pathlib import Path

import pytest
import torch

import paper_2510_21048_amd as xm
from paper_2510_21048_amd import ops

ROOT = Path(__file__).resolve().parents[1]
HEADER = ROOT / "include" / "ops" / "xmem_ops.h"
OK, EINVAL, EWORKSPACE = 0, -1, -5


def test_library_exports_what_the_header_declares():
    text = re.sub(r"/\*.*?\*/", "", HEADER.read_text(), flags=re.S)
    names = sorted(set(re.findall(r"^(?:int|size_t) (xmem_[a-z_]+)\(", text, flags=re.M)))
    assert names == sorted([
        "xmem_linear_forward", "xmem_linear_forward_workspace_bytes", "xmem_linear_backward",
        "xmem_linear_backward_workspace_bytes", "xmem_policy_loss", "xmem_policy_loss_workspace_bytes", "xmem_muon_update",
        "xmem_muon_update_workspace_bytes"])
    lib = xm.load_ops()
    for name in names:
        assert hasattr(lib, name) and hasattr(xm, name), name
    subprocess.run(["gcc", "-std=c99", "-fsyntax-only", "-x", "c", f"-I{ROOT / 'include'}", str(HEADER)], check=True)


def forward(**over):
    a = dict(x=4096, ldx=64, w=8192, ldw=64, bias=None, r=None, ldr=0, m=8, n=32, k=64, dtype=xm.XMEM_BF16, act=0, y=16384, ldy=32,
             z=None, ldz=0, ws=None, size=0, stream=None)
    a.update(over)
    return xm.xmem_linear_forward(*a.values())


@pytest.mark.parametrize("over", [
    dict(m=-1), dict(n=-1), dict(k=-1), dict(m=1 << 31), dict(ldx=63), dict(ldw=63), dict(ldy=31), dict(r=64, ldr=31), dict(z=64, ldz=31),
    dict(x=None), dict(w=None), dict(y=None), dict(dtype=xm.XMEM_F32), dict(dtype=-1), dict(act=4), dict(act=-1), dict(ldx=1 << 41)])
def test_linear_forward_refuses(over):
    assert forward(**over) == EINVAL


def test_linear_forward_of_nothing():
    assert forward(m=0, x=None, y=None) == OK and forward(n=0, ldy=0, w=None, y=None) == OK


def backward(**over):
    a = dict(dy=4096, lddy=32, z=8192, ldz=32, x=4096, ldx=64, w=8192, ldw=64, m=8, n=32, k=64, dtype=xm.XMEM_BF16, act=2, dx=16384,
             lddx=64, dw=32768, lddw=64, db=65536, ws=1 << 20, size=1 << 20, stream=None)
    a.update(over)
    return xm.xmem_linear_backward(*a.values())


@pytest.mark.parametrize("over", [
    dict(m=-1), dict(n=1 << 31), dict(lddy=31), dict(ldz=31), dict(ldx=63), dict(ldw=63), dict(lddx=63), dict(lddw=63), dict(dy=None),
    dict(z=None), dict(x=None), dict(w=None), dict(dtype=xm.XMEM_F32), dict(act=7)])
def test_linear_backward_refuses(over):
    assert backward(**over) == EINVAL


def test_linear_backward_workspace():
    need = xm.xmem_linear_backward_workspace_bytes(8, 32, 64, 32, 64, 64, 2)
    assert need > 0 and xm.xmem_linear_backward_workspace_bytes(8, -32, 64, 32, 64, 64, 2) == 0
    for over in (dict(size=need - 1), dict(ws=None), dict(ws=(1 << 20) + 8)):
        assert backward(**over) == EWORKSPACE
    assert backward(dx=None, dw=None, db=None) == OK


def policy(**over):
    a = dict(x=4096, ldl=100, y=8192, w=None, old=4096, adv=4096, ref=None, tokens=8, vocab=100, dtype=xm.XMEM_BF16, low=0.2, high=0.2,
             beta=0.1, scale=1.0, stats=4096, lp=4096, dx=1 << 20, ldd=100, ws=1 << 20, size=1 << 20, stream=None)
    a.update(over)
    return xm.xmem_policy_loss(*a.values())


@pytest.mark.parametrize("over", [
    dict(tokens=-1), dict(tokens=1 << 31), dict(vocab=0), dict(vocab=1 << 31), dict(dtype=3), dict(ldl=99), dict(ldd=99), dict(low=-0.1),
    dict(high=float("nan")), dict(old=None), dict(adv=None), dict(stats=None), dict(x=None), dict(y=None), dict(lp=None),
    dict(dx=4096, ldd=101), dict(old=None, adv=None, stats=None), dict(old=None, adv=None, stats=None, dx=None, ref=64)])
def test_policy_loss_refuses(over):
    assert policy(**over) == EINVAL


def test_policy_loss_workspace():
    need = xm.xmem_policy_loss_workspace_bytes(8, 100)
    assert need > 0 and xm.xmem_policy_loss_workspace_bytes(-8, 100) == 0 == xm.xmem_policy_loss_workspace_bytes(0, 100)
    for over in (dict(size=need - 1), dict(ws=None), dict(ws=(1 << 20) + 128)):
        assert policy(**over) == EWORKSPACE


def muon(**over):
    a = dict(g=4096, dtype=xm.XMEM_BF16, m=8192, count=2, rows=16, cols=24, mu=0.9, nesterov=1, steps=5, scale=1.0, up=16384, ws=1 << 20,
             size=1 << 30, stream=None)
    a.update(over)
    return xm.xmem_muon_update(*a.values())


@pytest.mark.parametrize("over", [
    dict(count=-1), dict(count=1 << 16), dict(rows=-1), dict(cols=1 << 24), dict(dtype=5), dict(steps=-1), dict(steps=17), dict(g=None),
    dict(m=None), dict(up=None)])
def test_muon_update_refuses(over):
    assert muon(**over) == EINVAL


def test_muon_update_workspace():
    need = xm.xmem_muon_update_workspace_bytes(2, 16, 24)
    assert need > 0 and xm.xmem_muon_update_workspace_bytes(0, 16, 24) == 0
    for over in (dict(size=need - 1), dict(ws=None), dict(ws=(1 << 20) + 8)):
        assert muon(**over) == EWORKSPACE
    assert muon(count=0, g=None, m=None, up=None) == OK and muon(rows=0) == OK


def test_python_calls_refuse_what_the_kernels_cannot_take():
    x, w = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(3, 8, dtype=torch.bfloat16)
    for call in (lambda: xm.linear_forward(x, w),                                    # not on a GPU
                 lambda: xm.linear_forward(x.float(), w),                            # not a 16-bit type
                 lambda: xm.linear_forward(x, w, activation="tanh"),
                 lambda: xm.linear_backward(x, x, w),
                 lambda: xm.token_logp(x, torch.zeros(4, dtype=torch.int64)),
                 lambda: xm.policy_loss(x, torch.zeros(4, dtype=torch.int64), None, torch.zeros(4), torch.zeros(4)),
                 lambda: xm.muon_update(x, torch.zeros(4, 8)),
                 lambda: ops._matrix(torch.zeros(4, 8).cuda() if torch.cuda.is_available() else torch.zeros(2, 2, 2), "x", 3)):
        with pytest.raises(xm.XmemError):
            call()


def test_missing_library_fails_loudly(monkeypatch, tmp_path):
    monkeypatch.setattr(ops, "_lib", None)
    monkeypatch.setattr(ops, "_LIB_PATH", tmp_path / "absent.so")
    with pytest.raises(xm.XmemError):
        ops.load_ops()


def test_calls_run_on_the_device_of_their_tensors(monkeypatch):
    """A tensor's device that is not the current one is made current for the call, on its own current stream; where it is
    current already nothing is switched."""
    entered, now = [], [0]

    class Device:
        def __init__(self, d):
            self.to = torch.device(d).index

        def __enter__(self):
            entered.append(self.to)
            self.back, now[0] = now[0], self.to

        def __exit__(self, *_):
            now[0] = self.back
            return False

    class Stream:
        cuda_stream = 4096

    monkeypatch.setattr(torch.cuda, "current_device", lambda: now[0])
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: Stream())
    monkeypatch.setattr(ops, "_raw_stream", lambda d: 4096)
    with ops._on(torch.device("cuda", 1), None) as on:
        assert now[0] == 1 and on.raw == 4096
    assert now[0] == 0 and entered == [1]
    for stream in (None, 4096):
        with ops._on(torch.device("cuda", 0), stream) as on:
            assert now[0] == 0 and on.raw == 4096
    assert entered == [1]
    with ops._on(torch.device("cuda", 1), 4096):
        assert now[0] == 1
    assert now[0] == 0


def test_workspace_is_checked():
    """A caller's workspace has to be contiguous memory of the tensors' device; its bytes count, not its elements."""
    cpu, meta = torch.device("cpu"), torch.device("meta")
    space = torch.empty(1024, dtype=torch.uint8, device=meta)
    for bad, dev in ((space, cpu), (space[::2], meta), (space.view(32, 32).T, meta)):
        for need in (0, 16):
            with pytest.raises(xm.XmemError):
                ops._workspace(bad, need, dev)
    assert ops._workspace(space, 1024, meta) == (space, 1024)
    floats = torch.empty(256, device=meta)
    assert ops._workspace(floats, 1024, meta) == (floats, 1024)
    own, size = ops._workspace(space, 1025, meta)
    assert own is not space and size == own.numel() == 1025
    assert ops._workspace(None, 0, meta) == (None, 0)


def test_inputs_that_require_a_gradient_are_refused(monkeypatch):
    """The calls record nothing for autograd: while it records, an input that requires a gradient is an error, not a result
    without one; under no_grad it is taken."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(ops, "_raw_stream", lambda d: 4096)
    plain, leaf = torch.zeros(3), torch.zeros(3, requires_grad=True)
    for given in ((leaf,), (plain, None, leaf), (plain, leaf * 2)):
        with pytest.raises(xm.XmemError, match="gradient"):
            ops._on(torch.device("cuda", 0), None, *given)
        with torch.no_grad():
            assert ops._on(torch.device("cuda", 0), None, *given).raw == 4096
        assert ops._on(torch.device("cuda", 0), None, *(None if t is None else t.detach() for t in given)).raw == 4096
