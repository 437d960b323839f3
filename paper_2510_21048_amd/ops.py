"""ctypes binding of libxmem_ops.so (argument marshalling only): the operators of a dense
training step that allocate nothing by themselves (include/ops/xmem_ops.h).

The functions named ``xmem_*`` mirror the C ABI one to one and take raw device
pointers (ints) or torch CUDA tensors; ``linear_forward``, ``linear_backward``,
``policy_loss``, ``token_logp`` and ``muon_update`` check their tensors, allocate
outputs and workspace with torch and run on the current torch stream, or on the
raw ``stream`` given (then nothing waits for the current one by itself: the inputs
have to be ready on it).  They are no part of autograd's graph (the gradients are
calls of their own): inputs that require one are refused while it is recorded, so
call them on detached tensors, under ``torch.no_grad()`` or in a
``torch.autograd.Function``.
"""
from __future__ import annotations

import ctypes
from pathlib import Path

from .binding import XMEM_OK, XmemError, _ptr, xmem_strerror

_LIB_PATH = Path(__file__).resolve().parent / "libxmem_ops.so"

XMEM_BF16, XMEM_F16, XMEM_F32 = 0, 1, 2
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
XMEM_NS_MAX_STEPS = 16

_lib = None
_dtypes: dict = {}  # torch's types -> the C ABI's, filled when the library is loaded


def ops_lib_path() -> Path:
    return _LIB_PATH


def load_ops():
    """Load the operators' library; raises if it has not been built (no fallback)."""
    global _lib
    if _lib is None:
        if not _LIB_PATH.exists():
            raise XmemError(f"{_LIB_PATH} is missing: build it with paper_2510_21048_amd.build.build()")
        lib = ctypes.CDLL(str(_LIB_PATH))
        vp, i64, i32, f32, size = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
        for name, args, res in (
            ("xmem_linear_forward_workspace_bytes", [i64] * 5, size),
            ("xmem_linear_forward", [vp, i64, vp, i64, vp, vp, i64, i64, i64, i64, i32, i32, vp, i64, vp, i64, vp, size, vp], i32),
            ("xmem_linear_backward_workspace_bytes", [i64] * 6 + [i32], size),
            ("xmem_linear_backward", [vp, i64] * 4 + [i64] * 3 + [i32] * 2 + [vp, i64] * 2 + [vp, vp, size, vp], i32),
            ("xmem_policy_loss_workspace_bytes", [i64] * 2, size),
            ("xmem_policy_loss", [vp, i64] + [vp] * 5 + [i64] * 2 + [i32] + [f32] * 4 + [vp] * 3 + [i64, vp, size, vp], i32),
            ("xmem_muon_update_workspace_bytes", [i64] * 3, size),
            ("xmem_muon_update", [vp, i32, vp] + [i64] * 3 + [f32, i32, i32, f32, vp, vp, size, vp], i32),
        ):
            f = getattr(lib, name)
            f.argtypes, f.restype = args, res
        import torch
        _dtypes.update({torch.bfloat16: XMEM_BF16, torch.float16: XMEM_F16, torch.float32: XMEM_F32})
        _lib = lib
    return _lib


# ---------------------------------------------------------------- the C ABI


def xmem_linear_forward_workspace_bytes(m: int, n: int, k: int, ldx: int, ldw: int) -> int:
    return load_ops().xmem_linear_forward_workspace_bytes(m, n, k, ldx, ldw)


def xmem_linear_forward(d_x, ldx, d_w, ldw, d_bias, d_residual, ldr, m, n, k, dtype, activation, d_y, ldy, d_z, ldz,
                        d_workspace, workspace_bytes, stream) -> int:
    return load_ops().xmem_linear_forward(_ptr(d_x), ldx, _ptr(d_w), ldw, _ptr(d_bias), _ptr(d_residual), ldr, m, n, k, dtype,
                                          activation, _ptr(d_y), ldy, _ptr(d_z), ldz, _ptr(d_workspace), workspace_bytes,
                                          _ptr(stream))


def xmem_linear_backward_workspace_bytes(m: int, n: int, k: int, lddy: int, ldx: int, ldw: int, activation: int) -> int:
    return load_ops().xmem_linear_backward_workspace_bytes(m, n, k, lddy, ldx, ldw, activation)


def xmem_linear_backward(d_dy, lddy, d_z, ldz, d_x, ldx, d_w, ldw, m, n, k, dtype, activation, d_dx, lddx, d_dw, lddw, d_db,
                         d_workspace, workspace_bytes, stream) -> int:
    return load_ops().xmem_linear_backward(_ptr(d_dy), lddy, _ptr(d_z), ldz, _ptr(d_x), ldx, _ptr(d_w), ldw, m, n, k, dtype,
                                           activation, _ptr(d_dx), lddx, _ptr(d_dw), lddw, _ptr(d_db), _ptr(d_workspace),
                                           workspace_bytes, _ptr(stream))


def xmem_policy_loss_workspace_bytes(tokens: int, vocab: int) -> int:
    return load_ops().xmem_policy_loss_workspace_bytes(tokens, vocab)


def xmem_policy_loss(d_logits, ldl, d_tokens, d_weights, d_old_logp, d_advantages, d_ref_logp, tokens, vocab, dtype, clip_low,
                     clip_high, kl_coef, grad_scale, d_stats, d_logp, d_dlogits, ldd, d_workspace, workspace_bytes,
                     stream) -> int:
    return load_ops().xmem_policy_loss(_ptr(d_logits), ldl, _ptr(d_tokens), _ptr(d_weights), _ptr(d_old_logp),
                                       _ptr(d_advantages), _ptr(d_ref_logp), tokens, vocab, dtype, clip_low, clip_high, kl_coef,
                                       grad_scale, _ptr(d_stats), _ptr(d_logp), _ptr(d_dlogits), ldd, _ptr(d_workspace),
                                       workspace_bytes, _ptr(stream))


def xmem_muon_update_workspace_bytes(count: int, rows: int, cols: int) -> int:
    return load_ops().xmem_muon_update_workspace_bytes(count, rows, cols)


def xmem_muon_update(d_grad, grad_dtype, d_momentum, count, rows, cols, mu, nesterov, steps, scale, d_update, d_workspace,
                     workspace_bytes, stream) -> int:
    return load_ops().xmem_muon_update(_ptr(d_grad), grad_dtype, _ptr(d_momentum), count, rows, cols, mu, int(nesterov), steps,
                                       scale, _ptr(d_update), _ptr(d_workspace), workspace_bytes, _ptr(stream))


# ---------------------------------------------------------------- on torch tensors


# A small call costs its host as much as the GPU: these look at each tensor once, and ask torch for little.


def _check(rc: int, what: str) -> None:
    if rc != XMEM_OK:
        raise XmemError(f"{what}: {xmem_strerror(rc)} ({rc})")


def _dtype(t, what: str, allow=(XMEM_BF16, XMEM_F16)) -> int:
    code = _dtypes.get(t.dtype)
    if code not in allow:
        raise XmemError(f"{what}: {t.dtype} is not supported here")
    return code


def _matrix(t, what: str, rows: int | None = None, cols: int | None = None, dtype=None, device=None) -> int:
    """Row distance of a 2-d tensor whose rows are contiguous; raises on anything else."""
    shape = t.shape
    if len(shape) != 2 or (rows is not None and shape[0] != rows) or (cols is not None and shape[1] != cols):
        raise XmemError(f"{what}: shape {tuple(shape)} where ({'*' if rows is None else rows}, {'*' if cols is None else cols}) is wanted")
    if dtype is not None and t.dtype != dtype:
        raise XmemError(f"{what}: {t.dtype} where {dtype} is wanted")
    if not t.is_cuda or (device is not None and t.device != device):
        raise XmemError(f"{what}: on {t.device}" + ("" if device is None else f" where {device} is wanted"))
    r, c = shape
    ld, along = t.stride()
    if c > 1 and along != 1 and r:
        raise XmemError(f"{what}: its rows are not contiguous (strides {t.stride()})")
    if r <= 1:
        return c
    if ld < c:
        if c and r:
            raise XmemError(f"{what}: its rows overlap (strides {t.stride()})")
        return c
    return ld


def _vector(t, what: str, n: int, dtype, device):
    if t is not None and (t.shape != (n,) or t.dtype != dtype or t.device != device or (n > 1 and t.stride(0) != 1)):
        raise XmemError(f"{what}: a contiguous {dtype} [{n}] on {device} is wanted, got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t


def _workspace(workspace, need: int, device):
    """The caller's workspace where it is large enough, else one of torch's."""
    if workspace is not None and (workspace.device != device or not workspace.is_contiguous()):
        raise XmemError(f"workspace: a contiguous tensor on {device} is wanted, got strides {workspace.stride()} on {workspace.device}")
    if need == 0:
        return None, 0
    if workspace is not None and workspace.nbytes >= need:
        return workspace, workspace.nbytes
    import torch
    return torch.empty(need, dtype=torch.uint8, device=device), need


def _raw_stream(device) -> int:
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)  # what current_stream() wraps, at a tenth of its time
    return raw(device.index) if raw is not None else torch.cuda.current_stream(device).cuda_stream


class _Here:
    """A call on the current stream: torch's allocator orders what it takes by that stream already."""

    __slots__ = ("raw",)

    def __init__(self, raw):
        self.raw = raw

    def __enter__(self):
        return self

    def __exit__(self, kind, value, trace):
        return False

    def out(self, *tensors):
        return tensors if len(tensors) > 1 else tensors[0]


class _There:
    """A call on another stream or device than the current one.  Launches go to the current device, so the tensors' own is
    made current.  Outputs and workspace are taken from the stream's memory, which the allocator gives to nothing else before
    what the stream has been asked for, and what both streams see is kept until both are done with it."""

    def __init__(self, device, raw, given):
        import torch
        self.raw = raw
        self.before = torch.cuda.current_stream(device)
        if raw == self.before.cuda_stream:
            self.context = torch.cuda.device(device)
            return
        stream = torch.cuda.ExternalStream(raw, device=device)
        for t in given:
            if t is not None and t.is_cuda:
                t.record_stream(stream)
        self.context = torch.cuda.stream(stream)

    def __enter__(self):
        self.context.__enter__()
        return self

    def __exit__(self, *raised):
        return self.context.__exit__(*raised)

    def out(self, *tensors):
        for t in tensors:
            if t is not None:
                t.record_stream(self.before)
        return tensors if len(tensors) > 1 else tensors[0]


def _on(device, stream, *given):
    """Where a call on checked tensors (the workspace among them) runs."""
    import torch
    if torch.is_grad_enabled():
        for t in given:
            if t is not None and t.requires_grad:
                raise XmemError("an input requires a gradient, which is not recorded here: detach it or call under torch.no_grad()")
    here = _raw_stream(device)
    raw = here if stream is None else stream
    return _Here(here) if raw == here and torch.cuda.current_device() == device.index else _There(device, raw, given)


def _written(tensor) -> None:
    """An input was overwritten: a graph that saved it has to see that, as after torch's own in-place operations."""
    import torch
    torch.autograd.graph.increment_version(tensor)


def _activation(name: str) -> int:
    if name not in ACTIVATIONS:
        raise XmemError(f"activation {name!r}: one of {', '.join(ACTIVATIONS)} is wanted")
    return ACTIVATIONS[name]


def linear_forward(x, w, bias=None, residual=None, activation: str = "none", save_z: bool = False, workspace=None, stream=None):
    """y = act(x w^T + bias) + residual on torch CUDA tensors: x [m, k], w [n, k], residual [m, n] in bfloat16 or
    float16 (rows may be strided), bias float32 [n].  Returns (y, z): z = x w^T + bias where save_z (what
    ``linear_backward`` needs of an activation), else None."""
    import torch
    lib = load_ops()
    act, code, dt, dev = _activation(activation), _dtype(x, "x"), x.dtype, x.device
    ldx, (m, k) = _matrix(x, "x"), x.shape
    ldw, n = _matrix(w, "w", None, k, dt, dev), w.shape[0]
    ldr = 0 if residual is None else _matrix(residual, "residual", m, n, dt, dev)
    _vector(bias, "bias", n, torch.float32, dev)
    with _on(dev, stream, x, w, bias, residual, workspace) as on:
        y = x.new_empty((m, n))
        z = x.new_empty((m, n)) if save_z else None
        workspace, size = _workspace(workspace, lib.xmem_linear_forward_workspace_bytes(m, n, k, ldx, ldw), dev)
        _check(xmem_linear_forward(x, ldx, w, ldw, bias, residual, ldr, m, n, k, code, act, y, n, z, n, workspace, size, on.raw),
               "xmem_linear_forward")
        return on.out(y, z)


def linear_backward(dy, x, w, z=None, activation: str = "none", need_dx: bool = True, need_dw: bool = True, need_db: bool = True,
                    workspace=None, stream=None):
    """Gradients of ``linear_forward`` for an output gradient dy [m, n]; z as it was saved (not looked at without an activation).
    Returns (dx [m, k], dw [n, k], db float32 [n]), None in the place of what is not needed.  The residual's gradient
    is dy itself."""
    import torch
    load_ops()
    act, code, dev = _activation(activation), _dtype(dy, "dy"), dy.device
    lddy = _matrix(dy, "dy")
    m, n = dy.shape
    k = x.shape[1] if x.dim() == 2 else 0
    ldx, ldw = _matrix(x, "x", m, None, dy.dtype, dev), _matrix(w, "w", n, k, dy.dtype, dev)
    if z is None and act != ACTIVATIONS["none"]:
        raise XmemError("z: wanted with an activation (linear_forward's save_z)")
    ldz = 0 if z is None else _matrix(z, "z", m, n, dy.dtype, dev)
    with _on(dev, stream, dy, x, w, z, workspace) as on:
        dx = dy.new_empty((m, k)) if need_dx else None
        dw = dy.new_empty((n, k)) if need_dw else None
        db = torch.empty(n, dtype=torch.float32, device=dev) if need_db else None
        workspace, size = _workspace(workspace, xmem_linear_backward_workspace_bytes(m, n, k, lddy, ldx, ldw, act), dev)
        _check(xmem_linear_backward(dy, lddy, z, ldz, x, ldx, w, ldw, m, n, k, code, act, dx, k, dw, k, db, workspace, size, on.raw),
               "xmem_linear_backward")
        return on.out(dx, dw, db)


_ANY = (XMEM_BF16, XMEM_F16, XMEM_F32)


def token_logp(logits, tokens, weights=None, stream=None):
    """Log-probabilities float32 [t] of the tokens (int64 [t]) under logits [t, v] (bfloat16, float16 or float32, rows
    may be strided); 0 where the weight is."""
    import torch
    load_ops()
    code, dev, ldl = _dtype(logits, "logits", _ANY), logits.device, _matrix(logits, "logits")
    t, v = logits.shape
    _vector(tokens, "tokens", t, torch.int64, dev)
    _vector(weights, "weights", t, torch.float32, dev)
    with _on(dev, stream, logits, tokens, weights) as on:
        logp = torch.empty(t, dtype=torch.float32, device=dev)
        _check(xmem_policy_loss(logits, ldl, tokens, weights, None, None, None, t, v, code, 0.0, 0.0, 0.0, 1.0, None, logp, None, 0,
                                None, 0, on.raw), "xmem_policy_loss")
        return on.out(logp)


def policy_loss(logits, tokens, weights, old_logp, advantages, ref_logp=None, clip_low: float = 0.2, clip_high: float = 0.2,
                kl_coef: float = 0.0, grad_scale: float = 1.0, need_dlogits: bool = True, in_place: bool = False, workspace=None,
                stream=None):
    """The clipped policy loss with a KL term and the logits' gradient (xmem_policy_loss): logits [t, v], tokens int64
    [t], the rest float32 [t]; weights (None: 1/t each) carry the mask and the normalisation.  Returns (stats float32
    [4]: loss, policy part, KL part, clipped weight; logp float32 [t]; dlogits, which is logits itself with in_place,
    or None)."""
    import torch
    load_ops()
    code, dev, ldl = _dtype(logits, "logits", _ANY), logits.device, _matrix(logits, "logits")
    t, v = logits.shape
    _vector(tokens, "tokens", t, torch.int64, dev)
    if old_logp is None or advantages is None:
        raise XmemError("old_logp and advantages are wanted (token_logp needs neither)")
    for a, name in ((weights, "weights"), (old_logp, "old_logp"), (advantages, "advantages"), (ref_logp, "ref_logp")):
        _vector(a, name, t, torch.float32, dev)
    with _on(dev, stream, logits, tokens, weights, old_logp, advantages, ref_logp, workspace) as on:
        stats = torch.empty(4, dtype=torch.float32, device=dev)
        logp = torch.empty(t, dtype=torch.float32, device=dev)
        dlogits, ldd = None, 0
        if need_dlogits:
            dlogits, ldd = (logits, ldl) if in_place else (logits.new_empty((t, v)), v)
        workspace, size = _workspace(workspace, xmem_policy_loss_workspace_bytes(t, v), dev)
        _check(xmem_policy_loss(logits, ldl, tokens, weights, old_logp, advantages, ref_logp, t, v, code, clip_low, clip_high,
                                kl_coef, grad_scale, stats, logp, dlogits, ldd, workspace, size, on.raw), "xmem_policy_loss")
        if dlogits is logits:
            _written(logits)
        return on.out(stats, logp, dlogits)


def muon_update(grad, momentum, mu: float = 0.95, nesterov: bool = True, steps: int = 5, scale: float = 1.0, workspace=None,
                stream=None):
    """Momentum (float32, updated in place) and the orthogonalised update (bfloat16, returned) of matrices: grad
    [rows, cols] or [count, rows, cols], contiguous, bfloat16, float16 or float32."""
    import torch
    load_ops()
    code, dev = _dtype(grad, "grad", _ANY), grad.device
    if grad.dim() not in (2, 3) or not grad.is_cuda or not grad.is_contiguous():
        raise XmemError("grad: a contiguous CUDA tensor of 2 or 3 dimensions is wanted")
    if momentum.shape != grad.shape or momentum.dtype != torch.float32 or momentum.device != dev or not momentum.is_contiguous():
        raise XmemError("momentum: a contiguous float32 tensor shaped as grad is wanted")
    count, (rows, cols) = (1 if grad.dim() == 2 else grad.shape[0]), grad.shape[-2:]
    with _on(dev, stream, grad, momentum, workspace) as on:
        update = torch.empty(grad.shape, dtype=torch.bfloat16, device=dev)
        workspace, size = _workspace(workspace, xmem_muon_update_workspace_bytes(count, rows, cols), dev)
        _check(xmem_muon_update(grad, code, momentum, count, rows, cols, mu, nesterov, steps, scale, update, workspace, size, on.raw),
               "xmem_muon_update")
        _written(momentum)
        return on.out(update)
