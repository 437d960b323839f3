"""ctypes binding of libxmem_ops.so (argument marshalling only), continued: what a training step does around its
products (include/ops/xmem_step.h).

The functions named ``xmem_*`` mirror the C ABI one to one and take raw device pointers (ints) or torch CUDA tensors;
``residual_norm_forward``, ``residual_norm_backward``, ``embedding_forward``, ``embedding_backward`` and
``clip_grad_norm`` check their tensors, allocate outputs and workspace with torch and run on the current torch stream
or the raw ``stream`` given, as the calls in ``ops`` do: inputs that require a gradient are refused while one is
recorded, and what a call overwrites counts as modified.  An input or a workspace that shares memory with what a
call overwrites is refused.
"""
from __future__ import annotations

import ctypes
from array import array

from .binding import XmemError, _ptr
from .ops import _ANY, XMEM_F32, _check, _dtype, _dtypes, _matrix, _on, _vector, _workspace, _written, load_ops

NORMS = {"none": 0, "rms": 1, "layer": 2}
GATES = {"none": 0, "sigmoid": 1, "silu": 2}
XMEM_NO_PADDING = -(1 << 63)


# ---------------------------------------------------------------- the C ABI


def xmem_residual_norm_forward(d_r, ldr, d_h, ldh, d_gate, ldg, d_scale, alpha, post, d_w1, d_b1, pre, d_w2, d_b2, gate_activation, eps,
                               tokens, width, dtype, d_out, ldo, d_y, ldy, d_stats, stream) -> int:
    return load_ops().xmem_residual_norm_forward(_ptr(d_r), ldr, _ptr(d_h), ldh, _ptr(d_gate), ldg, _ptr(d_scale), alpha, post, _ptr(d_w1),
                                                 _ptr(d_b1), pre, _ptr(d_w2), _ptr(d_b2), gate_activation, eps, tokens, width, dtype,
                                                 _ptr(d_out), ldo, _ptr(d_y), ldy, _ptr(d_stats), _ptr(stream))


def xmem_residual_norm_backward_workspace_bytes(tokens: int, width: int, dtype: int) -> int:
    return load_ops().xmem_residual_norm_backward_workspace_bytes(tokens, width, dtype)


def xmem_residual_norm_backward(d_dy, lddy, d_dout, lddout, d_out, ldo, d_stats, d_h, ldh, d_gate, ldg, d_scale, alpha, post, d_w1, d_b1,
                                pre, d_w2, gate_activation, tokens, width, dtype, d_dr, lddr, d_dh, lddh, d_dgate, lddg, d_dscale, d_dw1,
                                d_db1, d_dw2, d_db2, d_workspace, workspace_bytes, stream) -> int:
    return load_ops().xmem_residual_norm_backward(_ptr(d_dy), lddy, _ptr(d_dout), lddout, _ptr(d_out), ldo, _ptr(d_stats), _ptr(d_h), ldh,
                                                  _ptr(d_gate), ldg, _ptr(d_scale), alpha, post, _ptr(d_w1), _ptr(d_b1), pre, _ptr(d_w2),
                                                  gate_activation, tokens, width, dtype, _ptr(d_dr), lddr, _ptr(d_dh), lddh, _ptr(d_dgate),
                                                  lddg, _ptr(d_dscale), _ptr(d_dw1), _ptr(d_db1), _ptr(d_dw2), _ptr(d_db2),
                                                  _ptr(d_workspace), workspace_bytes, _ptr(stream))


def xmem_embedding_forward(d_table, ldt, d_ids, tokens, vocab, width, dtype, scale, padding_id, d_y, ldy, stream) -> int:
    return load_ops().xmem_embedding_forward(_ptr(d_table), ldt, _ptr(d_ids), tokens, vocab, width, dtype, scale, padding_id, _ptr(d_y), ldy,
                                             _ptr(stream))


def xmem_embedding_backward_workspace_bytes(tokens: int, vocab: int, width: int) -> int:
    return load_ops().xmem_embedding_backward_workspace_bytes(tokens, vocab, width)


def xmem_embedding_backward(d_dy, lddy, d_ids, tokens, vocab, width, dtype, scale, padding_id, add, out_dtype, d_dtable, ldd, d_workspace,
                            workspace_bytes, stream) -> int:
    return load_ops().xmem_embedding_backward(_ptr(d_dy), lddy, _ptr(d_ids), tokens, vocab, width, dtype, scale, padding_id, int(add),
                                              out_dtype, _ptr(d_dtable), ldd, _ptr(d_workspace), workspace_bytes, _ptr(stream))


def xmem_clip_grad_norm_workspace_bytes() -> int:
    return load_ops().xmem_clip_grad_norm_workspace_bytes()


def xmem_clip_grad_norm(d_tensors, sizes, dtypes, count, max_norm, scale, d_stats, d_workspace, workspace_bytes, stream) -> int:
    """d_tensors, sizes, dtypes: sequences of device pointers (or tensors), of numbers of elements and of element types."""
    at = None if d_tensors is None else (ctypes.c_void_p * len(d_tensors))(*map(_ptr, d_tensors))
    n = None if sizes is None else (ctypes.c_int64 * len(sizes))(*sizes)
    kinds = None if dtypes is None else (ctypes.c_int * len(dtypes))(*dtypes)
    return load_ops().xmem_clip_grad_norm(at, n, kinds, count, max_norm, scale, _ptr(d_stats), _ptr(d_workspace), workspace_bytes,
                                          _ptr(stream))


# ---------------------------------------------------------------- on torch tensors


def _norm(name: str, what: str) -> int:
    if name not in NORMS:
        raise XmemError(f"{what} {name!r}: one of {', '.join(NORMS)} is wanted")
    return NORMS[name]


def _gate(name: str) -> int:
    if name not in GATES:
        raise XmemError(f"gate_activation {name!r}: one of {', '.join(GATES)} is wanted")
    return GATES[name]


def _at(t):
    return None if t is None else t.data_ptr()


def _no(what: str, why: str, *given) -> None:
    for t in given:
        if t is not None:
            raise XmemError(f"{what}: not without {why}")


def _rows(t):
    """First byte, bytes of a row, from row to row, and rows of a matrix or of what lies in one piece."""
    if t.is_contiguous():
        return t.data_ptr(), t.nbytes, t.nbytes, 1
    (r, c), size = t.shape, t.element_size()
    return t.data_ptr(), c * size, t.stride(0) * size, r


def _apart(over, name: str, **read) -> None:
    """Refuses tensors that a call reads while it writes `over`: their rows may lie between its rows (halves of one matrix), not on them."""
    mine = _rows(over)
    begin, end = mine[0], mine[0] + (mine[3] - 1) * mine[2] + mine[1]
    for what, t in read.items():
        if t is None:
            continue
        first = t.data_ptr()
        if first >= end or (first + t.nbytes <= begin and t.is_contiguous()) or not t.numel() or begin == end:  # most are far away
            continue
        (at, wide, ld, r), (at2, wide2, ld2, r2) = sorted((mine, _rows(t)))
        gap = at2 - at
        if gap >= (r - 1) * ld + wide:
            continue
        if r > 1 and (r2 == 1 or ld == ld2) and wide <= gap % ld <= ld - wide2:
            continue
        raise XmemError(f"{what}: shares memory with {name}, which is overwritten")


def residual_norm_forward(residual, h=None, gate=None, scale=None, alpha: float = 1.0, post: str = "none", post_weight=None, post_bias=None,
                          pre: str = "rms", pre_weight=None, pre_bias=None, gate_activation: str = "none", eps: float = 1e-5,
                          save_stats: bool = False, in_place: bool = False, stream=None):
    """Between two blocks of a residual stream: out = residual + alpha scale a(gate) (norm(h) post_weight + post_bias), y = norm(out)
    pre_weight + pre_bias.  residual, h (the block's output) and gate are [t, n] in bfloat16, float16 or float32 (rows may be strided),
    scale, weights and biases float32 [n]; post and pre are "none", "rms" or "layer"; a is what ``gate_activation`` says ("none": the
    gate itself, "sigmoid", "silu").  Without h, y is the norm of residual.  Returns (out, which is residual itself with in_place or
    without h; y, or None with pre "none"; stats float32 [4, t] where save_stats (what ``residual_norm_backward`` needs), else None)."""
    import torch
    lib = load_ops()
    code, dt, dev, ldr = _dtype(residual, "residual", _ANY), residual.dtype, residual.device, _matrix(residual, "residual")
    t, n = residual.shape
    k1, k2, act = _norm(post, "post"), _norm(pre, "pre"), _gate(gate_activation)
    ldh = ldg = 0
    if h is None:
        _no("gate, scale", "h", gate, scale)
        if k1:
            raise XmemError("post: a norm of h, which is not given")
    else:
        ldh = _matrix(h, "h", t, n, dt, dev)
    if gate is not None:
        ldg = _matrix(gate, "gate", t, n, dt, dev)
    if not k1:
        _no("post_weight, post_bias", "post", post_weight, post_bias)
    if not k2:
        _no("pre_weight, pre_bias", "pre", pre_weight, pre_bias)
    for v, name in ((scale, "scale"), (post_weight, "post_weight"), (post_bias, "post_bias"), (pre_weight, "pre_weight"), (pre_bias, "pre_bias")):
        if v is not None:
            _vector(v, name, n, torch.float32, dev)
    if in_place and h is not None:
        _apart(residual, "residual", h=h, gate=gate, scale=scale, post_weight=post_weight, post_bias=post_bias, pre_weight=pre_weight,
               pre_bias=pre_bias)
    with _on(dev, stream, residual, h, gate, scale, post_weight, post_bias, pre_weight, pre_bias) as on:
        out, ldo = (residual, ldr) if in_place or h is None else (residual.new_empty((t, n)), n)
        y = residual.new_empty((t, n)) if k2 else None
        stats = torch.empty((4, t), dtype=torch.float32, device=dev) if save_stats else None
        _check(lib.xmem_residual_norm_forward(residual.data_ptr(), ldr, _at(h), ldh, _at(gate), ldg, _at(scale), alpha, k1, _at(post_weight),
                                              _at(post_bias), k2, _at(pre_weight), _at(pre_bias), act, eps, t, n, code,
                                              None if h is None else out.data_ptr(), ldo, _at(y), n, _at(stats), on.raw),
               "xmem_residual_norm_forward")
        if out is residual and h is not None:
            _written(residual)
        return on.out(out, y, stats)


def residual_norm_backward(dy, dout, out, stats, h=None, gate=None, scale=None, alpha: float = 1.0, post: str = "none", post_weight=None,
                           post_bias=None, pre: str = "rms", pre_weight=None, pre_bias=None, gate_activation: str = "none",
                           need_vectors: bool = True, in_place: bool = False, workspace=None, stream=None):
    """Gradients of ``residual_norm_forward`` for dy of y (None with pre "none") and dout of out (None: nothing else came from it): out
    and stats as that call returned them, the rest as it was given.  Returns the gradients of (residual, which is dout itself with
    in_place; h; gate; scale; post_weight; post_bias; pre_weight; pre_bias), None in the place of what was not given, and of the five
    vectors without need_vectors."""
    import torch
    lib = load_ops()
    k1, k2, act = _norm(post, "post"), _norm(pre, "pre"), _gate(gate_activation)
    if (dy is None) == (k2 != 0):
        raise XmemError("dy: wanted with a norm before the next block, and only then")
    if dy is None and dout is None:
        raise XmemError("dout: wanted without dy")
    if stats is None or (out is None and dy is not None):
        raise XmemError("out, stats: wanted as residual_norm_forward returned them (save_stats)")
    first = dout if dy is None else dy
    code, dt, dev = _dtype(first, "dout" if dy is None else "dy", _ANY), first.dtype, first.device
    lddy = 0 if dy is None else _matrix(dy, "dy")
    t, n = first.shape if first.dim() == 2 else (0, 0)
    lddo = 0 if dout is None else _matrix(dout, "dout", t, n, dt, dev)
    ldo = 0 if dy is None else _matrix(out, "out", t, n, dt, dev)
    if stats.shape != (4, t) or stats.dtype != torch.float32 or stats.device != dev or not stats.is_contiguous():
        raise XmemError("stats: a contiguous float32 [4, t] is wanted (residual_norm_forward's save_stats)")
    ldh = ldg = 0
    if h is None:
        _no("gate, scale", "h", gate, scale)
        if k1:
            raise XmemError("post: a norm of h, which is not given")
    else:
        ldh = _matrix(h, "h", t, n, dt, dev)
    if gate is not None:
        ldg = _matrix(gate, "gate", t, n, dt, dev)
    if not k1:
        _no("post_weight, post_bias", "post", post_weight, post_bias)
    if not k2:
        _no("pre_weight, pre_bias", "pre", pre_weight, pre_bias)
    if in_place and dout is None:
        raise XmemError("in_place: dout is wanted")
    vectors = (scale, post_weight, post_bias, pre_weight, pre_bias)
    for v, name in zip(vectors, ("scale", "post_weight", "post_bias", "pre_weight", "pre_bias")):
        if v is not None:
            _vector(v, name, n, torch.float32, dev)
    if in_place:
        _apart(dout, "dout", dy=dy, out=None if dy is None else out, stats=stats, h=h, gate=gate, scale=scale, post_weight=post_weight,
               post_bias=post_bias, pre_weight=pre_weight, pre_bias=pre_bias)
    with _on(dev, stream, dy, dout, out, stats, h, gate, *vectors, workspace) as on:
        dr, lddr = (dout, lddo) if in_place else (first.new_empty((t, n)), n)
        dh = None if h is None else first.new_empty((t, n))
        dg = None if gate is None else first.new_empty((t, n))
        sums = [None if v is None or not need_vectors else torch.empty(n, dtype=torch.float32, device=dev) for v in vectors]
        wanted = any(v is not None for v in sums)
        workspace, size = _workspace(workspace, lib.xmem_residual_norm_backward_workspace_bytes(t, n, code) if wanted else 0, dev)
        _check(lib.xmem_residual_norm_backward(_at(dy), lddy, _at(dout), lddo, None if dy is None else out.data_ptr(), ldo, stats.data_ptr(),
                                               _at(h), ldh, _at(gate), ldg, _at(scale), alpha, k1, _at(post_weight), _at(post_bias), k2,
                                               _at(pre_weight), act, t, n, code, dr.data_ptr(), lddr, _at(dh), n, _at(dg), n, *map(_at, sums),
                                               _at(workspace), size, on.raw), "xmem_residual_norm_backward")
        if in_place:
            _written(dout)
        return on.out(dr, dh, dg, *sums)


def embedding_forward(table, ids, scale: float = 1.0, padding_id: int | None = None, stream=None):
    """y [t, n] = scale table[ids]: table [vocab, n] in bfloat16, float16 or float32 (rows may be strided), ids int64 [t].  A token equal
    to padding_id gives a row of 0, any other outside [0, vocab) a row of NaN."""
    import torch
    load_ops()
    code, dev, ldt = _dtype(table, "table", _ANY), table.device, _matrix(table, "table")
    (vocab, n), t = table.shape, ids.shape[0] if ids.dim() == 1 else -1
    _vector(ids, "ids", t, torch.int64, dev)
    with _on(dev, stream, table, ids) as on:
        y = table.new_empty((t, n))
        _check(xmem_embedding_forward(table, ldt, ids, t, vocab, n, code, scale, XMEM_NO_PADDING if padding_id is None else padding_id, y, n,
                                      on.raw), "xmem_embedding_forward")
        return on.out(y)


def embedding_backward(dy, ids, vocab: int, scale: float = 1.0, padding_id: int | None = None, into=None, dtype=None, workspace=None,
                       stream=None):
    """The gradient [vocab, n] of ``embedding_forward``'s table for dy [t, n]: scale times the sum of each token's rows, in 32 bits and
    a fixed order.  Tokens equal to padding_id or outside [0, vocab) add nothing; rows without a token are 0.  It is of dy's type, or float32 with ``dtype``; with
    ``into`` (either type, rows may be strided) it is added to that, which is returned."""
    import torch
    load_ops()
    code, dev, lddy = _dtype(dy, "dy", _ANY), dy.device, _matrix(dy, "dy")
    t, n = dy.shape
    _vector(ids, "ids", t, torch.int64, dev)
    if dtype is None:
        dtype = dy.dtype if into is None else into.dtype
    if dtype not in (dy.dtype, torch.float32):
        raise XmemError(f"dtype: {dy.dtype} or float32 is wanted, got {dtype}")
    ldd = n if into is None else _matrix(into, "into", vocab, n, dtype, dev)
    if vocab < 1:
        raise XmemError("vocab: at least 1 is wanted")
    if into is not None:
        _apart(into, "into", dy=dy, ids=ids)
    with _on(dev, stream, dy, ids, into, workspace) as on:
        out = torch.empty((vocab, n), dtype=dtype, device=dev) if into is None else into
        workspace, size = _workspace(workspace, xmem_embedding_backward_workspace_bytes(t, vocab, n), dev)
        _check(xmem_embedding_backward(dy, lddy, ids, t, vocab, n, code, scale, XMEM_NO_PADDING if padding_id is None else padding_id,
                                       into is not None, XMEM_F32 if dtype == torch.float32 else code, out, ldd, workspace, size, on.raw),
               "xmem_embedding_backward")
        if into is not None:
            _written(into)
        return on.out(out)


def clip_grad_norm(grads, max_norm: float, scale: float = 1.0, workspace=None, stream=None):
    """The 2-norm of all gradients as one vector, times scale, and their scaling in place: each is multiplied by factor = scale min(1,
    max_norm / (norm + 1e-6)).  grads: tensors of any shapes in bfloat16, float16 or float32 on one device, each contiguous (or the
    transpose of one that is), None among them left out.  Returns float32 [2]: norm and factor, on the device.  max_norm = math.inf
    with scale 1 computes the norm alone."""
    import torch
    lib = load_ops()
    grads = [g for g in grads if g is not None]
    if not grads:
        raise XmemError("grads: at least one tensor is wanted")
    dev = grads[0].device
    where = dev.index if dev.type == "cuda" else None
    try:
        kinds = [_dtypes[g.dtype] for g in grads]
    except KeyError as e:
        raise XmemError(f"grads: {e.args[0]} is not supported here") from None
    for g in grads:
        if g.get_device() != where or not (g.is_contiguous() or (g.dim() > 1 and g.mT.is_contiguous())):
            raise XmemError(f"grads: contiguous tensors on one GPU are wanted, got strides {g.stride()} on {g.device}")
    at, sizes, kinds = array("Q", [g.data_ptr() for g in grads]), array("q", [g.numel() for g in grads]), array("i", kinds)
    with _on(dev, stream, *grads, workspace) as on:
        stats = torch.empty(2, dtype=torch.float32, device=dev)
        workspace, size = _workspace(workspace, lib.xmem_clip_grad_norm_workspace_bytes(), dev)
        _check(lib.xmem_clip_grad_norm(at.buffer_info()[0], sizes.buffer_info()[0], kinds.buffer_info()[0], len(grads), max_norm, scale,
                                       stats.data_ptr(), workspace.data_ptr(), size, on.raw), "xmem_clip_grad_norm")
        if max_norm != float("inf") or scale != 1.0:
            _written(grads)
        return on.out(stats)
