"""The operators of a transformer training step on torch tensors.

`binding` marshals the calls of eager_model.h with buffers that the caller owns; the functions
here check shapes, types and devices, allocate what the caller does not bring (outputs,
workspaces, through torch's allocator) and call them.  Outputs that are given (gradients of
weights in a process's gradient arena, parts of one buffer) are written in place.  All calls go to
the current stream, none of them waits.

A small call runs for a few microseconds, so the usual forms (tensors as described, all on the
current device) are checked and handed over by the extension module _marshal; whatever it does not
take comes back as NotImplemented and is checked and refused, or called, here.

    q, k = qk_norm_rope(q, k, wq, wk, cos, sin, positions)
    out, lse = attention(q, k, v, cu_seqlens)
    loss, lse = cross_entropy(x, w, target)
    y, s, stats = layer_norm(x, w, b, residual=r)
    q, k = rotary(q, k, cos, sin, positions)              # of rotary_table(positions, part)
    loss, lse, picked = distillation(x, w, index, logits, temperature)

each with its `_backward`, and `QKNormRope`, `Attention`, `CrossEntropy`, `LayerNorm`, `AddLayerNorm`, `Rotary`,
`Distillation` for torch's autograd (first derivatives; asked for the derivatives of gradients they raise).  All calls
can be captured into a graph, and so can a backward pass, with leaves of its own: torch ends the process when an eager
graph of the same leaves is still alive.
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional

import torch

from . import binding as eb

_DTYPES = {torch.float32: eb.F32, torch.bfloat16: eb.BF16}
_MAX_STRIDE = 1 << 21            # elements from row to row


def _refuse(text: str):
    raise eb.EagerError(eb.EINVAL, text)


def _dtype(*tensors) -> int:
    first = tensors[0]
    if first.dtype not in _DTYPES:
        _refuse(f"unsupported type {first.dtype}: float32 or bfloat16")
    for t in tensors:
        if t.dtype != first.dtype or t.device != first.device:
            _refuse(f"expected {first.dtype} on {first.device}, got {t.dtype} on {t.device}")
    if not first.is_cuda:
        _refuse("expected tensors on the GPU")
    return _DTYPES[first.dtype]


def _expect(t, shape, dtype, device, name, contiguous=True):
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype or t.device != device or (contiguous and not t.is_contiguous()):
        _refuse(f"{name}: expected {'contiguous ' if contiguous else ''}{dtype} {tuple(shape)} on {device}, got "
                f"{t.dtype} {tuple(t.shape)} with strides {t.stride()} on {t.device}")


def _workspace(nbytes: int, like):
    return like.new_empty(max(nbytes, 16), dtype=torch.uint8)


def _result(like):
    """A contiguous tensor of the same shape and type (in a third of the time of torch.empty with both named)."""
    return torch.empty_like(like, memory_format=torch.contiguous_format)


eb._marshal.bind_model(tuple(ctypes.cast(getattr(eb.lib, f), ctypes.c_void_p).value for f in (
    "eager_qk_norm_rope", "eager_qk_norm_rope_workspace_bytes", "eager_qk_norm_rope_backward",
    "eager_attention", "eager_attention_workspace_bytes", "eager_attention_backward",
    "eager_cross_entropy", "eager_cross_entropy_workspace_bytes", "eager_cross_entropy_backward",
    "eager_layer_norm", "eager_layer_norm_workspace_bytes", "eager_layer_norm_backward", "eager_rotary_table", "eager_rotary",
    "eager_rotary_backward", "eager_distillation", "eager_distillation_workspace_bytes", "eager_distillation_backward")),
    (torch.float32, torch.bfloat16, torch.int32, torch.int64), _workspace)


def _taken(status, what: str) -> bool:
    """Whether the extension module has made the call."""
    if status is NotImplemented:
        return False
    eb._status(status, what)
    return True


def _on(t):
    """Calls go to the current stream of the tensors' device."""
    return torch.cuda.device(t.device) if t.device.index != torch.cuda.current_device() else _NOTHING


class _Nothing:
    def __enter__(self):
        return None

    def __exit__(self, *_):
        return False


_NOTHING = _Nothing()


class _Once(torch.autograd.Function):
    """Gradients as they are, in a graph that wants to go on from them: it ends here with an error."""

    @staticmethod
    def forward(ctx, what, count, *tensors):
        ctx.what = what
        return tuple(t.view_as(t) for t in tensors[:count])

    @staticmethod
    def backward(ctx, *_):
        _refuse(f"{ctx.what}: second derivatives are not formed")


def _upstream(t):
    """A gradient [tokens, heads, head_dim] or [rows, width] that autograd hands over, copied only if the kernels do
    not take its strides (a broadcast or transposed one) or its place in memory."""
    each = 16 // t.element_size()
    if t.dim() == 2:
        row, one = t.stride()
        taken = one == 1 and row >= t.shape[1] and row % each == 0 and row <= _MAX_STRIDE and t.data_ptr() % 16 == 0
        return t if taken else t.clone(memory_format=torch.contiguous_format)
    row, head, one = t.stride()
    taken = (one == 1 and row >= t.shape[2] and head >= t.shape[2] and row % each == 0 and head % each == 0 and
             row <= _MAX_STRIDE and t.data_ptr() % 16 == 0)
    return t if taken else t.clone(memory_format=torch.contiguous_format)


def _once(what: str, grads, *depends):
    """The gradients that a backward pass returns.  In one that is recorded (create_graph) they depend on
    `depends`, through a node that refuses: without it they would count as constants there."""
    if not torch.is_grad_enabled():
        return tuple(grads)
    given = [g for g in grads if g is not None]
    marked = iter(_Once.apply(what, len(given), *given, *depends))
    return tuple(None if g is None else next(marked) for g in grads)


# ------------------------------------------------------------------------------ heads

def _rotation(q, cos, sin, positions):
    T, _, D = q.shape
    if cos.dim() != 2:
        _refuse("cos: expected [positions, head_dim / 2]")
    _expect(cos, (cos.shape[0], D // 2), torch.float32, q.device, "cos")
    _expect(sin, cos.shape, torch.float32, q.device, "sin")
    _expect(positions, (T,), torch.int32, q.device, "positions")
    return eb.Rotation(cos.data_ptr(), sin.data_ptr(), positions.data_ptr(), cos.shape[0])


def _heads_shape(q, k, wq, wk):
    if q.dim() != 3 or k.dim() != 3 or q.shape[0] != k.shape[0] or q.shape[2] != k.shape[2]:
        _refuse(f"expected q [tokens, q_heads, head_dim] and k [tokens, kv_heads, head_dim], got {tuple(q.shape)}, {tuple(k.shape)}")
    for w, name in ((wq, "wq"), (wk, "wk")):
        _expect(w, (q.shape[2],), q.dtype, q.device, name)
    return eb.packed(q.shape[0], q.shape[1], k.shape[1], q.shape[2])


def qk_norm_rope(q, k, wq, wk, cos, sin, positions, eps: float = 1e-6, q_out=None, k_out=None):
    """RMS norm of every head of q [tokens, q_heads, head_dim] and k [tokens, kv_heads, head_dim]
    with gains wq, wk [head_dim], then the rotation by `positions` (int32 [tokens]) of the tables
    cos, sin (fp32 [positions, head_dim / 2]).  q_out, k_out may be q, k."""
    q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device) if q_out is None else q_out
    k_out = torch.empty(k.shape, dtype=k.dtype, device=k.device) if k_out is None else k_out
    if _taken(eb._marshal.qk_norm_rope(q, k, wq, wk, cos, sin, positions, eps, q_out, k_out), "eager_qk_norm_rope"):
        return q_out, k_out
    dtype = _dtype(q, k)
    shape = _heads_shape(q, k, wq, wk)
    rotation = _rotation(q, cos, sin, positions)
    _expect(q_out, q.shape, q.dtype, q.device, "q_out", False)
    _expect(k_out, k.shape, k.dtype, k.device, "k_out", False)
    with _on(q):
        eb.eager_qk_norm_rope(dtype, shape, eb.heads(q), eb.heads(k), wq, wk, rotation, eps, eb.heads(q_out),
                              eb.heads(k_out))
    return q_out, k_out


def qk_norm_rope_backward(dq_out, dk_out, q, k, wq, wk, cos, sin, positions, eps: float = 1e-6, dq=None, dk=None,
                          dwq=None, dwk=None):
    """Gradients dq, dk, dwq, dwk from those of the outputs; dq, dk may be dq_out, dk_out."""
    dq = torch.empty(q.shape, dtype=q.dtype, device=q.device) if dq is None else dq
    dk = torch.empty(k.shape, dtype=k.dtype, device=k.device) if dk is None else dk
    dwq = torch.empty_like(wq) if dwq is None else dwq
    dwk = torch.empty_like(wk) if dwk is None else dwk
    if _taken(eb._marshal.qk_norm_rope(q, k, wq, wk, cos, sin, positions, eps, dq_out, dk_out, dq, dk, dwq, dwk),
              "eager_qk_norm_rope_backward"):
        return dq, dk, dwq, dwk
    dtype = _dtype(q, k, dq_out, dk_out)
    shape = _heads_shape(q, k, wq, wk)
    rotation = _rotation(q, cos, sin, positions)
    for t, like, name in ((dq_out, q, "dq_out"), (dk_out, k, "dk_out"), (dq, q, "dq"), (dk, k, "dk")):
        _expect(t, like.shape, q.dtype, q.device, name, False)
    for t, like, name in ((dwq, wq, "dwq"), (dwk, wk, "dwk")):
        _expect(t, like.shape, q.dtype, q.device, name)
    nbytes = eb.eager_qk_norm_rope_workspace_bytes(dtype, shape)
    with _on(q):
        eb.eager_qk_norm_rope_backward(dtype, shape, eb.heads(dq_out), eb.heads(dk_out), eb.heads(q), eb.heads(k), wq,
                                       wk, rotation, eps, eb.heads(dq), eb.heads(dk), dwq, dwk,
                                       _workspace(nbytes, q), nbytes)
    return dq, dk, dwq, dwk


class QKNormRope(torch.autograd.Function):
    """q, k = QKNormRope.apply(q, k, wq, wk, cos, sin, positions, eps)"""

    @staticmethod
    def forward(ctx, q, k, wq, wk, cos, sin, positions, eps):
        ctx.save_for_backward(q, k, wq, wk, cos, sin, positions)
        ctx.eps = eps
        return qk_norm_rope(q, k, wq, wk, cos, sin, positions, eps)

    @staticmethod
    def backward(ctx, dq_out, dk_out):
        q, k, wq, wk, cos, sin, positions = ctx.saved_tensors
        grads = qk_norm_rope_backward(_upstream(dq_out), _upstream(dk_out), q, k, wq, wk, cos, sin, positions, ctx.eps)
        return (*_once("QKNormRope", grads, dq_out, dk_out, q, k, wq, wk), None, None, None, None)


# ------------------------------------------------------------------------------ attention

def _packed_shape(q, k, v, cu_seqlens):
    if q.dim() != 3 or k.dim() != 3 or q.shape[0] != k.shape[0] or q.shape[2] != k.shape[2]:
        _refuse(f"expected q [tokens, q_heads, head_dim], k and v [tokens, kv_heads, head_dim], got {tuple(q.shape)}, {tuple(k.shape)}")
    _expect(v, k.shape, k.dtype, k.device, "v", False)
    if cu_seqlens.dim() != 1 or cu_seqlens.numel() < 2:
        _refuse("cu_seqlens: expected sequences + 1 values")
    _expect(cu_seqlens, cu_seqlens.shape, torch.int32, q.device, "cu_seqlens")
    return eb.packed(q.shape[0], q.shape[1], k.shape[1], q.shape[2], cu_seqlens)


def attention(q, k, v, cu_seqlens, scale: Optional[float] = None, out=None):
    """Causal attention inside each of the packed sequences [cu_seqlens[s], cu_seqlens[s + 1])
    (int32, on the GPU) of q [tokens, q_heads, head_dim] over k, v [tokens, kv_heads, head_dim].
    Returns out, like q, and the log-sum-exp of every row's scores, fp32 [q_heads, tokens]."""
    if q.dim() != 3:
        _refuse(f"expected q [tokens, q_heads, head_dim], got {tuple(q.shape)}")
    scale = 1.0 / math.sqrt(q.shape[2]) if scale is None else scale
    out = torch.empty(q.shape, dtype=q.dtype, device=q.device) if out is None else out
    lse = torch.empty((q.shape[1], q.shape[0]), dtype=torch.float32, device=q.device)
    if _taken(eb._marshal.attention(q, k, v, cu_seqlens, scale, out, lse), "eager_attention"):
        return out, lse
    dtype = _dtype(q, k, v)
    shape = _packed_shape(q, k, v, cu_seqlens)
    _expect(out, q.shape, q.dtype, q.device, "out", False)
    with _on(q):
        eb.eager_attention(dtype, shape, eb.heads(q), eb.heads(k), eb.heads(v), scale, eb.heads(out), lse)
    return out, lse


def attention_backward(dout, q, k, v, out, lse, cu_seqlens, scale: Optional[float] = None, dq=None, dk=None, dv=None):
    """Gradients dq, dk, dv from dout and what the forward pass took and gave."""
    if q.dim() != 3:
        _refuse(f"expected q [tokens, q_heads, head_dim], got {tuple(q.shape)}")
    scale = 1.0 / math.sqrt(q.shape[2]) if scale is None else scale
    dq, dk, dv = (torch.empty(x.shape, dtype=x.dtype, device=x.device) if d is None else d
                  for d, x in ((dq, q), (dk, k), (dv, v)))
    if _taken(eb._marshal.attention(q, k, v, cu_seqlens, scale, out, lse, dout, dq, dk, dv), "eager_attention_backward"):
        return dq, dk, dv
    dtype = _dtype(q, k, v, out, dout)
    shape = _packed_shape(q, k, v, cu_seqlens)
    for t, like, name in ((dout, q, "dout"), (out, q, "out"), (dq, q, "dq"), (dk, k, "dk"), (dv, v, "dv")):
        _expect(t, like.shape, q.dtype, q.device, name, False)
    _expect(lse, (q.shape[1], q.shape[0]), torch.float32, q.device, "lse")
    nbytes = eb.eager_attention_workspace_bytes(dtype, shape)
    with _on(q):
        eb.eager_attention_backward(dtype, shape, eb.heads(q), eb.heads(k), eb.heads(v), eb.heads(out), lse,
                                    eb.heads(dout), scale, eb.heads(dq), eb.heads(dk), eb.heads(dv), _workspace(nbytes, q), nbytes)
    return dq, dk, dv


class Attention(torch.autograd.Function):
    """out = Attention.apply(q, k, v, cu_seqlens, scale)"""

    @staticmethod
    def forward(ctx, q, k, v, cu_seqlens, scale):
        out, lse = attention(q, k, v, cu_seqlens, scale)
        ctx.save_for_backward(q, k, v, out, lse, cu_seqlens)
        ctx.scale = scale
        return out

    @staticmethod
    def backward(ctx, dout):
        q, k, v, out, lse, cu_seqlens = ctx.saved_tensors
        grads = attention_backward(_upstream(dout), q, k, v, out, lse, cu_seqlens, ctx.scale)
        return (*_once("Attention", grads, dout, q, k, v), None, None)


# ------------------------------------------------------------------------------ loss

def _sides(x, w):
    if x.dim() != 2 or w.dim() != 2 or x.shape[1] != w.shape[1] or x.stride(1) != 1 or w.stride(1) != 1:
        _refuse(f"expected x [rows, width] and w [vocab, width] with contiguous rows, got {tuple(x.shape)}, {tuple(w.shape)} "
                f"with strides {x.stride()}, {w.stride()}")
    # a lone row may have any stride
    return eb.Projection(x.shape[0], x.shape[1], w.shape[0], x.stride(0) if x.shape[0] > 1 else x.shape[1],
                         w.stride(0) if w.shape[0] > 1 else w.shape[1])


def _projection(x, w, target):
    shape = _sides(x, w)
    _expect(target, (x.shape[0],), torch.int64, x.device, "target")
    return shape


def cross_entropy(x, w, target):
    """Losses log sum exp(x w^T) - (x w^T)[target], fp32 [rows], and the log-sum-exps, of hidden
    states x [rows, width], projection w [vocab, width] and int64 targets; a negative target masks
    its row (loss 0).  No logits are kept."""
    loss = torch.empty(x.shape[0], dtype=torch.float32, device=x.device)
    lse = torch.empty(x.shape[0], dtype=torch.float32, device=x.device)
    if _taken(eb._marshal.cross_entropy(x, w, target, loss, lse), "eager_cross_entropy"):
        return loss, lse
    dtype = _dtype(x, w)
    shape = _projection(x, w, target)
    nbytes = eb.eager_cross_entropy_workspace_bytes(dtype, shape, False)
    with _on(x):
        eb.eager_cross_entropy(dtype, shape, x, w, target, loss, lse, _workspace(nbytes, x), nbytes)
    return loss, lse


def cross_entropy_backward(dloss, x, w, target, lse, dx=None, dw=None, want=(True, True)):
    """Gradients dx, dw from those of the losses (fp32 [rows]); want: which of the two are formed.
    dx and dw are laid out like x and w."""
    if dx is None and want[0]:
        dx = torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device=x.device)
    if dw is None and want[1]:
        dw = torch.empty_strided(w.shape, w.stride(), dtype=w.dtype, device=w.device)
    if _taken(eb._marshal.cross_entropy(x, w, target, lse, dloss, dx, dw), "eager_cross_entropy_backward"):
        return dx, dw
    dtype = _dtype(x, w)
    shape = _projection(x, w, target)
    _expect(dloss, target.shape, torch.float32, x.device, "dloss")
    _expect(lse, target.shape, torch.float32, x.device, "lse")
    for t, given, name in ((x, dx, "dx"), (w, dw, "dw")):
        if given is not None:
            _expect(given, t.shape, t.dtype, t.device, name, False)
            if given.stride(1) != 1 or (t.shape[0] > 1 and given.stride(0) != t.stride(0)):
                _refuse(f"{name}: expected strides {t.stride()}, got {given.stride()}")
    nbytes = eb.eager_cross_entropy_workspace_bytes(dtype, shape, True)
    with _on(x):
        eb.eager_cross_entropy_backward(dtype, shape, x, w, target, lse, dloss, dx, dw, _workspace(nbytes, x), nbytes)
    return dx, dw


class CrossEntropy(torch.autograd.Function):
    """losses = CrossEntropy.apply(x, w, target)"""

    @staticmethod
    def forward(ctx, x, w, target):
        loss, lse = cross_entropy(x, w, target)
        ctx.save_for_backward(x, w, target, lse)
        return loss

    @staticmethod
    def backward(ctx, dloss):
        x, w, target, lse = ctx.saved_tensors
        if not any(ctx.needs_input_grad[:2]):
            return None, None, None
        grads = cross_entropy_backward(dloss.contiguous(), x, w, target, lse, want=ctx.needs_input_grad[:2])
        return (*_once("CrossEntropy", grads, dloss, x, w), None)


# ------------------------------------------------------------------------------ hidden states

def _rows_shape(x, w, b):
    if x.dim() != 2:
        _refuse(f"expected rows [rows, width], got {tuple(x.shape)}")
    for t, name in ((w, "w"), (b, "b")):
        if t is not None:
            _expect(t, (x.shape[1],), x.dtype, x.device, name)


def layer_norm(x, w, b=None, eps: float = 1e-5, residual=None, s=None, y=None):
    """Layer norm of the rows of s = x + residual [rows, width] (of x, without one), with gain w and bias b (or none)
    [width]: y, s (x itself without a residual) and stats, fp32 [2, rows]: means and inverse deviations.  s and y may
    each be x or residual, but not the same one."""
    y = _result(x) if y is None else y
    if residual is not None and s is None:
        s = _result(x)
    if x.dim() != 2:
        _refuse(f"expected rows [rows, width], got {tuple(x.shape)}")
    stats = x.new_empty((2, x.shape[0]), dtype=torch.float32)
    if _taken(eb._marshal.layer_norm(x, residual, w, b, eps, s, y, stats), "eager_layer_norm"):
        return y, x if residual is None else s, stats
    if residual is None and s is not None:
        _refuse("s: there is no sum to store without a residual")
    dtype = _dtype(x)
    _rows_shape(x, w, b)
    for t, name in ((residual, "residual"), (s, "s"), (y, "y")):
        if t is not None:
            _expect(t, x.shape, x.dtype, x.device, name, False)
    with _on(x):
        eb.eager_layer_norm(dtype, x.shape[0], x.shape[1], eb.rows(x), residual if residual is None else eb.rows(residual), w, b,
                            eps, s if s is None else eb.rows(s), eb.rows(y), stats)
    return y, x if residual is None else s, stats


def layer_norm_backward(dy, s, w, stats, ds=None, dx=None, dw=None, db=None, want=(True, True)):
    """Gradients dx (of x and of the residual alike), dw, db from those of y and, where the sum s is used elsewhere,
    of s.  want: whether dw and db are formed.  dx may be dy or ds."""
    dx = _result(s) if dx is None else dx
    dw = torch.empty_like(w) if dw is None and want[0] else dw
    db = torch.empty_like(w) if db is None and want[1] else db
    if _taken(eb._marshal.layer_norm_backward(dy, ds, s, w, stats, dx, dw, db), "eager_layer_norm_backward"):
        return dx, dw, db
    dtype = _dtype(s)
    _rows_shape(s, w, None)
    for t, name in ((dy, "dy"), (ds, "ds"), (dx, "dx")):
        if t is not None:
            _expect(t, s.shape, s.dtype, s.device, name, False)
    for t, name in ((dw, "dw"), (db, "db")):
        if t is not None:
            _expect(t, w.shape, s.dtype, s.device, name)
    _expect(stats, (2, s.shape[0]), torch.float32, s.device, "stats")
    nbytes = eb.eager_layer_norm_workspace_bytes(dtype, s.shape[0], s.shape[1])
    with _on(s):
        eb.eager_layer_norm_backward(dtype, s.shape[0], s.shape[1], eb.rows(dy), ds if ds is None else eb.rows(ds), eb.rows(s), w,
                                     stats, eb.rows(dx), dw, db, _workspace(nbytes, s), nbytes)
    return dx, dw, db


class LayerNorm(torch.autograd.Function):
    """y = LayerNorm.apply(x, w, b, eps); b may be None"""

    @staticmethod
    def forward(ctx, x, w, b, eps):
        y, _, stats = layer_norm(x, w, b, eps)
        ctx.save_for_backward(x, w, stats)
        return y

    @staticmethod
    def backward(ctx, dy):
        x, w, stats = ctx.saved_tensors
        grads = layer_norm_backward(_upstream(dy), x, w, stats, want=ctx.needs_input_grad[1:3])
        return (*_once("LayerNorm", grads, dy, x, w), None)


class AddLayerNorm(torch.autograd.Function):
    """s, y = AddLayerNorm.apply(x, residual, w, b, eps): s = x + residual, y its layer norm; b may be None"""

    @staticmethod
    def forward(ctx, x, residual, w, b, eps):
        y, s, stats = layer_norm(x, w, b, eps, residual)
        ctx.save_for_backward(s, w, stats)
        ctx.set_materialize_grads(False)
        return s, y

    @staticmethod
    def backward(ctx, ds, dy):
        s, w, stats = ctx.saved_tensors
        if dy is None:                                   # the norm went nowhere
            grads = ds, None, None
        else:
            grads = layer_norm_backward(_upstream(dy), s, w, stats, None if ds is None else _upstream(ds),
                                        want=ctx.needs_input_grad[2:4])
        dx, dw, db = _once("AddLayerNorm", grads, *(t for t in (ds, dy) if t is not None), s, w)
        return dx, dx, dw, db, None


# ------------------------------------------------------------------------------ rotation

_SCALINGS = {"none": eb.ANGLES_PLAIN, "linear": eb.ANGLES_LINEAR, "base": eb.ANGLES_BASE, "parts": eb.ANGLES_PARTS}


def rotary_table(positions: int, part: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                 original: float = 0.0, low: float = 1.0, high: float = 32.0, magnitude: float = 1.0, device="cuda",
                 cos=None, sin=None):
    """Cosines and sines, fp32 [positions, part / 2], of the angles position * base^(-2 i / part), formed in 64 bits.
    Scaled for contexts longer than those of training by `factor`: "linear" divides every frequency by it, "base" the
    slowest by it and the others by less (a larger base), "parts" those of at most `low` turns over the `original`
    context, keeps those of `high` and more and goes from one to the other in between.  magnitude multiplies both
    tables."""
    if scaling not in _SCALINGS:
        _refuse(f"scaling: one of {', '.join(_SCALINGS)}, got {scaling!r}")
    if positions < 0 or part < 2:
        _refuse(f"expected a number of positions and of rotated elements, got {positions}, {part}")
    shape = (positions, part // 2)
    cos = torch.empty(shape, dtype=torch.float32, device=device) if cos is None else cos
    sin = torch.empty_like(cos) if sin is None else sin
    if _taken(eb._marshal.rotary_table(positions, part, _SCALINGS[scaling], base, factor, original, low, high, magnitude, cos, sin),
              "eager_rotary_table"):
        return cos, sin
    for t, name in ((cos, "cos"), (sin, "sin")):
        _expect(t, shape, torch.float32, cos.device, name)
    if not cos.is_cuda:
        _refuse("expected tensors on the GPU")
    with _on(cos):
        eb.eager_rotary_table(eb.Angles(positions, part, _SCALINGS[scaling], base, factor, original, low, high, magnitude),
                              cos, sin)
    return cos, sin


def _rotate(what, call, q, k, cos, sin, positions, interleaved, q_out, k_out, names):
    dtype = _dtype(q, k)
    if q.dim() != 3 or k.dim() != 3 or q.shape[0] != k.shape[0] or q.shape[2] != k.shape[2]:
        _refuse(f"{what}: expected [tokens, q_heads, head_dim] and [tokens, kv_heads, head_dim], got {tuple(q.shape)}, {tuple(k.shape)}")
    if cos.dim() != 2:
        _refuse("cos: expected [positions, part / 2]")
    _expect(cos, cos.shape, torch.float32, q.device, "cos")
    _expect(sin, cos.shape, torch.float32, q.device, "sin")
    _expect(positions, (q.shape[0],), torch.int32, q.device, "positions")
    _expect(q_out, q.shape, q.dtype, q.device, names[0], False)
    _expect(k_out, k.shape, k.dtype, k.device, names[1], False)
    shape = eb.packed(q.shape[0], q.shape[1], k.shape[1], q.shape[2])
    rotation = eb.Rotation(cos.data_ptr(), sin.data_ptr(), positions.data_ptr(), cos.shape[0])
    layout = eb.ROTARY_INTERLEAVED if interleaved else eb.ROTARY_HALVES
    with _on(q):
        call(dtype, shape, eb.heads(q), eb.heads(k), rotation, 2 * cos.shape[1], layout, eb.heads(q_out), eb.heads(k_out))


def rotary(q, k, cos, sin, positions, interleaved: bool = False, q_out=None, k_out=None):
    """The first part = 2 * cos.shape[1] elements of every head of q [tokens, q_heads, head_dim] and
    k [tokens, kv_heads, head_dim] turned by the angles of `positions` (int32 [tokens]) in the tables cos, sin (fp32
    [positions, part / 2]); the others as they are.  Pairs are the elements i and i + part / 2, or 2 i and 2 i + 1
    (interleaved).  q_out, k_out may be q, k."""
    q_out = _result(q) if q_out is None else q_out
    k_out = _result(k) if k_out is None else k_out
    if not _taken(eb._marshal.rotary(q, k, cos, sin, positions, bool(interleaved), q_out, k_out, False), "eager_rotary"):
        _rotate("rotary", eb.eager_rotary, q, k, cos, sin, positions, interleaved, q_out, k_out, ("q_out", "k_out"))
    return q_out, k_out


def rotary_backward(dq_out, dk_out, cos, sin, positions, interleaved: bool = False, dq=None, dk=None):
    """Gradients dq, dk from those of the outputs: turned back.  dq, dk may be dq_out, dk_out."""
    dq = _result(dq_out) if dq is None else dq
    dk = _result(dk_out) if dk is None else dk
    if not _taken(eb._marshal.rotary(dq_out, dk_out, cos, sin, positions, bool(interleaved), dq, dk, True), "eager_rotary_backward"):
        _rotate("rotary_backward", eb.eager_rotary_backward, dq_out, dk_out, cos, sin, positions, interleaved, dq, dk, ("dq", "dk"))
    return dq, dk


class Rotary(torch.autograd.Function):
    """q, k = Rotary.apply(q, k, cos, sin, positions, interleaved); the tables are constants: a backward pass through ones
    that require a gradient is refused"""

    @staticmethod
    def forward(ctx, q, k, cos, sin, positions, interleaved):
        ctx.save_for_backward(cos, sin, positions)
        ctx.interleaved = interleaved
        return rotary(q, k, cos, sin, positions, interleaved)

    @staticmethod
    def backward(ctx, dq_out, dk_out):
        if any(ctx.needs_input_grad[2:4]):
            _refuse("Rotary: gradients of the tables are not formed; detach them")
        cos, sin, positions = ctx.saved_tensors
        grads = rotary_backward(_upstream(dq_out), _upstream(dk_out), cos, sin, positions, ctx.interleaved)
        return (*_once("Rotary", grads, dq_out, dk_out), None, None, None, None)


# ------------------------------------------------------------------------------ a teacher's logits

def _teacher(x, index, logits, temperature):
    if index.dim() != 2 or index.shape[0] != x.shape[0]:
        _refuse(f"index: expected [rows, entries] for {x.shape[0]} rows, got {tuple(index.shape)}")
    _expect(index, index.shape, torch.int64, x.device, "index")
    _expect(logits, index.shape, torch.float32, x.device, "logits")
    return eb.Teacher(index.data_ptr(), logits.data_ptr(), index.shape[1], temperature)


def distillation(x, w, index, logits, temperature: float = 1.0):
    """Divergences sum q (log q - log p), fp32 [rows], of p = softmax(x w^T / temperature) from a teacher's
    q = softmax(logits / temperature) over the entries of each row: the words `index` (int64 [rows, entries]) with the
    teacher's `logits` (fp32 [rows, entries]); negative words count nothing, and a row without any has loss 0.  Also the
    log-sum-exps of x w^T / temperature and the student's logits of the entries (fp32 [rows, entries]).  The loss is not
    multiplied by the temperature's square."""
    loss = x.new_empty(x.shape[0], dtype=torch.float32)
    lse, picked = torch.empty_like(loss), _result(logits)
    if _taken(eb._marshal.distillation(x, w, index, logits, temperature, loss, lse, picked), "eager_distillation"):
        return loss, lse, picked
    dtype = _dtype(x, w)
    shape = _sides(x, w)
    teacher = _teacher(x, index, logits, temperature)
    nbytes = eb.eager_distillation_workspace_bytes(dtype, shape, index.shape[1], False)
    with _on(x):
        eb.eager_distillation(dtype, shape, x, w, teacher, loss, lse, picked, _workspace(nbytes, x), nbytes)
    return loss, lse, picked


def distillation_backward(dloss, x, w, index, logits, lse, picked, temperature: float = 1.0, dx=None, dw=None,
                          want=(True, True)):
    """Gradients dx, dw from those of the losses (fp32 [rows]) and what the forward pass took and gave; want: which of
    the two are formed.  dx and dw are laid out like x and w."""
    if dx is None and want[0]:
        dx = torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device=x.device)
    if dw is None and want[1]:
        dw = torch.empty_strided(w.shape, w.stride(), dtype=w.dtype, device=w.device)
    if _taken(eb._marshal.distillation(x, w, index, logits, temperature, lse, picked, dloss, dx, dw), "eager_distillation_backward"):
        return dx, dw
    dtype = _dtype(x, w)
    shape = _sides(x, w)
    teacher = _teacher(x, index, logits, temperature)
    _expect(picked, index.shape, torch.float32, x.device, "picked")
    for t, name in ((lse, "lse"), (dloss, "dloss")):
        _expect(t, (x.shape[0],), torch.float32, x.device, name)
    for t, given, name in ((x, dx, "dx"), (w, dw, "dw")):
        if given is not None:
            _expect(given, t.shape, t.dtype, t.device, name, False)
            if given.stride(1) != 1 or (t.shape[0] > 1 and given.stride(0) != t.stride(0)):
                _refuse(f"{name}: expected strides {t.stride()}, got {given.stride()}")
    nbytes = eb.eager_distillation_workspace_bytes(dtype, shape, index.shape[1], True)
    with _on(x):
        eb.eager_distillation_backward(dtype, shape, x, w, teacher, lse, picked, dloss, dx, dw, _workspace(nbytes, x), nbytes)
    return dx, dw


class Distillation(torch.autograd.Function):
    """losses = Distillation.apply(x, w, index, logits, temperature); the teacher's logits are constants: a backward pass
    through ones that require a gradient is refused"""

    @staticmethod
    def forward(ctx, x, w, index, logits, temperature):
        loss, lse, picked = distillation(x, w, index, logits, temperature)
        ctx.save_for_backward(x, w, index, logits, lse, picked)
        ctx.temperature = temperature
        return loss

    @staticmethod
    def backward(ctx, dloss):
        if ctx.needs_input_grad[3]:
            _refuse("Distillation: gradients of the teacher's logits are not formed; detach them")
        x, w, index, logits, lse, picked = ctx.saved_tensors
        if not any(ctx.needs_input_grad[:2]):
            return None, None, None, None, None
        grads = distillation_backward(dloss.contiguous(), x, w, index, logits, lse, picked, ctx.temperature,
                                      want=ctx.needs_input_grad[:2])
        return (*_once("Distillation", grads, dloss, x, w), None, None, None)
