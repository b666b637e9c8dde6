"""Layers on learned vertex rows (see include/coop.h for the contract of every call): a dense layer with its epilogue, the projections of
a gated feed-forward block, the norms and the residual between two blocks, and the gradients' norm ahead of an AdamW step.

What an activation was of is worth keeping (want_pre, then pre=) for rows of some 1,000 elements and more; for shorter ones the gradient call makes it
again in less time than 32 bits of it take to be written and read, and in no memory.

Marshalling only, as in binding.py and learn.py; streams are as there.
"""
import ctypes as C
import functools

import torch

from . import binding
from .binding import _check, _stream_ptr
from .learn import COOP_F32, _DTYPES, _matrix, _new, _vector, _workspace

COOP_ACT_NONE, COOP_ACT_RELU, COOP_ACT_GELU, COOP_ACT_SILU = 0, 1, 2, 3
_AFTER, _BEFORE, _RMS = 1, 2, 4


class _CGradTensor(C.Structure):
    _fields_ = [("grad", C.c_void_p), ("n_rows_dev", C.c_void_p), ("n_rows", C.c_int64), ("dim", C.c_int64), ("dtype", C.c_int32), ("reserved", C.c_int32)]


_P, _I, _L, _F, _S = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_size_t
_SIGNATURES = {
    "coop_linear_workspace_bytes": (_S, [_L, _I, _I, C.c_int, C.c_int]),
    "coop_linear": (C.c_int, [_P, _L, _I, _P, _I, C.c_int, _P, C.c_int, _F, _P, _P, _P, _P, _S, _P]),
    "coop_linear_grad_workspace_bytes": (_S, [_L, _I, _I, C.c_int, C.c_int, C.c_int, C.c_int]),
    "coop_linear_grad": (C.c_int, [_P, _P, _L, _I, _P, _I, C.c_int, _P, C.c_int, _F, _P, _P, _P, C.c_int, _P, _P, _S, _P]),
    "coop_gated_workspace_bytes": (_S, [_L, _I, _I, C.c_int, C.c_int]),
    "coop_gated": (C.c_int, [_P, _L, _I, _P, _P, _I, C.c_int, _P, _P, C.c_int, _P, _P, _P, _S, _P]),
    "coop_gated_grad_workspace_bytes": (_S, [_L, _I, _I, C.c_int, C.c_int, C.c_int]),
    "coop_gated_grad": (C.c_int, [_P, _P, _L, _I, _P, _P, _I, C.c_int, _P, _P, C.c_int, _P, _P, _P, _P, C.c_int, _P, _P, _P, _S, _P]),
    "coop_residual_norm": (C.c_int, [_P, _P, _L, _I, C.c_int, C.c_int, _P, C.c_int, _F, C.c_int] + [_P] * 4 + [C.c_int, _F] + [_P] * 4),
    "coop_residual_norm_grad_workspace_bytes": (_S, [_L, _I, C.c_int]),
    "coop_residual_norm_grad": (C.c_int, [_P] * 4 + [_L, _I, C.c_int, C.c_int, _P, _P, C.c_int, _F, C.c_int] + [_P] * 3 + [C.c_int] + [_P] * 8 + [_S, _P]),
    "coop_grad_norm_workspace_bytes": (_S, [_P, C.c_int]),
    "coop_grad_norm": (C.c_int, [_P, C.c_int, C.c_double, _P, _P, _P, _P, _S, _P]),
    "coop_grad_scale": (C.c_int, [_P, C.c_int, _P, _P]),
}
_lib = None


def lib():
    global _lib
    if _lib is None:
        L = binding.lib()
        for name, (res, args) in _SIGNATURES.items():
            f = getattr(L, name)
            f.restype, f.argtypes = res, args
        _lib = L
    return _lib


@functools.lru_cache(maxsize=4096)
def _need(call, *sizes):
    """Bytes of workspace that a call of these sizes takes."""
    return getattr(lib(), call + "_workspace_bytes")(*sizes)


def _same(t, like, what, rows=None, dim=None):
    p = _matrix(t, what, rows, dim)
    assert t.dtype == like.dtype, "%s: %s" % (what, like.dtype)
    return p


# (of a result like an argument; torch.empty with a type and a device takes half a microsecond more)
def _new_like(t, stream, shape=None):
    if stream is None:
        return torch.empty_like(t) if shape is None else t.new_empty(shape)
    return _new(shape or t.shape, t.dtype, t.device, stream)


def _bias(b, n, like, what):
    return None if b is None else _vector(b, n, like.dtype, what)


def _kept(pre, shape):
    if pre is None:
        return None
    assert pre.is_cuda and pre.is_contiguous() and pre.dtype == torch.float32 and tuple(pre.shape) == shape, "pre: contiguous fp32 %s" % (shape,)
    return pre.data_ptr()


def coop_linear(x, weight, bias=None, act=COOP_ACT_NONE, alpha=1.0, residual=None, want_pre=False, out=None, workspace=None, stream=None):
    """alpha act(x weight^T + bias) + residual, for x [n, k] and weight [m, k]; with want_pre (it, what the activation was of, fp32 [n, m])."""
    xp, wp = _matrix(x, "x"), _same(weight, x, "weight", dim=x.shape[1])
    (n, k), m, dtype = x.shape, weight.shape[0], _DTYPES[x.dtype]
    if out is None:
        out = _new_like(x, stream, (n, m))
    op = _same(out, x, "out", n, m)
    pre = _new((n, m), torch.float32, x.device, stream) if want_pre else None
    rp = None if residual is None else _same(residual, x, "residual", n, m)
    keep, sp, sb = _workspace(_need("coop_linear", n, k, m, dtype, (xp | wp) & 15 == 0), workspace, x.device, stream)
    _check(lib().coop_linear(xp, n, k, wp, m, dtype, _bias(bias, m, x, "bias"), act, alpha, rp, op, pre.data_ptr() if want_pre else None, sp, sb,
                             _stream_ptr(stream)))
    return (out, pre) if want_pre else out


def coop_linear_grad(dout, x, weight, bias=None, pre=None, act=COOP_ACT_NONE, alpha=1.0, want_x=True, want_weight=True, want_bias=True,
                     grad_dtype=None, workspace=None, stream=None):
    """(dx, dweight, dbias) of coop_linear; None for one that is not wanted.  pre: what it kept; without it that is computed again, with the
    bias.  grad_dtype: of dweight (the weight's, or fp32); dbias is fp32.  The residual's gradient is dout."""
    xp, wp = _matrix(x, "x"), _same(weight, x, "weight", dim=x.shape[1])
    (n, k), m, dtype = x.shape, weight.shape[0], _DTYPES[x.dtype]
    dp = _same(dout, x, "dout", n, m)
    grad_dtype = grad_dtype or x.dtype
    dx = _new_like(x, stream) if want_x else None
    dw = _new((m, k), grad_dtype, x.device, stream) if want_weight else None
    db = _new(m, torch.float32, x.device, stream) if want_bias else None
    need = _need("coop_linear_grad", n, k, m, dtype, act, pre is not None, (xp | wp | dp) & 15 == 0)
    keep, sp, sb = _workspace(need, workspace, x.device, stream)
    _check(lib().coop_linear_grad(dp, xp, n, k, wp, m, dtype, _bias(bias, m, x, "bias"), act, alpha, _kept(pre, (n, m)),
                                  dx.data_ptr() if want_x else None, dw.data_ptr() if want_weight else None, _DTYPES[grad_dtype],
                                  db.data_ptr() if want_bias else None, sp, sb, _stream_ptr(stream)))
    return dx, dw, db


def coop_gated(x, gate, up, gate_bias=None, up_bias=None, act=COOP_ACT_SILU, want_pre=False, out=None, workspace=None, stream=None):
    """act(x gate^T + gate_bias) (x up^T + up_bias), for x [n, k] and gate, up [f, k]; with want_pre (it, both factors' products, fp32 [2, n, f])."""
    xp, gp = _matrix(x, "x"), _same(gate, x, "gate", dim=x.shape[1])
    (n, k), f, dtype = x.shape, gate.shape[0], _DTYPES[x.dtype]
    upp = _same(up, x, "up", f, k)
    if out is None:
        out = _new_like(x, stream, (n, f))
    op = _same(out, x, "out", n, f)
    pre = _new((2, n, f), torch.float32, x.device, stream) if want_pre else None
    keep, sp, sb = _workspace(_need("coop_gated", n, k, f, dtype, (xp | gp | upp) & 15 == 0), workspace, x.device, stream)
    _check(lib().coop_gated(xp, n, k, gp, upp, f, dtype, _bias(gate_bias, f, x, "gate_bias"), _bias(up_bias, f, x, "up_bias"), act, op,
                            pre.data_ptr() if want_pre else None, sp, sb, _stream_ptr(stream)))
    return (out, pre) if want_pre else out


def coop_gated_grad(dout, x, gate, up, gate_bias=None, up_bias=None, pre=None, act=COOP_ACT_SILU, want_x=True, want_weight=True, want_bias=True,
                    grad_dtype=None, workspace=None, stream=None):
    """(dx, dgate, dup, dgate_bias, dup_bias) of coop_gated; None for those that are not wanted.  pre, grad_dtype: as in coop_linear_grad."""
    xp, gp = _matrix(x, "x"), _same(gate, x, "gate", dim=x.shape[1])
    (n, k), f, dtype = x.shape, gate.shape[0], _DTYPES[x.dtype]
    upp, dp = _same(up, x, "up", f, k), _same(dout, x, "dout", n, f)
    grad_dtype = grad_dtype or x.dtype
    dx = _new_like(x, stream) if want_x else None
    dw = [_new((f, k), grad_dtype, x.device, stream) for _ in range(2)] if want_weight else [None] * 2
    db = [_new(f, torch.float32, x.device, stream) for _ in range(2)] if want_bias else [None] * 2
    need = _need("coop_gated_grad", n, k, f, dtype, pre is not None, (xp | gp | upp) & 15 == 0)
    keep, sp, sb = _workspace(need, workspace, x.device, stream)
    _check(lib().coop_gated_grad(dp, xp, n, k, gp, upp, f, dtype, _bias(gate_bias, f, x, "gate_bias"), _bias(up_bias, f, x, "up_bias"), act,
                                 _kept(pre, (2, n, f)), dx.data_ptr() if want_x else None, *(w.data_ptr() if want_weight else None for w in dw),
                                 _DTYPES[grad_dtype], *(b.data_ptr() if want_bias else None for b in db), sp, sb, _stream_ptr(stream)))
    return (dx, *dw, *db)


def _seam(x, f, gate, after, after_weight, after_bias, before, before_weight, before_bias, rms):
    """(shape, types, gate form, flags, addresses) that both calls have in common"""
    fp, (n, dim) = _matrix(f, "f"), f.shape
    assert after or after_weight is None and after_bias is None, "without the norm behind the block it has no weights"
    assert before or before_weight is None and before_bias is None, "without the norm in front of the next block it has no weights"
    assert not rms or after_bias is None and before_bias is None, "a root-mean-square norm has no bias"
    columns = gate is not None and gate.dim() == 1
    dtype, ps = None, []
    for w in (gate if columns else None, after_weight, after_bias, before_weight, before_bias):
        if w is None:
            ps.append(None)
            continue
        if dtype is None:
            dtype = w.dtype
            assert dtype in _DTYPES, "weights, biases and the columns' gate have one type: fp32, fp16 or bf16"
        ps.append(_vector(w, dim, dtype, "weight"))
    gp = ps.pop(0)
    if gate is not None and not columns:
        gp = _same(gate, f, "gate", n, dim)
    return (fp, n, dim, COOP_F32 if dtype is None else _DTYPES[dtype], gp, 0 if gate is None else 1 if columns else 2,
            after * _AFTER | before * _BEFORE | rms * _RMS, ps)


def coop_residual_norm(x, f, gate=None, alpha=1.0, after=True, after_weight=None, after_bias=None, before=True, before_weight=None, before_bias=None,
                       rms=False, eps=1e-5, out=None, stream=None):
    """(r, y, stats): r = alpha x + gate N_after(f), the residual stream behind a block, and y = N_before(r), the next block's input (None with
    before=False; after=False: f itself).  x [n, dim]: of f's type or fp32; gate: None, [dim] (of the weights' type) or [n, dim] (of f's); out: for r."""
    fp, n, dim, weight_dtype, gp, form, norms, ps = _seam(x, f, gate, after, after_weight, after_bias, before, before_weight, before_bias, rms)
    xp = _matrix(x, "x", n, dim)
    assert x.dtype in (torch.float32, f.dtype), "x: fp32 or f's type"
    if out is None:
        out = _new_like(x, stream)
    op = _same(out, x, "out", n, dim)
    y = _new_like(f, stream) if before else None
    stats = _new((4, n), torch.float32, x.device, stream)
    _check(lib().coop_residual_norm(xp, fp, n, dim, _DTYPES[f.dtype], _DTYPES[x.dtype], gp, form, alpha, norms, *ps, weight_dtype, eps, op,
                                    y.data_ptr() if before else None, stats.data_ptr(), _stream_ptr(stream)))
    return out, y, stats


def coop_residual_norm_grad(dr, dy, x, f, stats, gate=None, alpha=1.0, after=True, after_weight=None, after_bias=None, before=True, before_weight=None,
                            rms=False, want_weight=True, workspace=None, stream=None):
    """(dx, df, dgate, dafter_weight, dafter_bias, dbefore_weight, dbefore_bias) of coop_residual_norm, from the gradients of r (None: zeros)
    and y; x, f as they were given, and what the gate and the norms had.  None for what there is not, and for the last four with
    want_weight=False; those and the gradient of a gate [dim] are fp32."""
    fp, n, dim, weight_dtype, gp, form, norms, ps = _seam(x, f, gate, after, after_weight, after_bias, before, before_weight, None, rms)
    xp = _matrix(x, "x", n, dim)
    assert x.dtype in (torch.float32, f.dtype), "x: fp32 or f's type"
    rp = None if dr is None else _same(dr, x, "dr", n, dim)
    yp = _same(dy, f, "dy", n, dim) if before else None
    assert before or dr is not None, "without the norm in front of the next block r's gradient is all there is"
    assert stats.is_cuda and stats.is_contiguous() and stats.dtype == torch.float32 and tuple(stats.shape) == (4, n), "stats: as coop_residual_norm gives them"
    dx, df = _new_like(x, stream), _new_like(f, stream)
    # (the sums over the rows, fp32 [dim]: one allocation for all of them)
    there = (form == 1, *(want_weight and t for t in (after, after and not rms, before, before and not rms)))
    sums = iter(_new((sum(there), dim), torch.float32, x.device, stream).unbind() if any(there) else ())
    dgate, *grads = (next(sums) if t else None for t in there)
    if form == 2:
        dgate = _new_like(gate, stream)
    need = _need("coop_residual_norm_grad", n, dim, _DTYPES[f.dtype]) if want_weight or form == 1 else 0
    keep, wp, wb = _workspace(need, workspace, x.device, stream)
    _check(lib().coop_residual_norm_grad(rp, yp, xp, fp, n, dim, _DTYPES[f.dtype], _DTYPES[x.dtype], stats.data_ptr(), gp, form, alpha, norms, *ps[:3],
                                         weight_dtype, dx.data_ptr(), df.data_ptr(), None if gate is None else dgate.data_ptr(),
                                         *(None if g is None else g.data_ptr() for g in grads), wp, wb, _stream_ptr(stream)))
    return (dx, df, dgate, *grads)


class GradNorm:
    """The norm of many gradients together and the factor that clips it (coop_grad_norm), over the tensors that hold the gradients at every step
    (set_grads replaces them).  A gradient of touched rows, as coop_embed_grad_rows returns it without waiting, is given as (gradients, count)."""

    def __init__(self, grads):
        self.set_grads(grads)

    def set_grads(self, grads):
        grads = [g if isinstance(g, (tuple, list)) else (g, None) for g in grads]
        for g, count in grads:
            assert g.is_cuda and g.is_contiguous() and g.dtype in _DTYPES and (count is None or g.dim() == 2)
            assert count is None or _vector(count, 1, torch.int32, "count")
        c = (_CGradTensor * max(len(grads), 1))()
        for t, (g, count) in zip(c, grads):
            t.grad, t.dtype = g.data_ptr(), _DTYPES[g.dtype]
            t.n_rows, t.dim = g.shape if count is not None else (1, g.numel())
            t.n_rows_dev = None if count is None else count.data_ptr()
        self.grads, self._c, self._n = grads, c, len(grads)
        self._bytes = lib().coop_grad_norm_workspace_bytes(c, self._n)
        self._device = grads[0][0].device if grads else torch.device("cuda")

    def measure(self, max_norm=float("inf"), grad_scale=None, workspace=None, stream=None):
        """(norm, factor), fp32 [1] on the device: norm = |s| sqrt(sum of g^2) with s = grad_scale (fp32 [1] on the device; None: 1) and
        factor = s min(1, max_norm / (norm + 1e-6)): AdamW.step's grad_scale, or apply's factor."""
        norm, factor = (_new(1, torch.float32, self._device, stream) for _ in range(2))
        gs = None if grad_scale is None else _vector(grad_scale, 1, torch.float32, "grad_scale")
        keep, wp, wb = _workspace(self._bytes, workspace, self._device, stream)
        _check(lib().coop_grad_norm(self._c, self._n, max_norm, gs, norm.data_ptr(), factor.data_ptr(), wp, wb, _stream_ptr(stream)))
        return norm, factor

    def apply(self, factor, stream=None):
        """The gradients times the factor (fp32 [1] on the device), where they lie."""
        _check(lib().coop_grad_scale(self._c, self._n, _vector(factor, 1, torch.float32, "factor"), _stream_ptr(stream)))
