"""Layers on learned vertex rows (see include/coop.h for the contract of every call): a dense layer with its epilogue, the projections of
a gated feed-forward block, the norms and the residual between two blocks, and the gradients' norm ahead of an AdamW step.

Marshalling only, as in binding.py and learn.py; streams are as there.
"""
import ctypes as C

import torch

from . import binding, learn
from .binding import _check, _stream_ptr
from .learn import _DTYPES, _matrix, _new, _vector, _workspace

COOP_ACT_NONE, COOP_ACT_RELU, COOP_ACT_GELU, COOP_ACT_SILU = 0, 1, 2, 3

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


def _same(t, like, what, rows=None, dim=None):
    p = _matrix(t, what, rows, dim)
    assert t.dtype == like.dtype, "%s: %s" % (what, like.dtype)
    return p


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
        out = _new((n, m), x.dtype, x.device, stream)
    op = _same(out, x, "out", n, m)
    pre = _new((n, m), torch.float32, x.device, stream) if want_pre else None
    rp = None if residual is None else _same(residual, x, "residual", n, m)
    keep, sp, sb = _workspace(lib().coop_linear_workspace_bytes(n, k, m, dtype, (xp | wp) & 15 == 0), workspace, x.device, stream)
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
    dx = _new((n, k), x.dtype, x.device, stream) if want_x else None
    dw = _new((m, k), grad_dtype, x.device, stream) if want_weight else None
    db = _new(m, torch.float32, x.device, stream) if want_bias else None
    need = lib().coop_linear_grad_workspace_bytes(n, k, m, dtype, act, pre is not None, (xp | wp | dp) & 15 == 0)
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
        out = _new((n, f), x.dtype, x.device, stream)
    op = _same(out, x, "out", n, f)
    pre = _new((2, n, f), torch.float32, x.device, stream) if want_pre else None
    keep, sp, sb = _workspace(lib().coop_gated_workspace_bytes(n, k, f, dtype, (xp | gp | upp) & 15 == 0), workspace, x.device, stream)
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
    dx = _new((n, k), x.dtype, x.device, stream) if want_x else None
    dw = [_new((f, k), grad_dtype, x.device, stream) for _ in range(2)] if want_weight else [None] * 2
    db = [_new(f, torch.float32, x.device, stream) for _ in range(2)] if want_bias else [None] * 2
    need = lib().coop_gated_grad_workspace_bytes(n, k, f, dtype, pre is not None, (xp | gp | upp) & 15 == 0)
    keep, sp, sb = _workspace(need, workspace, x.device, stream)
    _check(lib().coop_gated_grad(dp, xp, n, k, gp, upp, f, dtype, _bias(gate_bias, f, x, "gate_bias"), _bias(up_bias, f, x, "up_bias"), act,
                                 _kept(pre, (2, n, f)), dx.data_ptr() if want_x else None, *(w.data_ptr() if want_weight else None for w in dw),
                                 _DTYPES[grad_dtype], *(b.data_ptr() if want_bias else None for b in db), sp, sb, _stream_ptr(stream)))
    return (dx, *dw, *db)
