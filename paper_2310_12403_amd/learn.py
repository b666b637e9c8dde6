"""Operators of learned vertex representations (see include/coop.h for the contract of every call): rows of a table looked
up with a scale and their gradient, layer norm, softmax cross entropy over a large vocabulary, AdamW.

Marshalling only, as in binding.py: the results and the workspaces are torch's, the work is the library's.

stream: a stream to work on in the place of torch's current one.  What is given has to be ready on it and to stay until it is through; what
comes back is ready when it is.
"""
import ctypes as C

import torch

from . import binding
from .binding import COOP_F16, COOP_F32, _check, _dev_ptr, _stream_ptr, _torch_stream

COOP_BF16 = 2
COOP_NO_PAD = -(1 << 31)
ADAMW_BLOCK = 256   # elements of a row that share a scale in an 8-bit moment

_DTYPES = {torch.float32: COOP_F32, torch.float16: COOP_F16, torch.bfloat16: COOP_BF16}


class _CAdamWTensor(C.Structure):
    _fields_ = [("param", C.c_void_p), ("grad", C.c_void_p), ("copy", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p),
                ("m_scale", C.c_void_p), ("v_scale", C.c_void_p), ("rows", C.c_void_p), ("n_list_dev", C.c_void_p),
                ("n_list", C.c_int64), ("n_rows", C.c_int64), ("dim", C.c_int64),
                ("param_dtype", C.c_int32), ("grad_dtype", C.c_int32), ("copy_dtype", C.c_int32), ("reserved", C.c_int32)]


_P, _I, _L, _F, _S = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_size_t
_SIGNATURES = {
    "coop_embed": (C.c_int, [_P, _L, _I, C.c_int, _P, _L, _P, _F, _I, _P, C.c_int, _P]),
    "coop_embed_grad_workspace_bytes": (_S, [_L, _I]),
    "coop_embed_grad": (C.c_int, [_P, C.c_int, _P, _L, _P, _F, _I, _L, _I, _P, C.c_int, _P, _S, _P]),
    "coop_embed_grad_rows": (C.c_int, [_P, C.c_int, _P, _L, _P, _F, _I, _L, _I, _P, _P, C.c_int, _P, _P, _S, _P]),
    "coop_layer_norm": (C.c_int, [_P, _L, _I, C.c_int, _P, _P, C.c_int, _F, _P, _P, _P, _P]),
    "coop_layer_norm_grad_workspace_bytes": (_S, [_L, _I, C.c_int]),
    "coop_layer_norm_grad": (C.c_int, [_P, _P, _L, _I, C.c_int, _P, _P, _P, C.c_int, _P, _P, _P, _P, _S, _P]),
    "coop_softmax_xent_workspace_bytes": (_S, [_L, _L, _I, C.c_int, C.c_int, C.c_int]),
    "coop_softmax_xent": (C.c_int, [_P, _L, _P, _L, _I, C.c_int, _P, _F, _I, _P, _P, _P, _S, _P]),
    "coop_softmax_xent_grad": (C.c_int, [_P, _L, _P, _L, _I, C.c_int, _P, _F, _I, _P, _P, _P, _P, _P, _S, _P]),
    "coop_adamw": (C.c_int, [_P, C.c_int, C.c_int] + [C.c_double] * 5 + [_L, C.c_uint64, _P, _P]),
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


def _matrix(t, what, rows=None, dim=None):
    assert t.is_cuda and t.dim() == 2 and t.is_contiguous() and t.dtype in _DTYPES, "%s: a contiguous 2-d cuda tensor of fp32, fp16 or bf16" % what
    assert (rows is None or t.shape[0] == rows) and (dim is None or t.shape[1] == dim), "%s: shape %s" % (what, tuple(t.shape))
    return t.data_ptr()


def _vector(t, n, dtype, what):
    assert t.is_cuda and t.dim() == 1 and t.is_contiguous() and t.dtype == dtype and t.numel() == n, "%s: a contiguous cuda tensor of %d %s" % (what, n, dtype)
    return t.data_ptr()


# What the calls take from torch is the memory of the stream that they work on: memory of torch's current stream may still be in use there by
# what was queued before the tensor over it went.  Of results torch is told that its current stream uses them too.
def _scratch(shape, dtype, device, stream):
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(_torch_stream(stream)):
        return torch.empty(shape, dtype=dtype, device=device)


def _new(shape, dtype, device, stream):
    t = _scratch(shape, dtype, device, stream)
    if stream is not None:
        t.record_stream(torch.cuda.current_stream(device))
    return t


def _workspace(nbytes, given, device, stream):
    """(tensor to keep until the call is queued, address, bytes): the caller's, or torch's for this call"""
    if given is not None:
        assert given.is_cuda and given.is_contiguous()
        return given, given.data_ptr(), given.numel() * given.element_size()
    if nbytes == 0:
        return None, None, 0
    t = _scratch(nbytes, torch.uint8, device, stream)
    return t, t.data_ptr(), nbytes


def _pad(pad):
    return COOP_NO_PAD if pad is None else int(pad)


def coop_embed(table, ids, scale=None, alpha=1.0, pad=None, dtype=None, out=None, stream=None):
    """out[i, :] = alpha scale[i] table[ids[i], :], as `dtype` (the table's by default); zeros where ids[i] == pad."""
    tp = _matrix(table, "table")
    n, dim = ids.numel(), table.shape[1]
    if out is None:
        out = _new((n, dim), dtype or table.dtype, ids.device, stream)
    op = _matrix(out, "out", n, dim)
    assert dtype is None or out.dtype == dtype
    _check(lib().coop_embed(tp, table.shape[0], dim, _DTYPES[table.dtype], _dev_ptr(ids, torch.int32), n,
                            None if scale is None else _vector(scale, n, torch.float32, "scale"), alpha, _pad(pad), op, _DTYPES[out.dtype],
                            _stream_ptr(stream)))
    return out


def coop_embed_grad(dout, ids, n_rows, scale=None, alpha=1.0, pad=None, dtype=torch.float32, out=None, workspace=None, stream=None):
    """The gradient [n_rows, dim] of coop_embed's table: sums over the places of each id, zeros for the others."""
    n = ids.numel()
    dp = _matrix(dout, "dout", n)
    dim = dout.shape[1]
    if out is None:
        out = _new((n_rows, dim), dtype, dout.device, stream)
    op = _matrix(out, "out", n_rows, dim)
    keep, wp, wb = _workspace(lib().coop_embed_grad_workspace_bytes(n, dim), workspace, dout.device, stream)
    _check(lib().coop_embed_grad(dp, _DTYPES[dout.dtype], _dev_ptr(ids, torch.int32), n,
                                 None if scale is None else _vector(scale, n, torch.float32, "scale"), alpha, _pad(pad), n_rows, dim, op,
                                 _DTYPES[out.dtype], wp, wb, _stream_ptr(stream)))
    return out


def coop_embed_grad_rows(dout, ids, n_rows, scale=None, alpha=1.0, pad=None, dtype=torch.float32, workspace=None, wait=True, stream=None):
    """The same for the touched rows only: (rows int32, ascending; their gradients).  With wait=False nothing waits for their
    number: (rows, gradients, count), where the first count[0] of the min(n, n_rows) rows and gradients are there; AdamW.step
    takes the three as they are."""
    n = ids.numel()
    dp = _matrix(dout, "dout", n)
    dim, most = dout.shape[1], min(n, n_rows)
    rows = _new(most, torch.int32, dout.device, stream)
    grad = _new((most, dim), dtype, dout.device, stream)
    count = _new(1, torch.int32, dout.device, stream)
    _matrix(grad, "gradient")
    keep, wp, wb = _workspace(lib().coop_embed_grad_workspace_bytes(n, dim), workspace, dout.device, stream)
    _check(lib().coop_embed_grad_rows(dp, _DTYPES[dout.dtype], _dev_ptr(ids, torch.int32), n,
                                      None if scale is None else _vector(scale, n, torch.float32, "scale"), alpha, _pad(pad), n_rows, dim,
                                      rows.data_ptr(), grad.data_ptr(), _DTYPES[dtype], count.data_ptr(), wp, wb, _stream_ptr(stream)))
    if not wait:
        return rows, grad, count
    if stream is not None:
        stream.synchronize()
    k = int(count)
    return rows[:k], grad[:k]


def _weight_dtype(x, *weights):
    given = {w.dtype for w in weights if w is not None}
    assert len(given) <= 1 and given <= set(_DTYPES), "weight and bias have one type: fp32, fp16 or bf16"
    return _DTYPES[given.pop()] if given else COOP_F32


def coop_layer_norm(x, weight=None, bias=None, eps=1e-5, out=None, stream=None):
    """(y, mean, rstd) of the rows of x [n, dim]: y = (x - mean) rstd weight + bias."""
    xp = _matrix(x, "x")
    n, dim = x.shape
    if out is None:
        out = _new((n, dim), x.dtype, x.device, stream)
    op = _matrix(out, "out", n, dim)
    assert out.dtype == x.dtype
    mean, rstd = _new(n, torch.float32, x.device, stream), _new(n, torch.float32, x.device, stream)
    _check(lib().coop_layer_norm(xp, n, dim, _DTYPES[x.dtype], None if weight is None else _vector(weight, dim, weight.dtype, "weight"),
                                 None if bias is None else _vector(bias, dim, bias.dtype, "bias"), _weight_dtype(x, weight, bias), eps, op,
                                 mean.data_ptr(), rstd.data_ptr(), _stream_ptr(stream)))
    return out, mean, rstd


def coop_layer_norm_grad(dy, x, mean, rstd, weight=None, want_weight=True, out=None, workspace=None, stream=None):
    """(dx, dweight, dbias) of coop_layer_norm; the last two fp32, None where want_weight is false."""
    xp = _matrix(x, "x")
    n, dim = x.shape
    dp = _matrix(dy, "dy", n, dim)
    assert dy.dtype == x.dtype
    if out is None:
        out = _new((n, dim), x.dtype, x.device, stream)
    op = _matrix(out, "out", n, dim)
    assert out.dtype == x.dtype
    dw = _new(dim, torch.float32, x.device, stream) if want_weight else None
    db = _new(dim, torch.float32, x.device, stream) if want_weight else None
    need = lib().coop_layer_norm_grad_workspace_bytes(n, dim, _DTYPES[x.dtype]) if want_weight else 0
    keep, wp, wb = _workspace(need, workspace, x.device, stream)
    _check(lib().coop_layer_norm_grad(dp, xp, n, dim, _DTYPES[x.dtype], _vector(mean, n, torch.float32, "mean"),
                                      _vector(rstd, n, torch.float32, "rstd"), None if weight is None else _vector(weight, dim, weight.dtype, "weight"),
                                      _weight_dtype(x, weight), op, dw.data_ptr() if want_weight else None,
                                      db.data_ptr() if want_weight else None, wp, wb, _stream_ptr(stream)))
    return out, dw, db


def coop_softmax_xent(hidden, weight, targets, alpha=1.0, ignore=-1, workspace=None, stream=None):
    """(loss, lse), fp32 [n]: cross entropy of softmax(alpha hidden weight^T) against targets (int32; `ignore`: none, loss 0)."""
    hp, wp = _matrix(hidden, "hidden"), _matrix(weight, "weight", dim=hidden.shape[1])
    assert weight.dtype == hidden.dtype
    (n, dim), vocab, dtype = hidden.shape, weight.shape[0], _DTYPES[hidden.dtype]
    assert targets.numel() == n
    loss, lse = _new(n, torch.float32, hidden.device, stream), _new(n, torch.float32, hidden.device, stream)
    keep, sp, sb = _workspace(lib().coop_softmax_xent_workspace_bytes(n, vocab, dim, dtype, (hp | wp) & 15 == 0, 0), workspace, hidden.device, stream)
    _check(lib().coop_softmax_xent(hp, n, wp, vocab, dim, dtype, _dev_ptr(targets, torch.int32), alpha, ignore, loss.data_ptr(), lse.data_ptr(),
                                   sp, sb, _stream_ptr(stream)))
    return loss, lse


def coop_softmax_xent_grad(hidden, weight, targets, lse, dloss, alpha=1.0, ignore=-1, want_hidden=True, want_weight=True, workspace=None,
                           stream=None):
    """(dhidden, dweight) for the gradient dloss (fp32 [n]) of coop_softmax_xent's losses; None for one that is not wanted."""
    hp, wp = _matrix(hidden, "hidden"), _matrix(weight, "weight", dim=hidden.shape[1])
    assert weight.dtype == hidden.dtype
    (n, dim), vocab, dtype = hidden.shape, weight.shape[0], _DTYPES[hidden.dtype]
    assert targets.numel() == n
    dh = _new((n, dim), hidden.dtype, hidden.device, stream) if want_hidden else None
    dw = _new((vocab, dim), weight.dtype, hidden.device, stream) if want_weight else None
    keep, sp, sb = _workspace(lib().coop_softmax_xent_workspace_bytes(n, vocab, dim, dtype, (hp | wp) & 15 == 0, 1), workspace, hidden.device, stream)
    _check(lib().coop_softmax_xent_grad(hp, n, wp, vocab, dim, dtype, _dev_ptr(targets, torch.int32), alpha, ignore,
                                        _vector(lse, n, torch.float32, "lse"), _vector(dloss, n, torch.float32, "dloss"),
                                        dh.data_ptr() if want_hidden else None, dw.data_ptr() if want_weight else None, sp, sb,
                                        _stream_ptr(stream)))
    return dh, dw


class AdamW:
    """AdamW over a list of parameters (coop_adamw), and its moments: in 32 bits, or with bits=8 in 8-bit floats of m and of
    the root of v over fp32 scales.

    grads: the tensors that hold the gradients at every step (set_grads replaces them); None for a parameter whose touched
    rows are given to step.  by_rows (one for all, or one for each parameter): 8-bit moments are scaled within the rows of a
    2-d parameter, which is what lets a step touch some rows only; else the parameter is one row.  copies: tensors that get
    the new parameters as well, rounded to their type.  state: lists "m", "v" (and "m_scale", "v_scale") of existing moments;
    otherwise they begin at zero.

    Every step works on the memory that parameters, copies and moments have when the optimizer is made: new values go there
    by copy_; a tensor put in the place of one of them (p.data = ..., state["m"][0] = ...) is not seen."""

    def __init__(self, params, grads=None, bits=32, by_rows=False, copies=None, state=None):
        assert bits in (8, 32)
        self.params, self.bits = list(params), bits
        n = len(self.params)
        self.by_rows = list(by_rows) if isinstance(by_rows, (list, tuple)) else [by_rows] * n
        self.copies = list(copies) if copies is not None else [None] * n
        assert len(self.by_rows) == n and len(self.copies) == n
        self.shapes = []
        for p, by in zip(self.params, self.by_rows):
            assert p.is_cuda and p.is_contiguous() and p.dtype in _DTYPES and (not by or p.dim() == 2)
            self.shapes.append(tuple(p.shape) if by else (1, p.numel()))
        scales = [rows * -(-dim // ADAMW_BLOCK) for rows, dim in self.shapes]
        kind = torch.float32 if bits == 32 else torch.float8_e4m3fn
        names = ("m", "v") if bits == 32 else ("m", "v", "m_scale", "v_scale")
        if state is None:
            state = {x: [torch.zeros(s if x.endswith("scale") else p.numel(), dtype=torch.float32 if x.endswith("scale") else kind, device=p.device)
                         for p, s in zip(self.params, scales)] for x in names}
        self.state = {x: list(state[x]) for x in names}
        assert all(len(self.state[x]) == n for x in names)
        self._c = (_CAdamWTensor * max(n, 1))()
        for c, p, copy, shape, s, *mine in zip(self._c, self.params, self.copies, self.shapes, scales, *(self.state[x] for x in names)):
            k = p.numel()
            for i, t in enumerate(mine):
                assert t.is_cuda and t.is_contiguous() and t.dtype == (kind if i < 2 else torch.float32) and t.numel() == (k if i < 2 else s), \
                    "%s of a parameter: %d %s" % (names[i], k if i < 2 else s, kind if i < 2 else torch.float32)
            c.param, c.param_dtype, c.n_rows, c.dim = p.data_ptr(), _DTYPES[p.dtype], *shape
            c.m, c.v = mine[0].data_ptr(), mine[1].data_ptr()
            if bits == 8:
                c.m_scale, c.v_scale = mine[2].data_ptr(), mine[3].data_ptr()
            if copy is not None:
                assert copy.is_cuda and copy.is_contiguous() and copy.numel() == k and copy.dtype in _DTYPES
                c.copy, c.copy_dtype = copy.data_ptr(), _DTYPES[copy.dtype]
        # (what the plan's addresses point to stays, whatever becomes of the tensors)
        self._memory = [t.untyped_storage() for ts in (self.params, self.copies, *self.state.values()) for t in ts if t is not None]
        self.set_grads([None] * n if grads is None else grads)

    def set_grads(self, grads):
        grads = tuple(grads)
        assert len(grads) == len(self.params)
        for p, g in zip(self.params, grads):
            assert g is None or g.is_cuda and g.is_contiguous() and g.numel() == p.numel() and g.dtype in _DTYPES
        self.grads = grads  # (none is taken before all are looked at: the ones in the plan are those that are kept)
        for c, g in zip(self._c, grads):
            c.grad, c.grad_dtype = (None, 0) if g is None else (g.data_ptr(), _DTYPES[g.dtype])

    def step(self, step, lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, rows=None, seed=0, grad_scale=None, stream=None):
        """One step; `step` counts from 1.  rows: {parameter's place in the list: (rows, gradients, count or None)}, as
        coop_embed_grad_rows returns them, for parameters of which only these rows change.  grad_scale: fp32 [1] on the device,
        multiplied into every gradient.  Captured into a graph, every replay is this same step again: step, rates and seed are
        the captured ones."""
        rows = rows or {}
        assert all(0 <= i < len(self.params) for i in rows)
        for i, g in enumerate(self.grads):
            assert g is not None or i in rows, "parameter %d has no gradient" % i
        listed = []
        for i, (ids, g, count) in rows.items():  # (all of them are looked at before the plan is changed for the call)
            assert self.by_rows[i] or self.bits == 32 and self.params[i].dim() == 2
            n_rows, dim = self.params[i].shape
            listed.append((self._c[i], dict(
                n_rows=n_rows, dim=dim, grad=_matrix(g, "row gradients", ids.numel(), dim), grad_dtype=_DTYPES[g.dtype],
                rows=_vector(ids, ids.numel(), torch.int32, "rows") or 1, n_list=ids.numel(),  # (an empty list has no address)
                n_list_dev=None if count is None else _vector(count, 1, torch.int32, "count"))))
        gs = None if grad_scale is None else _vector(grad_scale, 1, torch.float32, "grad_scale")
        try:
            for c, fields in listed:
                for name, value in fields.items():
                    setattr(c, name, value)
            _check(lib().coop_adamw(self._c, len(self.params), self.bits, lr, beta1, beta2, eps, weight_decay, step, seed, gs, _stream_ptr(stream)))
        finally:
            for i in rows:
                c, g = self._c[i], self.grads[i]
                c.rows = c.n_list_dev = None
                c.n_list, (c.n_rows, c.dim) = 0, self.shapes[i]
                c.grad, c.grad_dtype = (None, 0) if g is None else (g.data_ptr(), _DTYPES[g.dtype])
