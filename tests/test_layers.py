"""The layers on learned rows against plain implementations in 64 bits: at the sizes, types and values where they can go wrong; gradients
against the formulas and against differences; refusals.

Tolerances are bounds, elementwise, as in test_learn.py: u = 2^-24 for an operation in 32 bits, the sums' worst order included (twice over
in the matrix units, which need not round every partial sum to nearest), and half a unit in the last place of every type that something is
rounded to."""
import ctypes as C
import math

import pytest
import torch

import paper_2310_12403_amd as P
from paper_2310_12403_amd import layers

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}
TYPES = [torch.float32, torch.float16, torch.bfloat16]
IDS = ["f32", "f16", "bf16"]
ACTS = [P.COOP_ACT_NONE, P.COOP_ACT_RELU, P.COOP_ACT_GELU, P.COOP_ACT_SILU]
gpu = pytest.mark.gpu


def rng(seed=0):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def unaligned(t):
    """The same values at an address that is no multiple of more than the element's size."""
    flat = torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)[1:]
    flat.copy_(t.reshape(-1))
    return flat.view(t.shape)


def within(got, want, bound, what=""):
    got, want = got.double(), want.double()
    assert got.shape == want.shape, what
    off = (got - want).abs()
    bad = ~(off <= bound) & ~((got == want) | (torch.isnan(got) & torch.isnan(want)))
    assert not bad.any(), "%s: %d of %d, worst %g times its bound" % (what, bad.sum(), bad.numel(), (off / bound)[bad].max())


def rounded(value, bound, dtype):
    """The bound of what is within `bound` of `value`, rounded to the type."""
    return bound + (value.abs() + bound) * HALF[dtype] + TINY[dtype]


# ---- dense layer and gated block ------------------------------------------------------------------------------------------------
def act64(z, act):
    """(act(z), its slope)"""
    if act == P.COOP_ACT_NONE:
        return z, torch.ones_like(z)
    if act == P.COOP_ACT_RELU:
        return z.clamp(min=0), (z > 0).double()
    if act == P.COOP_ACT_GELU:
        p = 0.5 * torch.erfc(z * -math.sqrt(0.5))   # (1 + erf would lose the tail)
        return z * p, p + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    p = torch.sigmoid(z)
    return z * p, p * (1 + z * (1 - p))


def product64(x, w, b):
    """(x w' + b, how far 32 bits may be from it)"""
    x, w = x.double(), w.double()
    z, size = x @ w.t(), x.abs() @ w.abs().t()
    if b is not None:
        z, size = z + b.double(), size + b.double().abs()
    return z, size * (2 * (x.shape[1] + 4) * U)


def act_bound(z, ez, act):
    """How far act(z) and its slope may be, of a z that is off by up to ez.  Slopes are at most 1.13 and change by at most 1 for a step of 1
    (but relu's, anywhere near 0).  The functions themselves: the distribution's tail q is exact to 24 u and 2 z^2 u of the exponential's argument, with
    q <= 1/2 and q z^2 <= 1/5, and 1 - q to one u more; the logistic function to 5 u, z times its slope's share bounded by 1/3."""
    if act == P.COOP_ACT_NONE:
        return ez, torch.zeros_like(z)
    slope = (z.abs() <= ez).double() if act == P.COOP_ACT_RELU else ez + 40 * U
    return 1.2 * ez + 16 * z.abs() * U, slope


def gradients64(dzs, edzs, x, weights, dtype, grad_dtype, rounds):
    """[(dx, bound), (dw, bound).., (db, bound)..] of dz's that are off by up to edz and, where `rounds`, rounded to the type"""
    x, weights = x.double(), [w.double() for w in weights]
    dx = sum(d @ w for d, w in zip(dzs, weights))
    off = [e + (d.abs() + e) * HALF[dtype] + TINY[dtype] if rounds else e for d, e in zip(dzs, edzs)]
    terms = sum(w.shape[0] for w in weights)
    ex = sum(o @ w.abs() + 2 * (terms + 4) * U * ((d.abs() + o) @ w.abs()) for d, o, w in zip(dzs, off, weights))
    out = [(dx, rounded(dx, ex, dtype))]
    for d, o in zip(dzs, off):
        dw = d.t().contiguous() @ x
        out.append((dw, rounded(dw, o.t().contiguous() @ x.abs() + 2 * (x.shape[0] + 4) * U * ((d.abs() + o).t().contiguous() @ x.abs()), grad_dtype)))
    for d, e in zip(dzs, edzs):
        out.append((d.sum(0), e.sum(0) + (x.shape[0] + 8) * U * (d.abs() + e).sum(0)))
    return out


# (one tile, none whole, many rows, many columns, long k, tiles of 256 in each of the products)
SIZES = [(0, 5, 3), (1, 1, 1), (3, 7, 5), (1, 4096, 64), (17, 2000, 300), (33, 64, 128), (130, 100, 75), (257, 129, 300), (300, 602, 41), (1000, 16, 8),
         (20000, 33, 40), (5000, 128, 128), (70000, 128, 64), (2049, 32, 128), (64, 127, 121), (31, 8, 8), (3000, 64, 31), (70001, 24, 20), (4097, 72, 4100), (4097, 4100, 72), (72, 4100, 4104), (1, 2, 9000), (2, 9000, 1)]


@gpu
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("n,k,m", SIZES)
def test_linear(dtype, n, k, m):
    g = rng(n + k + m)
    place = unaligned if (n + k + m) % 2 else (lambda t: t)
    x, w = place(normal(g, n, k, dtype=dtype)), place(normal(g, m, k, dtype=dtype, scale=1.5 / math.sqrt(k)))
    b, res, dy = place(normal(g, m, dtype=dtype, scale=0.3)), place(normal(g, n, m, dtype=dtype)), place(normal(g, n, m, dtype=dtype))
    grad_dtype = torch.float32 if k % 2 else dtype
    for act in ACTS:
        bias, residual, alpha = (b, res, 0.7) if act % 2 else (None, None, 1.0)
        z, ez = product64(x, w, bias)
        a, slope = act64(z, act)
        ea, es = act_bound(z, ez, act)
        out, pre = P.coop_linear(x, w, bias, act=act, alpha=alpha, residual=residual, want_pre=True)
        want = a * alpha + (0 if residual is None else residual.double())
        size = a.abs() * alpha + (0 if residual is None else residual.double().abs())
        within(out, want, rounded(want, ea * alpha + 4 * U * (size + ea), dtype), "out")
        within(pre, z, ez + TINY[torch.float32], "pre")
        assert torch.equal(out, P.coop_linear(x, w, bias, act=act, alpha=alpha, residual=residual))
        d = dy.double() * alpha
        dz, edz = d * slope, d.abs() * (es + 4 * U * (slope.abs() + es))
        if act == P.COOP_ACT_NONE:
            edz = edz * 0
        wants = gradients64([dz], [edz], x, [w], dtype, grad_dtype, act != P.COOP_ACT_NONE)
        for kept in (pre, None):
            got = P.coop_linear_grad(dy, x, w, bias, pre=kept, act=act, alpha=alpha, grad_dtype=grad_dtype)
            for name, have, (value, bound) in zip(("dx", "dw", "db"), got, wants):
                within(have, value, bound + 4 * U * value.abs(), "%s, act %d, kept %s" % (name, act, kept is not None))


@gpu
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("n,k,f", SIZES)
def test_gated(dtype, n, k, f):
    g = rng(n + k + f + 1)
    place = unaligned if (n + k + f) % 2 else (lambda t: t)
    x = place(normal(g, n, k, dtype=dtype))
    wg, wu = (place(normal(g, f, k, dtype=dtype, scale=1.5 / math.sqrt(k))) for _ in range(2))
    bg, bu, dy = place(normal(g, f, dtype=dtype, scale=0.3)), place(normal(g, f, dtype=dtype, scale=0.3)), place(normal(g, n, f, dtype=dtype))
    grad_dtype = torch.float32 if k % 2 else dtype
    for act, biases in ((P.COOP_ACT_SILU, (None, None)), (P.COOP_ACT_GELU, (bg, bu)), (P.COOP_ACT_RELU, (bg, None)), (P.COOP_ACT_NONE, (None, bu))):
        (zg, eg), (zu, eu) = product64(x, wg, biases[0]), product64(x, wu, biases[1])
        a, slope = act64(zg, act)
        ea, es = act_bound(zg, eg, act)
        want = a * zu
        bound = ea * (zu.abs() + eu) + a.abs() * eu + 4 * U * (a.abs() + ea) * (zu.abs() + eu)
        out, pre = P.coop_gated(x, wg, wu, *biases, act=act, want_pre=True)
        within(out, want, rounded(want, bound, dtype), "out")
        within(pre, torch.stack([zg, zu]), torch.stack([eg, eu]) + TINY[torch.float32], "pre")
        assert torch.equal(out, P.coop_gated(x, wg, wu, *biases, act=act))
        d = dy.double()
        dg, edg = d * zu * slope, d.abs() * ((zu.abs() + eu) * (es + 4 * U * (slope.abs() + es)) + eu * slope.abs())
        du, edu = d * a, d.abs() * (ea + 4 * U * (a.abs() + ea))
        wants = gradients64([dg, du], [edg, edu], x, [wg, wu], dtype, grad_dtype, True)
        for kept in (pre, None):
            got = P.coop_gated_grad(dy, x, wg, wu, *biases, pre=kept, act=act, grad_dtype=grad_dtype)
            for name, have, (value, bound) in zip(("dx", "dgate", "dup", "dgate_bias", "dup_bias"), got, wants):
                within(have, value, bound + 4 * U * value.abs(), "%s, act %d, kept %s" % (name, act, kept is not None))


@gpu
@pytest.mark.parametrize("act", ACTS)
def test_activations_over_their_range(act):
    """The functions alone, through a product with 1: tails to their own size (gelu's as exact as the exponential's argument), infinities, NaN."""
    z = torch.cat([torch.linspace(-14, 14, 20001), torch.tensor([0.0, -0.0, 1e-30, -1e-30, 100.0, -100.0, 1e30, float("inf"), float("nan")])]).cuda()[:, None]
    one = torch.ones((1, 1), device="cuda")
    out, pre = P.coop_linear(z, one, act=act, want_pre=True)
    want, slope = act64(z.double(), act)
    assert torch.equal(pre, z) or torch.equal(pre[:-1], z[:-1])
    relative = {P.COOP_ACT_NONE: 0, P.COOP_ACT_RELU: 0, P.COOP_ACT_GELU: 30 + 2 * z.double() ** 2, P.COOP_ACT_SILU: 8 + 3 * z.double().abs()}[act]
    # (below 2^-126 the exponential is rounded to zero)
    within(out[:-1], want[:-1], (relative * U * want.abs() + 2.0 ** -120)[:-1] if act >= 2 else TINY[torch.float32])
    assert math.isnan(out[-1])
    dx = P.coop_linear_grad(torch.ones_like(z), z, one, act=act)[0]
    finite = slice(0, -2)
    within(dx[finite], slope[finite], 40 * U)
    assert math.isnan(dx[-1]) == (act != P.COOP_ACT_NONE)


# ---- the seam between two blocks -------------------------------------------------------------------------------------------------
class Norm64:
    """A norm of the rows of v, which is known to `ev`, and how far 32 bits may be from what follows."""

    def __init__(self, v, ev, w, b, rms, eps):
        n = v.shape[1]
        self.rms, self.n = rms, n
        one = torch.ones(n, dtype=torch.float64, device=v.device)
        self.w, self.b = one if w is None else w.double(), 0 * one if b is None else b.double()
        size = v.abs().mean(1, keepdim=True)
        mean = 0 * size if rms else v.mean(1, keepdim=True)
        emean = 0 * size if rms else ev.mean(1, keepdim=True) + (n + 2) * U * (size + ev.mean(1, keepdim=True))
        c = v - mean
        ec = ev + emean + U * (c.abs() + ev + emean)
        var = (c * c).mean(1, keepdim=True)
        evar = (2 * c.abs() * ec + ec * ec).mean(1, keepdim=True) + (n + 4) * U * ((c.abs() + ec) ** 2).mean(1, keepdim=True)
        self.rstd = 1 / (var + eps).sqrt()
        # (1 / sqrt falls by at most this from what is `evar` lower, or eps)
        low = (var - evar).clamp(min=0) + eps
        self.erstd = (1 / low.sqrt() - 1 / (var + evar + eps).sqrt()) + 6 * U / low.sqrt()
        self.h = c * self.rstd
        self.eh = ec * (self.rstd + self.erstd) + c.abs() * self.erstd + 2 * U * (c.abs() + ec) * (self.rstd + self.erstd)
        self.y = self.h * self.w + self.b
        self.ey = self.eh * self.w.abs() + 4 * U * ((self.h.abs() + self.eh) * self.w.abs() + self.b.abs())
        self.mean, self.emean = mean, emean

    def back(self, d, ed):
        """(gradient through the norm, how far 32 bits may be), for d that is known to ed"""
        n, dw, edw = self.n, d * self.w, (ed + 2 * U * (d.abs() + ed)) * self.w.abs()
        top = dw.abs() + edw
        s1 = 0 if self.rms else dw.mean(1, keepdim=True)
        es1 = 0 if self.rms else edw.mean(1, keepdim=True) + (n + 2) * U * top.mean(1, keepdim=True)
        s2 = (dw * self.h).mean(1, keepdim=True)
        es2 = (edw * (self.h.abs() + self.eh) + dw.abs() * self.eh).mean(1, keepdim=True) + (n + 4) * U * (top * (self.h.abs() + self.eh)).mean(1, keepdim=True)
        inner = dw - s1 - self.h * s2
        einner = edw + es1 + self.eh * (s2.abs() + es2) + self.h.abs() * es2
        einner = einner + 4 * U * (top + (self.h.abs() + self.eh) * (s2.abs() + es2) + (0 if self.rms else s1.abs() + es1))
        return inner * self.rstd, einner * (self.rstd + self.erstd) + inner.abs() * self.erstd + U * (inner.abs() + einner) * self.rstd


SEAM_SIZES = [(0, 8), (1, 1), (3, 2), (5, 7), (1, 8), (65, 9), (700, 75), (33, 100), (257, 128), (3000, 96), (129, 511), (40, 513), (19, 1024), (21, 1031), (9, 2050),
              (300, 4096), (11, 5000), (5, 8191)]


@gpu
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("n,dim", SEAM_SIZES + [(3, 16384), (2, 9001)])
def test_residual_norm(dtype, n, dim):
    if dtype == torch.float32 and dim > 8192:
        dim //= 2
    g = rng(n + dim)
    eps = 1e-3
    for i, (norms, rms, gated) in enumerate([("both", False, "columns"), ("both", True, "rows"), ("after", False, "rows"), ("before", False, "columns"),
                                             ("both", False, None), ("after", True, "columns"), ("before", True, "rows")]):
        after, before = norms != "before", norms != "after"
        stream, wt = (torch.float32, dtype)[(i + n) % 2], (torch.float32, dtype)[(i // 2 + dim) % 2]
        place = unaligned if (i + dim) % 2 else (lambda t: t)
        x, f = place(normal(g, n, dim, dtype=stream)), place((normal(g, n, dim) + normal(g, n, 1)).to(dtype))
        gate = None if gated is None else place((0.5 + normal(g, *((dim,) if gated == "columns" else (n, dim)), scale=0.3)).to(wt if gated == "columns" else dtype))
        w1, w2 = (place((1 + normal(g, dim, scale=0.3)).to(wt)) if there and i != 4 else None for there in (after, before))
        b1, b2 = (place(normal(g, dim, scale=0.3).to(wt)) if there and not rms and i != 4 else None for there in (after, before))
        dr, dy = place(normal(g, n, dim, dtype=stream)) if i != 4 else None, place(normal(g, n, dim, dtype=dtype))
        alpha = 0.9 if i % 2 else 1.0
        kw = dict(gate=gate, alpha=alpha, after=after, after_weight=w1, after_bias=b1, before=before, before_weight=w2, rms=rms)
        r, y, stats = P.coop_residual_norm(x, f, before_bias=b2, eps=eps, **kw)
        # forward
        zero = torch.zeros((n, dim), dtype=torch.float64, device="cuda")
        N1 = Norm64(f.double(), zero, w1, b1, rms, eps) if after else None
        p, ep = (N1.y, N1.ey) if after else (f.double(), zero)
        gg = torch.ones(dim, dtype=torch.float64, device="cuda") if gate is None else gate.double()
        r64 = alpha * x.double() + gg * p
        er = gg.abs() * ep + 4 * U * (alpha * x.double().abs() + gg.abs() * (p.abs() + ep))
        within(r, r64, rounded(r64, er, stream), "r")
        N2 = Norm64(r64, er, w2, b2, rms, eps) if before else None
        if before:
            within(y, N2.y, rounded(N2.y, N2.ey, dtype), "y")
        else:
            assert y is None
        for k, N in ((0, N1), (2, N2)):
            if N is not None:
                within(stats[k], N.mean[:, 0], N.emean[:, 0], "mean")
                within(stats[k + 1], N.rstd[:, 0], N.erstd[:, 0], "rstd")
        # backward
        dx, df, dgate, dw1, db1, dw2, db2 = P.coop_residual_norm_grad(dr, dy if before else None, x, f, stats, **kw)
        d, ed = (zero if dr is None else dr.double()), zero
        if before:
            back, eback = N2.back(dy.double(), zero)
            d, ed = d + back, eback
            ed = ed + U * (d.abs() + ed + (0 if dr is None else dr.double().abs()))
        e, ee = d * gg, ed * gg.abs() + U * (d.abs() + ed) * gg.abs()
        within(dx, alpha * d, rounded(alpha * d, alpha * ed + U * (d.abs() + ed), stream), "dx")
        want, bound = N1.back(e, ee) if after else (e, ee)
        within(df, want, rounded(want, bound, dtype), "df")

        def sums(a, ea, b, eb, factor):     # of a b over the rows, times a factor of the column
            terms, off = (a.abs() + ea) * (b.abs() + eb), ea * (b.abs() + eb) + a.abs() * eb
            return (a * b).sum(0) * factor, (off.sum(0) + (n + 8) * U * terms.sum(0)) * abs(factor)

        one = torch.ones_like(zero)
        if gated == "rows":
            assert dgate.dtype == dtype
            within(dgate, d * p, rounded(d * p, ed * (p.abs() + ep) + d.abs() * ep + U * (d.abs() + ed) * (p.abs() + ep), dtype), "dgate")
        elif gated == "columns":
            if after:
                (s1, e1), (s0, e0) = sums(d, ed, N1.h, N1.eh, N1.w), sums(d, ed, one, 0 * one, N1.b)
                within(dgate, s1 + s0, e1 + e0 + 4 * U * (s1.abs() + s0.abs()), "dgate")
            else:
                within(dgate, *sums(d, ed, p, ep, 1.0), "dgate")
        else:
            assert dgate is None
        if after:
            per = gated == "rows"
            within(dw1, *sums(e if per else d, ee if per else ed, N1.h, N1.eh, 1.0 if per else gg), "dw1")
            if not rms:
                within(db1, *sums(e if per else d, ee if per else ed, one, 0 * one, 1.0 if per else gg), "db1")
        if before:
            within(dw2, *sums(dy.double(), zero, N2.h, N2.eh, 1.0), "dw2")
            if not rms:
                within(db2, *sums(dy.double(), zero, one, 0 * one, 1.0), "db2")
        assert (dw1 is None) == (not after) and (dw2 is None) == (not before) and (db1 is None) == (rms or not after) and (db2 is None) == (rms or not before)


# ---- the gradients' norm ------------------------------------------------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("sizes", [[1], [0], [], [7, 0, 16384, 16385, 3], [1000003], [5] * 1000, [40000, 1, 2, 300000]])
def test_grad_norm(sizes):
    g = rng(len(sizes))
    grads = [unaligned(normal(g, k, dtype=TYPES[i % 3], scale=10.0 ** (i % 5 - 2))) for i, k in enumerate(sizes)]
    plan = P.GradNorm(grads)
    want = math.sqrt(sum(float((x.double() ** 2).sum()) for x in grads))
    for scale in (None, torch.tensor([-0.25], device="cuda")):
        s = 1.0 if scale is None else -0.25
        for bound in (float("inf"), want * 0.1, 0.0):
            norm, factor = plan.measure(bound, grad_scale=scale)
            f = s * min(1.0, bound / (abs(s) * want + 1e-6))
            # (64 bits throughout: what is off is the rounding of the result)
            assert abs(float(norm) - abs(s) * want) <= 2 * U * abs(s) * want and abs(float(factor) - f) <= 2 * U * abs(f)
    norm, factor = plan.measure(want * 0.5)
    before = [x.clone() for x in grads]
    plan.apply(factor)
    for x, b in zip(grads, before):
        assert torch.equal(x, (b.float() * factor).to(b.dtype))
    plan.apply(torch.ones(1, device="cuda"))
    for x, b in zip(grads, before):
        assert torch.equal(x, (b.float() * factor).to(b.dtype))


@gpu
def test_grad_norm_of_extremes_and_of_what_is_not_finite():
    for dtype, value in ((torch.float32, 3e38), (torch.float32, 1e-45), (torch.bfloat16, 3e38), (torch.bfloat16, 1e-40), (torch.float16, 65504.0), (torch.float16, 6e-8)):
        x = torch.full((9,), value, device="cuda").to(dtype)
        norm, factor = P.GradNorm([x]).measure(1.0)
        want = 3 * float(x[0])
        assert (math.isinf(float(norm)) if want > 3.4028236e38 else abs(float(norm) - want) <= 2 * U * want + 2.0 ** -150), (dtype, value)
        assert abs(float(factor) - min(1.0, 1 / (want + 1e-6))) <= 2 * U + 2.0 ** -149
    x = torch.ones(100, device="cuda")
    x[57] = float("inf")
    norm, factor = P.GradNorm([torch.ones(3, device="cuda"), x]).measure(1.0)
    assert math.isinf(float(norm)) and float(factor) == 0.0
    x[3] = float("nan")
    norm, factor = P.GradNorm([x]).measure(1.0)
    assert math.isnan(float(norm)) and math.isnan(float(factor))


@gpu
def test_grad_norm_of_touched_rows_and_the_step_that_it_scales():
    """The rows that coop_embed_grad_rows gives, without waiting for their number: what lies behind them does not count and stays."""
    g = rng(5)
    ids = torch.randint(0, 40, (300,), generator=g, device="cuda", dtype=torch.int32)
    dout, dense = normal(g, 300, 75), normal(g, 33, dtype=torch.bfloat16)
    rows, grad, count = P.coop_embed_grad_rows(dout, ids, 50, wait=False)
    k = int(count)
    grad[k:] = 1e9
    plan = P.GradNorm([(grad, count), dense])
    norm, factor = plan.measure(1.0)
    want = math.sqrt(float((grad[:k].double() ** 2).sum() + (dense.double() ** 2).sum()))
    assert abs(float(norm) - want) <= 2 * U * want
    tables = [normal(rng(6), 50, 75) for _ in range(2)]
    opts = [P.AdamW([t], by_rows=True) for t in tables]
    opts[0].step(1, 1e-2, rows={0: (rows, grad, count)}, grad_scale=factor)
    plan.apply(factor)
    assert float(grad[k:].min()) == float(torch.tensor(1e9)) and abs(float(P.GradNorm([(grad, count), dense]).measure()[0]) - 1.0) < 1e-2
    opts[1].step(1, 1e-2, rows={0: (rows, grad, count)})
    assert torch.equal(tables[0], tables[1])
