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


# (one tile, none whole, many rows, many columns, long k, tiles of 64, 128 and 256 in each of the products, with k in parts and whole)
SIZES = [(0, 5, 3), (1, 1, 1), (3, 7, 5), (1, 4096, 64), (17, 2000, 300), (33, 64, 128), (130, 100, 75), (257, 129, 300), (300, 602, 41), (1000, 16, 8),
         (20000, 33, 40), (5000, 128, 128), (70000, 128, 64), (2049, 32, 128), (64, 127, 121), (31, 8, 8), (3000, 64, 31), (70001, 24, 20), (4097, 72, 4100), (4097, 4100, 72), (72, 4100, 4104), (1, 2, 9000), (2, 9000, 1), (33000, 1024, 2048)]


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


# ---- what dz loses to a type of 16 bits --------------------------------------------------------------------------------------------
# Where dz has up to 2^16 values, or a result (dx, or one weight's gradient) up to 2^12, dz is multiplied as the sum of two numbers of the type, whichever
# kernels do it: (n, k, m) of the small ones, of products in tiles with k whole and in parts, of the narrow ones, whole and ragged, and of few rows of
# wide layers, on both sides of what those kernels are chosen by.
KEPT_REST = [(1, 1, 1), (3, 7, 5), (15, 16, 17), (33, 31, 64), (1, 1024, 2048), (300, 64, 200), (1, 1024, 3080), (1, 64, 3100), (1, 4096, 520), (2, 2000, 6000), (20, 17, 3200),
             (24, 1030, 2000), (3100, 1, 20), (3080, 16, 16), (6000, 1024, 3), (20000, 300, 9), (70001, 24, 20), (20000, 33, 40), (5000, 64, 64), (4100, 128, 32), (4100, 128, 16),
             (9000, 100, 40), (9000, 32, 128), (5000, 30, 120), (5000, 40, 100), (20000, 128, 7), (3100, 1, 1024), (70000, 4, 600)]


def keeps_rest(n, k, m, both):
    return n * both <= 1 << 16 or min(n, m) * k <= 1 << 12


def nearly_rounded_once(got, want, dtype, what):
    """The results' distance from 64 bits is what rounding them to the type makes, and a tenth more; of results in 32 bits, a 16th of half a unit of dz's type.
    (In two parts a dz is off by HALF^2 of itself and by 32 bits' own, z's among them: some 64 u, 2^-18.  A result whose terms' signs are random is off by as
    much of itself, and is rounded to another number than 64 bits' only where it lies that near to the middle of two.  One rounding of dz alone makes 0.4 HALF.)"""
    off, want = float((got.double() - want).norm()), want.double()
    if got.dtype == torch.float32:
        assert off <= HALF[dtype] / 16 * float(want.norm()), "%s: %g of the most" % (what, off / (HALF[dtype] / 16 * float(want.norm())))
    else:
        once = float((want.to(dtype).double() - want).norm())
        assert off <= 1.1 * once + 2.0 ** -18 * float(want.norm()) + TINY[dtype], "%s: %g times one rounding" % (what, off / max(once, 1e-300))


@gpu
@pytest.mark.parametrize("dtype", TYPES[1:], ids=IDS[1:])
@pytest.mark.parametrize("n,k,m", KEPT_REST)
def test_few_values_or_results_keep_what_dz_loses(dtype, n, k, m):
    assert keeps_rest(n, k, m, m)
    for place in (lambda t: t, unaligned):
        g = rng(n + 3 * k + m)
        x, dy = place(normal(g, n, k, dtype=dtype)), place(normal(g, n, m, dtype=dtype))
        w, w2 = (place(normal(g, m, k, dtype=dtype, scale=1 / math.sqrt(k))) for _ in range(2))
        b = place(normal(g, m, dtype=dtype, scale=0.3))
        for act in (P.COOP_ACT_GELU, P.COOP_ACT_SILU):
            z, ez = product64(x, w, b)
            dz = dy.double() * act64(z, act)[1]
            dx, dw = dz @ w.double(), dz.t().contiguous() @ x.double()
            _, pre = P.coop_linear(x, w, b, act=act, want_pre=True)
            for kept in (pre, None):
                for grad_dtype in (dtype, torch.float32):
                    got = P.coop_linear_grad(dy, x, w, b, pre=kept, act=act, grad_dtype=grad_dtype)
                    for name, have, want in zip(("dx", "dw"), got, (dx, dw)):
                        nearly_rounded_once(have, want, dtype, "%s, act %d, kept %s" % (name, act, kept is not None))
        if not keeps_rest(n, k, m, 2 * m):
            continue
        (zg, _), (zu, _) = product64(x, w, b), product64(x, w2, None)
        a, slope = act64(zg, P.COOP_ACT_SILU)
        dg, du = dy.double() * zu * slope, dy.double() * a
        wants = dg @ w.double() + du @ w2.double(), dg.t().contiguous() @ x.double(), du.t().contiguous() @ x.double()
        _, pre = P.coop_gated(x, w, w2, b, None, want_pre=True)
        for kept in (pre, None):
            for grad_dtype in (dtype, torch.float32):
                got = P.coop_gated_grad(dy, x, w, w2, b, None, pre=kept, grad_dtype=grad_dtype)
                for name, have, want in zip(("dx", "dgate", "dup"), got, wants):
                    nearly_rounded_once(have, want, dtype, "gated %s, kept %s" % (name, kept is not None))


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


@gpu
@pytest.mark.parametrize("dim", [512, 1024, 1500, 2048, 4060, 4096])
@pytest.mark.parametrize("wt", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_residual_norm_of_more_rows_than_are_on_the_chip_at_once(dim, wt):
    """With all weights and biases, which take the most of LDS: the same as the rows a few at a time, bit for bit."""
    g = rng(dim)
    n = 5000
    x, f = normal(g, n, dim, dtype=torch.bfloat16), normal(g, n, dim, dtype=torch.bfloat16)
    w = [normal(g, dim, dtype=wt) for _ in range(5)]
    kw = dict(gate=w[0], after_weight=w[1], after_bias=w[2], before_weight=w[3], before_bias=w[4])
    r, y, stats = P.coop_residual_norm(x, f, **kw)
    for at in (0, 1777, n - 100):
        part = slice(at, at + 100)
        some = P.coop_residual_norm(x[part], f[part], **kw)
        assert torch.equal(r[part], some[0]) and torch.equal(y[part], some[1]) and torch.equal(stats[:, part], some[2])


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
@pytest.mark.parametrize("bound", [0.0, 1.0, 1e30, float("inf")])
def test_grad_norm_that_is_not_finite_by_any_bound(bound):
    """The factor of an infinite norm is 0 and of what is no number none, by a bound of infinity as by any other."""
    x = torch.ones(100, device="cuda", dtype=torch.bfloat16)
    x[57] = -float("inf")
    scale = torch.tensor([-2.0], device="cuda")
    for s in (None, scale):
        norm, factor = P.GradNorm([torch.ones(3, device="cuda"), x]).measure(bound, grad_scale=s)
        assert float(norm) == float("inf") and float(factor) == 0.0
    x[3] = float("nan")
    norm, factor = P.GradNorm([x]).measure(bound)
    assert math.isnan(float(norm)) and math.isnan(float(factor))
    x[:] = 3e38     # (a norm beyond 32 bits of gradients that are finite)
    norm, factor = P.GradNorm([x]).measure(bound)
    want = float(x[0].double()) * 10
    assert float(norm) == float("inf") and abs(float(factor) - min(1.0, bound / want)) <= 2 * U * min(1.0, bound / want) + 2.0 ** -149


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


# ---- every path of them: streams, graphs, workspaces, memory, rows by themselves -------------------------------------------------------
# (small, few rows; narrow, whole and ragged; tiles of 64, of 128 with k split, of 256)
PATHS = [(torch.bfloat16, 24, 64, 96), (torch.float32, 500, 70, 33), (torch.bfloat16, 40000, 128, 64), (torch.float16, 40000, 100, 77), (torch.float32, 4000, 72, 80),
         (torch.float16, 3500, 300, 520), (torch.bfloat16, 4100, 520, 4100), (torch.float32, 7, 3000, 40)]


def dense_calls(dtype, n, k, m, seed=0):
    """The calls' arguments, and f(stream, workspace of bytes) that makes all of them"""
    g = rng(seed + n)
    x, w, w2 = normal(g, n, k, dtype=dtype), normal(g, m, k, dtype=dtype, scale=k ** -0.5), normal(g, m, k, dtype=dtype, scale=k ** -0.5)
    b, res, dy = normal(g, m, dtype=dtype), normal(g, n, m, dtype=dtype), normal(g, n, m, dtype=dtype)

    def everything(stream=None, ws=lambda need: None):
        L, t, al = layers.lib(), layers._DTYPES[dtype], int(all(v.data_ptr() % 16 == 0 for v in (x, w, w2, dy)))
        need = [L.coop_linear_workspace_bytes(n, k, m, t, al), L.coop_gated_workspace_bytes(n, k, m, t, al)]
        out, pre = P.coop_linear(x, w, b, act=P.COOP_ACT_GELU, residual=res, want_pre=True, workspace=ws(need[0]), stream=stream)
        h, pre2 = P.coop_gated(x, w, w2, b, None, want_pre=True, workspace=ws(need[1]), stream=stream)
        got = [out, pre, h, pre2]
        for act, kept in ((P.COOP_ACT_GELU, pre), (P.COOP_ACT_GELU, None), (P.COOP_ACT_NONE, None)):
            need = L.coop_linear_grad_workspace_bytes(n, k, m, t, act, kept is not None, al)
            got += P.coop_linear_grad(dy, x, w, b, pre=kept, act=act, alpha=0.5, workspace=ws(need), stream=stream)
        for kept in (pre2, None):
            need = L.coop_gated_grad_workspace_bytes(n, k, m, t, kept is not None, al)
            got += P.coop_gated_grad(dy, x, w, w2, b, None, pre=kept, workspace=ws(need), stream=stream)
        return got

    return (x, w, w2, b, res, dy), everything


def seam_calls(dtype, n, dim, seed=0):
    g = rng(seed + dim)
    x, f, gate, dr, dy = normal(g, n, dim), normal(g, n, dim, dtype=dtype), normal(g, n, dim, dtype=dtype), normal(g, n, dim), normal(g, n, dim, dtype=dtype)
    w = [normal(g, dim) for _ in range(5)]

    def everything(stream=None, ws=lambda need: None):
        got = []
        for gt, kw in ((gate, {}), (w[4], {}), (None, dict(before=False)), (w[4], dict(after=False))):
            a = dict(after_weight=w[0], after_bias=w[1]) if kw.get("after", True) else {}
            b = dict(before_weight=w[2]) if kw.get("before", True) else {}
            r, y, stats = P.coop_residual_norm(x, f, gate=gt, before_bias=w[3] if b else None, stream=stream, **kw, **a, **b)
            need = layers.lib().coop_residual_norm_grad_workspace_bytes(n, dim, layers._DTYPES[dtype])
            got += [r, y, stats, *P.coop_residual_norm_grad(dr, dy if b else None, x, f, stats, gate=gt, workspace=ws(need), stream=stream, **kw, **a, **b)]
        return [v for v in got if v is not None]

    return (x, f, gate, dr, dy), everything


def clip_calls(seed=0):
    g = rng(seed)
    grads = [normal(g, k, dtype=TYPES[i % 3]) for i, k in enumerate((5, 16384, 70001, 300))]
    plan = P.GradNorm(grads)

    def everything(stream=None, ws=lambda need: None):
        return list(plan.measure(1.0, workspace=ws(plan._bytes), stream=stream))

    return tuple(grads), everything


CALLS = [lambda p=p: dense_calls(*p) for p in PATHS] + [lambda p=p: seam_calls(*p) for p in ((torch.bfloat16, 900, 100), (torch.float16, 300, 2050), (torch.float32, 70, 1000),
                                                                                             (torch.bfloat16, 30, 9000), (torch.bfloat16, 600, 4096))] + [clip_calls]
CALL_IDS = ["%s-%d-%d-%d" % ((str(p[0])[6:],) + p[1:]) for p in PATHS] + ["seam-100", "seam-2050", "seam-1000", "seam-9000", "seam-4096", "clip"]


def same(a, b):
    return len(a) == len(b) and all(x is y or torch.equal(x, y) for x, y in zip(a, b))


@gpu
@pytest.mark.parametrize("calls", CALLS, ids=CALL_IDS)
def test_same_bits_on_another_stream_with_any_workspace_and_in_a_graph(calls):
    inputs, everything = calls()
    kept = [v.clone() for v in inputs]
    want = everything()
    assert same(inputs, kept)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = everything(stream=side)
    assert same(want, everything())            # (beside the other stream's)
    side.synchronize()
    assert same(want, got)
    # (a workspace holds what it comes with, and not a byte behind it is written)
    kept_ws = []

    def given(need):
        ws = torch.full((need + 4096,), 0xFF, dtype=torch.uint8, device="cuda")
        kept_ws.append((ws, need))
        return ws[:need] if need else None

    assert same(want, everything(ws=given))
    assert all((ws[need:] == 0xFF).all() for ws, need in kept_ws)
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = everything()
    for i in range(3):
        for v in out:
            if v is not None:
                v.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert same(want, out), i
        assert same(want, everything())
        torch.ones(1 << 20, device="cuda").sum()
    # other inputs in the same places
    for v in inputs:
        v.mul_(0.5)
    graph.replay()
    torch.cuda.synchronize()
    assert same(everything(), out)


@gpu
@pytest.mark.parametrize("path", PATHS, ids=CALL_IDS[:len(PATHS)])
def test_what_is_asked_for_alone_is_the_same(path):
    """Each gradient by itself, and results at an address of their own with nothing written around them."""
    (x, w, w2, b, res, dy), _ = dense_calls(*path, seed=3)
    dtype, n, k, m = path
    for act in (P.COOP_ACT_NONE, P.COOP_ACT_SILU):
        want = P.coop_linear_grad(dy, x, w, b, act=act)
        for i, names in enumerate(("want_x", "want_weight", "want_bias")):
            only = dict(want_x=False, want_weight=False, want_bias=False)
            only[names] = True
            got = P.coop_linear_grad(dy, x, w, b, act=act, **only)
            assert torch.equal(got[i], want[i]) and sum(v is not None for v in got) == 1
    want = P.coop_gated_grad(dy, x, w, w2, b, b)
    got = P.coop_gated_grad(dy, x, w, w2, b, b, want_x=False, want_bias=False)
    assert torch.equal(got[1], want[1]) and torch.equal(got[2], want[2]) and got[0] is None and got[3] is None
    got = P.coop_gated_grad(dy, x, w, w2, b, b, want_x=False, want_weight=False)
    assert torch.equal(got[3], want[3]) and torch.equal(got[4], want[4])
    assert torch.equal(P.coop_gated_grad(dy, x, w, w2, b, b, want_weight=False, want_bias=False)[0], want[0])
    for shift in (0, 1):    # (elements; the residual is where the result goes)
        place = torch.full((n * m + 1024 + shift,), 3.0, dtype=dtype, device="cuda")
        out = place[512 + shift:512 + shift + n * m].view(n, m)
        out.copy_(res)
        got = P.coop_linear(x, w, b, act=P.COOP_ACT_GELU, residual=out, out=out)
        assert (place[:512 + shift] == 3).all() and (place[512 + shift + n * m:] == 3).all()
        assert torch.equal(got, P.coop_linear(x, w, b, act=P.COOP_ACT_GELU, residual=res))
        out.fill_(3.0)
        P.coop_gated(x, w, w2, b, b, out=out)
        assert (place[:512 + shift] == 3).all() and (place[512 + shift + n * m:] == 3).all()


@gpu
@pytest.mark.parametrize("path", PATHS, ids=CALL_IDS[:len(PATHS)])
def test_rows_are_by_themselves(path):
    """What is no number in a row stays in that row, of the results and of the input's gradient."""
    (x, w, w2, b, res, dy), _ = dense_calls(*path, seed=5)
    n = x.shape[0]
    bad = sorted({0, n // 2, n - 1})
    good = torch.ones(n, dtype=torch.bool, device="cuda")
    good[bad] = False
    calls = [lambda: P.coop_linear(x, w, b, act=P.COOP_ACT_SILU, residual=res), lambda: P.coop_gated(x, w, w2, b, b),
             lambda: P.coop_linear_grad(dy, x, w, b, act=P.COOP_ACT_SILU)[0], lambda: P.coop_gated_grad(dy, x, w, w2, b, b)[0],
             lambda: P.coop_linear_grad(dy, x, w, b)[0]]
    want = [call() for call in calls]
    x[bad[0], 3], x[bad[-1], 0] = float("nan"), float("inf")
    dy[bad] = float("nan")
    for i, (call, before) in enumerate(zip(calls, want)):
        got = call()
        assert torch.equal(got[good], before[good]), i
        assert torch.isnan(got[bad[0]]).any(), i


# (what dz loses is kept: tiles with k whole, and in parts, of few rows; narrow, whole and ragged; tiles where the narrow kernel's memory is too small; tiles of many rows)
REST_PATHS = [(torch.bfloat16, 1, 1024, 3080), (torch.float16, 20, 72, 3200), (torch.bfloat16, 4100, 128, 32), (torch.float16, 9000, 100, 40), (torch.bfloat16, 5000, 40, 100),
              (torch.float16, 20000, 300, 9)]


@gpu
@pytest.mark.parametrize("path", REST_PATHS, ids=["%s-%d-%d-%d" % ((str(p[0])[6:],) + p[1:]) for p in REST_PATHS])
def test_paths_that_keep_what_dz_loses(path):
    test_same_bits_on_another_stream_with_any_workspace_and_in_a_graph(lambda: dense_calls(*path))
    test_what_is_asked_for_alone_is_the_same(path)
    test_rows_are_by_themselves(path)


@gpu
@pytest.mark.parametrize("n", [4, 3500])
@pytest.mark.parametrize("dtype", TYPES[1:], ids=IDS[1:])
def test_gradients_that_leave_the_type(dtype, n):
    """An infinity in dout, and (fp16) a dz beyond its numbers, are infinities in the gradients, of a call of any size."""
    g = rng(4)
    x, w, dy = normal(g, n, 16, dtype=dtype).abs() + 1, normal(g, 24, 16, dtype=dtype).abs() + 0.5, normal(g, n, 24, dtype=dtype)
    dy[1, 5], dy[2, 7] = float("inf"), -60000.0
    for dx, dw, db in (P.coop_linear_grad(dy, x, w, act=P.COOP_ACT_RELU, alpha=2.0), P.coop_linear_grad(dy, x, w, act=P.COOP_ACT_SILU, alpha=2.0)):
        assert (dx[1] == float("inf")).all() and (dw[5] == float("inf")).all() and math.isinf(db[5]) and float(db[7]) < -1e5
        rows = [i for i in range(n) if i not in (1, 2)]
        assert torch.isfinite(dx[rows]).all()
        if dtype == torch.float16:
            assert (dx[2] == -float("inf")).all() and (dw[7] == -float("inf")).all()


@gpu
@pytest.mark.parametrize("alpha", [2.0 ** -18, 2.0 ** -24, 3.0 * 2.0 ** 12, -2.0 ** -20])
@pytest.mark.parametrize("n,k,m", [(300, 64, 200), (1, 1024, 3080), (5000, 128, 120), (9000, 100, 40), (4000, 300, 260), (700, 600, 9), (2049, 130, 1024)])
def test_factors_that_take_dz_out_of_fp16(n, k, m, alpha):
    """alpha far from 1, of which dout (of a large one) or the weight (of a small one) makes up, so that gradients are well within fp16: a dz that is below its numbers, with
    alpha or without, is still within half a unit of itself."""
    dtype = torch.float16
    g = rng(n + m)
    up = max(abs(alpha), 1.0)
    x, dy = normal(g, n, k, dtype=dtype, scale=2.0 ** -10), normal(g, n, m, dtype=dtype, scale=2 / up)
    w = normal(g, m, k, dtype=dtype, scale=2.0 ** 11 / math.sqrt(k))
    for act in (P.COOP_ACT_GELU, P.COOP_ACT_RELU):
        z, ez = product64(x, w, None)
        slope, es = act64(z, act)[1], act_bound(z, ez, act)[1]
        d = dy.double() * alpha
        dz, edz = d * slope, d.abs() * (es + 4 * U * (slope.abs() + es))
        # (rounded as dz / alpha, or as dz: what TINY is of)
        off = edz + (dz.abs() + edz) * HALF[dtype] + TINY[dtype] * min(1.0, abs(alpha))
        _, pre = P.coop_linear(x, w, act=act, want_pre=True)
        for kept in (pre, None):
            dx, dw, db = P.coop_linear_grad(dy, x, w, pre=kept, act=act, alpha=alpha, grad_dtype=torch.float32)
            want = dz.t().contiguous() @ x.double()
            within(dw, want, off.t().contiguous() @ x.double().abs() + 2 * (n + 8) * U * ((dz.abs() + off).t().contiguous() @ x.double().abs()), "dw")
            want, size = dz @ w.double(), (dz.abs() + off) @ w.double().abs()
            within(dx, want, rounded(want, off @ w.double().abs() + 2 * (m + 8) * U * size, dtype), "dx")
            within(db, dz.sum(0), edz.sum(0) + (n + 8) * U * (dz.abs() + edz).sum(0), "db")


@gpu
@pytest.mark.parametrize("n,dim,dtype", [(300, 1027, torch.bfloat16), (300, 523, torch.float32), (500, 100, torch.float16), (40, 4096, torch.bfloat16), (9, 16384, torch.float16)])
def test_residual_norm_in_place(n, dim, dtype):
    g = rng(dim)
    x, f, dr, dy, w = normal(g, n, dim, dtype=dtype), normal(g, n, dim, dtype=dtype), normal(g, n, dim, dtype=dtype), normal(g, n, dim, dtype=dtype), normal(g, dim)
    L, t = layers.lib(), layers._DTYPES[dtype]
    for norms in (1, 2, 3, 3 | 4):
        a, b = (w.data_ptr() if norms & 1 else None), (w.data_ptr() if norms & 2 else None)

        def forward(xx, ff, r, y):
            stats = torch.empty((4, n), device="cuda")
            assert L.coop_residual_norm(xx.data_ptr(), ff.data_ptr(), n, dim, t, t, w.data_ptr(), 1, 0.9, norms, a, None, b, None, 0, 1e-5, r.data_ptr(), y.data_ptr(),
                                        stats.data_ptr(), None) == 0
            return stats

        def backward(d, e, stats, dx, df):
            dgate = torch.empty(dim, device="cuda")
            ws = torch.empty(L.coop_residual_norm_grad_workspace_bytes(n, dim, t), dtype=torch.uint8, device="cuda")
            assert L.coop_residual_norm_grad(d.data_ptr(), e.data_ptr(), x.data_ptr(), f.data_ptr(), n, dim, t, t, stats.data_ptr(), w.data_ptr(), 1, 0.9, norms, a, None, b,
                                             0, dx.data_ptr(), df.data_ptr(), dgate.data_ptr(), None, None, None, None, ws.data_ptr(), ws.numel(), None) == 0
            torch.cuda.synchronize()
            return dgate

        torch.cuda.synchronize()
        r, y, r2, y2 = torch.empty_like(x), torch.zeros_like(f), x.clone(), f.clone()
        torch.cuda.synchronize()
        stats = forward(x, f, r, y)
        assert torch.equal(stats, forward(r2, y2, r2, y2)) and torch.equal(r, r2) and (not norms & 2 or torch.equal(y, y2))
        dx, df, dx2, df2 = torch.empty_like(x), torch.empty_like(f), dr.clone(), dy.clone()
        torch.cuda.synchronize()
        assert torch.equal(backward(dr, dy, stats, dx, df), backward(dx2, df2, stats, dx2, df2)) and torch.equal(dx, dx2) and torch.equal(df, df2)


@gpu
@pytest.mark.parametrize("dtype,n,k,m", [(torch.bfloat16, (1 << 31) // 128 + 4099, 128, 128), (torch.float16, (1 << 31) // 100 + 77, 100, 75),
                                         (torch.float32, (1 << 30) // 64 + 4099, 64, 72)])
def test_dense_offsets_beyond_32_bits(dtype, n, k, m):
    """The last rows of an input of more than 2^32 bytes, against the same rows alone: their own, in the input's gradient and the result."""
    torch.cuda.empty_cache()
    g = rng(8)
    x, dy = torch.empty((n, k), dtype=dtype, device="cuda"), torch.empty((n, m), dtype=dtype, device="cuda")
    x[:1 << 20], dy[:1 << 20] = normal(g, 1 << 20, k, dtype=dtype), normal(g, 1 << 20, m, dtype=dtype)
    for a in (x, dy):
        for i in range(1 << 20, n, 1 << 20):
            a[i:i + (1 << 20)] = a[:min(1 << 20, n - i)]
    w, b = normal(g, m, k, dtype=dtype, scale=k ** -0.5), normal(g, m, dtype=dtype)
    out = P.coop_linear(x, w, b, act=P.COOP_ACT_SILU)
    dx, dw, db = P.coop_linear_grad(dy, x, w, b, act=P.COOP_ACT_SILU)
    first, part = n - (n % (1 << 20)) - (1 << 20), slice(0, 1 << 20)
    want, wants = P.coop_linear(x[part], w, b, act=P.COOP_ACT_SILU), P.coop_linear_grad(dy[part], x[part], w, b, act=P.COOP_ACT_SILU)
    for i in (first, 0, 1 << 20):
        assert torch.equal(out[i:i + (1 << 20)], want) and torch.equal(dx[i:i + (1 << 20)], wants[0])
    # whole copies of the first 2^20 rows, and what is left: the weight's gradient is theirs added up, each rounded to the type, and 32 bits' sums
    rest, copies = slice(n - n % (1 << 20), n), n >> 20
    tail = P.coop_linear_grad(dy[rest], x[rest], w, b, act=P.COOP_ACT_SILU, grad_dtype=torch.float32)
    whole = P.coop_linear_grad(dy[part], x[part], w, b, act=P.COOP_ACT_SILU, grad_dtype=torch.float32)
    z, _ = product64(x[:1 << 18], w, b)
    dz = dy[:1 << 18].double() * act64(z, P.COOP_ACT_SILU)[1]
    size = (dz.abs().t().contiguous() @ x[:1 << 18].double().abs()) * (n / (1 << 18)) * 1.05
    value = whole[1].double() * copies + tail[1].double()
    # (sums in order of at most 2^10 parts of at most n / 2^10 rows and the tiles' own: some 2^15 roundings of a random sign at worst one after the other)
    bound = rounded(value, 2.0 ** 15 * U * size, dtype)
    # (fp16 has no numbers of 65,520 and more: of a value that may be one its infinity is right)
    over = torch.isinf(dw) & (value.abs() + bound >= torch.finfo(dtype).max) & (torch.sign(dw) == torch.sign(value))
    within(torch.where(over, value, dw.double()), value, bound, "dw")
    within(db, whole[2].double() * copies + tail[2].double(), 2.0 ** 15 * U * dz.abs().sum(0) * (n / (1 << 18)) * 1.05, "db")


@gpu
def test_residual_norm_offsets_beyond_32_bits():
    torch.cuda.empty_cache()
    n, dim = (1 << 31) // 128 + 1001, 128
    g = rng(9)
    x = torch.empty((n, dim), dtype=torch.bfloat16, device="cuda")
    x.view(-1).copy_(torch.arange(n * dim, device="cuda", dtype=torch.int32).bitwise_and_(1023).sub_(500))
    x[-1000:] = normal(g, 1000, dim, dtype=torch.bfloat16)
    gate, w = normal(g, dim), normal(g, dim)
    kw = dict(gate=gate, after_weight=w, before_weight=w)
    r, y, stats = P.coop_residual_norm(x, x, **kw)
    got = P.coop_residual_norm_grad(x, x, x, x, stats, want_weight=False, **kw)
    last = x[-1000:].clone()
    r2, y2, stats2 = P.coop_residual_norm(last, last, **kw)
    want = P.coop_residual_norm_grad(last, last, last, last, stats2, want_weight=False, **kw)
    assert torch.equal(r[-1000:], r2) and torch.equal(y[-1000:], y2) and torch.equal(stats[:, -1000:], stats2)
    assert torch.equal(got[0][-1000:], want[0]) and torch.equal(got[1][-1000:], want[1])


# ---- gradients against differences, and all of them together --------------------------------------------------------------------------
def model64(table, ids, target, blocks, out):
    """A residual feed-forward model on learned rows in 64 bits: its loss, a mean."""
    def norm(v, w, b, eps=1e-5):
        c = v - v.mean(1, keepdim=True)
        return c / (c.square().mean(1, keepdim=True) + eps).sqrt() * w + b

    r = table[ids]
    y = norm(r, *blocks[0]["before"])
    for i, p in enumerate(blocks):
        g, u = y @ p["gate"].t() + p["gate_bias"], y @ p["up"].t() + p["up_bias"]
        h = g * torch.sigmoid(g) * u
        f = h @ p["down"].t() + p["down_bias"]
        r = 0.9 * r + norm(f, *p["after"]) * p["scale"]
        y = norm(r, *blocks[i + 1]["before"]) if i + 1 < len(blocks) else norm(r, *p["last"])
    return torch.nn.functional.cross_entropy(y @ out.t(), target)


@gpu
def test_a_model_of_them_together():
    """Forward, backward, clipping and a step, as a training program has them: gradients against those of 64 bits and against differences of the
    64-bit loss, the norm, and a captured step against an eager one.

    Bound: each operator's gradients hold to some 2^-17 of the sizes of the terms that they are sums of (64 terms of 2 u and the activations'
    40 u, in the tests above); behind ten operators in a row whose gradients' terms cancel to an eighth at worst that is 2^-11 of the largest."""
    g = rng(12)
    n, vocab, dim, ff = 300, 90, 40, 56
    table, out = normal(g, vocab, dim), normal(g, vocab, dim, scale=dim ** -0.5)
    ids = torch.randint(0, vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
    target = torch.randint(0, vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
    vector = lambda: (1 + normal(g, dim, scale=0.2), normal(g, dim, scale=0.2))  # noqa: E731
    blocks = [dict(before=vector(), after=vector(), last=vector(), scale=1 + normal(g, dim, scale=0.2), gate=normal(g, ff, dim, scale=dim ** -0.5),
                   up=normal(g, ff, dim, scale=dim ** -0.5), gate_bias=normal(g, ff, scale=0.1), up_bias=normal(g, ff, scale=0.1),
                   down=normal(g, dim, ff, scale=ff ** -0.5), down_bias=normal(g, dim, scale=0.1)) for _ in range(2)]
    params = [table, out, *blocks[0]["before"], *blocks[1]["last"]]
    for p in blocks:
        params += [p["gate"], p["up"], p["gate_bias"], p["up_bias"], p["down"], p["down_bias"], *p["after"], p["scale"]]
    params += list(blocks[1]["before"])

    def gradients():
        r = P.coop_embed(table, ids)
        y, mean, rstd = P.coop_layer_norm(r, *blocks[0]["before"])
        first, kept = (r, mean, rstd), []
        for i, p in enumerate(blocks):
            h, pre = P.coop_gated(y, p["gate"], p["up"], p["gate_bias"], p["up_bias"], want_pre=True)
            f = P.coop_linear(h, p["down"], p["down_bias"])
            bw, bb = blocks[i + 1]["before"] if i + 1 < len(blocks) else p["last"]
            kw = dict(gate=p["scale"], alpha=0.9, after_weight=p["after"][0], after_bias=p["after"][1], before_weight=bw)
            r2, y2, stats = P.coop_residual_norm(r, f, before_bias=bb, **kw)
            kept.append((r, y, h, pre, f, stats, kw))
            r, y = r2, y2
        loss, lse = P.coop_softmax_xent(y, out, target)
        dy, dout = P.coop_softmax_xent_grad(y, out, target, lse, torch.full_like(loss, 1.0 / n))
        dr, found = None, {}
        for i in reversed(range(len(blocks))):
            p, (r0, y0, h, pre, f, stats, kw) = blocks[i], kept[i]
            dr, df, dscale, daw, dab, dbw, dbb = P.coop_residual_norm_grad(dr, dy, r0, f, stats, **kw)
            dh, ddown, ddown_bias = P.coop_linear_grad(df, h, p["down"], p["down_bias"])
            dy, dgate, dup, dgb, dub = P.coop_gated_grad(dh, y0, p["gate"], p["up"], p["gate_bias"], p["up_bias"], pre=pre)
            found[i] = [dgate, dup, dgb, dub, ddown, ddown_bias, daw, dab, dscale], [dbw, dbb]
        dx, dw, db = P.coop_layer_norm_grad(dy, *first, blocks[0]["before"][0])
        dtable = P.coop_embed_grad(dx + dr, ids, vocab)
        return loss.mean(), [dtable, dout, dw, db, *found[1][1], *found[0][0], *found[1][0], *found[0][1]]

    loss, grads = gradients()
    wide = {id(p): p.double().requires_grad_() for p in params}
    blocks64 = [{k: tuple(wide.get(id(x), x.double()) for x in v) if isinstance(v, tuple) else wide[id(v)] for k, v in p.items()} for p in blocks]
    loss64 = model64(wide[id(table)], ids.long(), target.long(), blocks64, wide[id(out)])
    wants = torch.autograd.grad(loss64, [wide[id(p)] for p in params])
    assert abs(float(loss) - float(loss64.detach())) <= 2.0 ** -17 * float(loss64.detach())
    for i, (have, want) in enumerate(zip(grads, wants)):
        assert have.shape == want.shape
        within(have, want, 2.0 ** -11 * want.abs().max() + 0 * want, i)
    # along a direction: the loss 64 bits' differences (error: a step's square times a third derivative, which is of the size of the loss)
    v = [normal(g, *p.shape).double() for p in params]
    for p, d in zip(params, v):
        d *= float(p.abs().max())
    with torch.no_grad():
        def at(h):
            moved = {id(p): p.double() + h * d for p, d in zip(params, v)}
            b64 = [{k: tuple(moved.get(id(x), x.double()) for x in q) if isinstance(q, tuple) else moved[id(q)] for k, q in p.items()} for p in blocks]
            return float(model64(moved[id(table)], ids.long(), target.long(), b64, moved[id(out)]))
        slope = (at(1e-5) - at(-1e-5)) / 2e-5
    got = sum(float((gr.double() * d).sum()) for gr, d in zip(grads, v))
    size = sum(float((gr.double() * d).abs().sum()) for gr, d in zip(grads, v))
    assert abs(got - slope) <= 2.0 ** -11 * size
    # clipping and the step, eager and captured
    want_norm = math.sqrt(sum(float(w.square().sum()) for w in wants))
    copies = [[p.clone() for p in params] for _ in range(2)]
    eager, again = (P.AdamW(c, grads) for c in copies)
    plan = P.GradNorm(grads)
    norm, factor = plan.measure(0.1 * want_norm)
    assert abs(float(norm) - want_norm) <= 2.0 ** -11 * want_norm and abs(float(factor) - 0.1) <= 2.0 ** -10
    eager.step(1, 1e-2, grad_scale=factor)
    torch.cuda.synchronize()
    kept = [x.clone() for x in grads]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss2, captured = gradients()
        captured_plan = P.GradNorm(captured)
        norm2, factor2 = captured_plan.measure(0.1 * want_norm)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert same(kept, captured) and torch.equal(norm, norm2) and torch.equal(factor, factor2) and torch.equal(loss, loss2)
        assert same(kept, gradients()[1])
    again.step(1, 1e-2, grad_scale=factor2)
    assert same(copies[0], copies[1])


# ---- refusals ----------------------------------------------------------------------------------------------------------------------------
def test_refusals_of_the_c_abi():
    """What the host can see is refused before anything is launched."""
    L = layers.lib()
    A, N = 0x1000, None
    need = L.coop_linear_workspace_bytes(5000, 3001, 3001, 2, 0)
    assert need > 0 and L.coop_linear_workspace_bytes(1, 4096, 4096, 2, 1) == 0     # (a call that is small takes none)
    assert L.coop_linear_workspace_bytes(-1, 8, 8, 2, 1) == L.coop_linear_workspace_bytes(5000, 0, 8, 2, 1) == L.coop_linear_workspace_bytes(5000, 8, 8, 3, 1) == 0
    good = dict(x=A, n=5000, k=3001, w=A, m=3001, dtype=2, bias=N, act=0, res=N, out=A, pre=N, ws=A, wb=need)

    def linear(**kw):
        a = dict(good, **kw)
        return L.coop_linear(a["x"], a["n"], a["k"], a["w"], a["m"], a["dtype"], a["bias"], a["act"], 1.0, a["res"], a["out"], a["pre"], a["ws"], a["wb"], N)

    for kw in (dict(dtype=3), dict(act=4), dict(act=-1), dict(n=-1), dict(n=1 << 31), dict(k=0), dict(m=0), dict(k=(1 << 18) + 1), dict(m=(1 << 18) + 1), dict(x=A + 1),
               dict(w=A + 1), dict(bias=A + 1), dict(res=A + 1), dict(out=A + 1), dict(pre=A + 2), dict(wb=need - 1), dict(ws=A + 16)):
        assert linear(**kw) == -4, kw
    for kw in (dict(x=N), dict(w=N), dict(out=N), dict(ws=N)):
        assert linear(**kw) == -1, kw
    assert linear(n=0, x=N, out=N, ws=N) == 0
    need = L.coop_linear_grad_workspace_bytes(5000, 3001, 3001, 2, 2, 0, 0)
    good = dict(dout=A, x=A, n=5000, k=3001, w=A, m=3001, dtype=2, bias=N, act=2, pre=N, dx=A, dw=A, gd=2, db=A, ws=A, wb=need)

    def grad(**kw):
        a = dict(good, **kw)
        return L.coop_linear_grad(a["dout"], a["x"], a["n"], a["k"], a["w"], a["m"], a["dtype"], a["bias"], a["act"], 1.0, a["pre"], a["dx"], a["dw"], a["gd"], a["db"],
                                  a["ws"], a["wb"], N)

    for kw in (dict(dtype=3), dict(act=4), dict(n=-1), dict(k=0), dict(m=(1 << 18) + 1), dict(gd=1), dict(gd=7), dict(dout=A + 1), dict(x=A + 1), dict(w=A + 1), dict(bias=A + 1),
               dict(dx=A + 1), dict(dw=A + 1), dict(gd=0, dw=A + 2), dict(db=A + 2), dict(pre=A + 2), dict(wb=need - 1), dict(ws=A + 16)):
        assert grad(**kw) == -4, kw
    for kw in (dict(dout=N), dict(x=N), dict(w=N), dict(ws=N)):
        assert grad(**kw) == -1, kw
    assert grad(dx=N, dw=N, db=N, ws=N) == 0 and grad(n=0, dw=N, db=N, dout=N, x=N, ws=N) == 0      # nothing asked for
    need = L.coop_gated_workspace_bytes(5000, 3001, 3001, 2, 0)
    good = dict(x=A, n=5000, k=3001, g=A, u=A, f=3001, dtype=2, gb=N, ub=N, act=3, out=A, pre=N, ws=A, wb=need)

    def gated(**kw):
        a = dict(good, **kw)
        return L.coop_gated(a["x"], a["n"], a["k"], a["g"], a["u"], a["f"], a["dtype"], a["gb"], a["ub"], a["act"], a["out"], a["pre"], a["ws"], a["wb"], N)

    for kw in (dict(dtype=-1), dict(act=9), dict(n=-5), dict(f=0), dict(g=A + 1), dict(u=A + 1), dict(gb=A + 1), dict(ub=A + 1), dict(out=A + 1), dict(pre=A + 1), dict(wb=0)):
        assert gated(**kw) == -4, kw
    for kw in (dict(x=N), dict(g=N), dict(u=N), dict(out=N), dict(ws=N)):
        assert gated(**kw) == -1, kw
    need = L.coop_gated_grad_workspace_bytes(5000, 3001, 3001, 2, 0, 0)
    good = dict(dout=A, x=A, n=5000, k=3001, g=A, u=A, f=3001, dtype=2, gb=N, ub=N, act=3, pre=N, dx=A, dg=A, du=A, gd=0, dgb=A, dub=A, ws=A, wb=need)

    def gated_grad(**kw):
        a = dict(good, **kw)
        return L.coop_gated_grad(a["dout"], a["x"], a["n"], a["k"], a["g"], a["u"], a["f"], a["dtype"], a["gb"], a["ub"], a["act"], a["pre"], a["dx"], a["dg"], a["du"],
                                 a["gd"], a["dgb"], a["dub"], a["ws"], a["wb"], N)

    for kw in (dict(dg=N), dict(du=N), dict(dgb=N), dict(dub=N), dict(gd=1), dict(dg=A + 2), dict(dub=A + 1), dict(wb=need - 1), dict(act=5)):
        assert gated_grad(**kw) == -4, kw
    for kw in (dict(dout=N), dict(u=N), dict(ws=N)):
        assert gated_grad(**kw) == -1, kw
    good = dict(x=A, f=A, n=5, dim=8, dtype=2, st=0, gate=A, form=1, norms=3, aw=A, ab=A, bw=A, bb=A, wt=0, eps=1e-5, r=A, y=A, stats=A)

    def seam(**kw):
        a = dict(good, **kw)
        return L.coop_residual_norm(a["x"], a["f"], a["n"], a["dim"], a["dtype"], a["st"], a["gate"], a["form"], 1.0, a["norms"], a["aw"], a["ab"], a["bw"], a["bb"], a["wt"],
                                    a["eps"], a["r"], a["y"], a["stats"], N)

    for kw in (dict(dtype=4), dict(st=1), dict(wt=1), dict(norms=0), dict(norms=4), dict(norms=8), dict(norms=7), dict(norms=1), dict(norms=2), dict(dim=0), dict(dim=16385), dict(n=-1),
               dict(dtype=0, dim=8193), dict(form=0), dict(form=3), dict(gate=N), dict(eps=-1.0), dict(eps=float("nan")), dict(x=A + 2), dict(f=A + 1), dict(gate=A + 2), dict(aw=A + 2),
               dict(r=A + 2), dict(y=A + 1), dict(stats=A + 2)):
        assert seam(**kw) == -4, kw
    for kw in (dict(x=N), dict(f=N), dict(r=N), dict(y=N), dict(stats=N)):
        assert seam(**kw) == -1, kw
    assert seam(n=0, x=N, f=N, r=N, y=N, stats=N) == 0
    need = L.coop_residual_norm_grad_workspace_bytes(5, 8, 2)
    assert need > 0 and L.coop_residual_norm_grad_workspace_bytes(5, 16385, 2) == 0
    good = dict(dr=A, dy=A, x=A, f=A, n=5, dim=8, dtype=2, st=0, stats=A, gate=A, form=1, norms=3, aw=A, ab=A, bw=A, wt=0, dx=A, df=A, dgate=A, daw=A, dab=A, dbw=A, dbb=A, ws=A, wb=need)

    def seam_grad(**kw):
        a = dict(good, **kw)
        return L.coop_residual_norm_grad(a["dr"], a["dy"], a["x"], a["f"], a["n"], a["dim"], a["dtype"], a["st"], a["stats"], a["gate"], a["form"], 1.0, a["norms"], a["aw"], a["ab"],
                                         a["bw"], a["wt"], a["dx"], a["df"], a["dgate"], a["daw"], a["dab"], a["dbw"], a["dbb"], a["ws"], a["wb"], N)

    for kw in (dict(norms=1), dict(norms=2), dict(norms=7), dict(gate=N), dict(dgate=N), dict(form=0), dict(dim=0), dict(wb=need - 1), dict(ws=A + 8), dict(dx=A + 2), dict(df=A + 1),
               dict(dgate=A + 2), dict(dbb=A + 1)):
        assert seam_grad(**kw) == -4, kw
    for kw in (dict(dy=N), dict(x=N), dict(f=N), dict(stats=N), dict(dx=N), dict(df=N), dict(ws=N)):
        assert seam_grad(**kw) == -1, kw
    t = (layers._CGradTensor * 2)()
    need = L.coop_grad_norm_workspace_bytes(t, 0)
    norm = lambda n=1, bound=1.0, ts=t, scale=N, out=A, ws=A, wb=1 << 20: L.coop_grad_norm(ts, n, bound, scale, out, A, ws, wb, N)  # noqa: E731
    assert norm(n=-1) == -4 and norm(ts=N) == -1 and norm(bound=-1.0) == -4 and norm(bound=float("nan")) == -4 and norm(ws=N) == -1 and norm(ws=A + 4) == -4
    assert norm(out=A + 2) == -4 and norm(scale=A + 1) == -4 and need > 0 and norm(n=0, wb=need - 1) == -4
    t[0].n_rows, t[0].dim = 3, 7
    assert norm() == -1 and L.coop_grad_scale(t, 1, A, N) == -1             # elements without an address
    t[0].grad, t[0].dtype = A, 3
    assert norm() == -4 and L.coop_grad_scale(t, 1, A, N) == -4
    t[0].dtype, t[0].grad = 0, A + 2
    assert norm() == -4
    t[0].grad, t[0].n_rows_dev = A, A + 1
    assert norm() == -4
    t[0].n_rows_dev, t[0].n_rows, t[0].dim = None, 1 << 30, 1 << 30
    assert norm() == -4 and L.coop_grad_norm_workspace_bytes(t, 1) == 0
    t[0].n_rows = -1
    assert norm() == -4
    t[0].n_rows = 3
    assert L.coop_grad_scale(t, 0, N, N) == 0 and L.coop_grad_scale(t, 1, N, N) == -1 and L.coop_grad_scale(t, 1, A + 2, N) == -4


def test_gradients_with_elements_in_common_are_not_scaled():
    """One given twice, one within another and one that begins within another are refused before anything is launched, in any order."""
    L = layers.lib()
    A = 0x10000

    def common(*tensors):
        t = (layers._CGradTensor * len(tensors))()
        for c, (at, rows, dim, dtype) in zip(t, tensors):
            c.grad, c.n_rows, c.dim, c.dtype = at, rows, dim, dtype
        return L.coop_grad_scale(t, len(tensors), A, None) == -4

    one = (A, 4, 8, 0)                       # 128 bytes
    for other in (one, (A + 124, 1, 1, 0), (A - 4, 1, 2, 0), (A + 64, 1, 8, 2), (A - 64, 1, 1000, 1)):
        assert common(one, other) and common(other, one) and common(one, (A + 4096, 1, 8, 0), (A - 4096, 0, 8, 0), other)


@gpu
def test_gradients_side_by_side_are_scaled():
    """Neighbours in memory have nothing in common, nor has one of no elements, in any order."""
    flat = torch.ones(96, device="cuda")
    parts = [flat[64:96], flat[0:32], flat[16:16], flat[32:64], flat[40:40]]
    P.GradNorm(parts).apply(torch.full((1,), 0.5, device="cuda"))
    assert (flat == 0.5).all()
    with pytest.raises(P.CoopError) as e:
        P.GradNorm([flat, flat[:1]]).apply(torch.full((1,), 0.5, device="cuda"))
    assert e.value.code == -4 and (flat == 0.5).all()
    norm, _ = P.GradNorm([flat, flat]).measure()
    assert abs(float(norm) - math.sqrt(48.0)) <= 2 * U * 7


@gpu
def test_refusals_of_the_binding():
    x, w, v = torch.zeros((8, 6), device="cuda"), torch.zeros((5, 6), device="cuda"), torch.zeros(6, device="cuda")
    y, stats = torch.zeros((8, 5), device="cuda"), torch.zeros((4, 8), device="cuda")
    for call in (lambda: P.coop_linear(x[:, ::2], w), lambda: P.coop_linear(x, w.half()), lambda: P.coop_linear(x, w[:, :4].contiguous()), lambda: P.coop_linear(x.double(), w.double()),
                 lambda: P.coop_linear(x, w, v), lambda: P.coop_linear(x, w, residual=x), lambda: P.coop_linear(x, w, out=x), lambda: P.coop_linear(x.cpu(), w),
                 lambda: P.coop_linear_grad(x, x, w), lambda: P.coop_linear_grad(y, x, w, pre=y.half(), act=1), lambda: P.coop_linear_grad(y, x, w, pre=x, act=1),
                 lambda: P.coop_gated(x, w, w[:4]), lambda: P.coop_gated(x, w, w.half()), lambda: P.coop_gated_grad(x, x, w, w), lambda: P.coop_gated_grad(y, x, w, w, pre=y),
                 lambda: P.coop_residual_norm(x, y), lambda: P.coop_residual_norm(x.half(), x), lambda: P.coop_residual_norm(x, x, gate=v[:5]),
                 lambda: P.coop_residual_norm(x, x, gate=y), lambda: P.coop_residual_norm(x, x, after_weight=v.double()), lambda: P.coop_residual_norm(x, x, rms=True, after_bias=v),
                 lambda: P.coop_residual_norm(x, x, after=False, after_weight=v), lambda: P.coop_residual_norm(x, x, before=False, before_bias=v),
                 lambda: P.coop_residual_norm_grad(x, None, x, x, stats), lambda: P.coop_residual_norm_grad(None, x, x, x, stats, before=False),
                 lambda: P.coop_residual_norm_grad(x, x, x, x, stats[:2]), lambda: P.GradNorm([x[:, ::2]]), lambda: P.GradNorm([x.double()]),
                 lambda: P.GradNorm([(x, v[:1])]), lambda: P.GradNorm([x]).measure(1.0, grad_scale=v), lambda: P.GradNorm([x]).apply(v)):
        with pytest.raises((AssertionError, AttributeError, TypeError)):
            call()
    for call in (lambda: P.coop_linear(x, w, act=7), lambda: P.coop_residual_norm(x, x, after=False, before=False), lambda: P.coop_residual_norm(x, x, eps=-1.0),
                 lambda: P.GradNorm([x]).measure(-1.0), lambda: P.GradNorm([x]).measure(1.0, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(P.CoopError) as e:
            call()
        assert e.value.code == -4
