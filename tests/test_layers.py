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
         (20000, 33, 40), (70001, 24, 20), (4097, 72, 4100), (4097, 4100, 72), (72, 4100, 4104), (1, 2, 9000), (2, 9000, 1)]


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
