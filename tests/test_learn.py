"""The operators of learned vertex representations against plain implementations in 64 bits: at the sizes, types, ids and
targets where they can go wrong; gradients against the formulas and against differences; refusals.

Tolerances are bounds, elementwise: u = 2^-24 for an operation in 32 bits, the sums' worst order included, and half a unit in
the last place of the type that a result is stored in (for fp16 also of its smallest numbers)."""
import ctypes as C
import gc
import importlib.util
import os
import types
import weakref

import numpy as np
import pytest
import torch

import paper_2310_12403_amd as P
import synth
from paper_2310_12403_amd import learn

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}
TYPES = [torch.float32, torch.float16, torch.bfloat16]
IDS = ["f32", "f16", "bf16"]
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


def within(got, want, bound):
    got, want = got.double(), want.double()
    assert got.shape == want.shape
    off = (got - want).abs()
    bad = ~(off <= bound) & ~((got == want) | (torch.isnan(got) & torch.isnan(want)))
    assert not bad.any(), "%d of %d, worst %g of a bound of %g" % (bad.sum(), bad.numel(), off[bad].max(), torch.as_tensor(bound).expand_as(off)[bad][off[bad].argmax()] if not torch.isnan(off[bad].max()) else float("nan"))


def status_is(code):
    try:
        P.coop_gather_status()
        return code == 0
    except P.CoopError as e:
        return e.code == code


# ---- lookup --------------------------------------------------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("out_dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("n,dim", [(0, 5), (1, 1), (3, 2), (65, 3), (1000, 7), (257, 8), (129, 75), (64, 128), (33, 1031), (5, 20000)])
def test_embed(dtype, out_dtype, n, dim):
    g = rng(n + dim)
    table = unaligned(normal(g, 50, dim, dtype=dtype))
    ids = torch.randint(-1, 50, (n,), generator=g, device="cuda", dtype=torch.int32)
    scale = torch.rand(n, generator=g, device="cuda")
    for s in (None, scale):
        got = P.coop_embed(table, ids, scale=s, alpha=3.3, pad=-1, dtype=out_dtype)
        want = table.double()[ids.long().clamp(min=0)] * 3.3 * (1.0 if s is None else s.double()[:, None])
        want[ids == -1] = 0.0
        within(got, want, want.abs() * (HALF[out_dtype] * (1 + 4 * U) + 4 * U) + TINY[out_dtype])
    assert status_is(0)


@gpu
def test_embed_ids_out_of_range_are_zero_and_reported():
    table = torch.ones((10, 64), device="cuda")
    ids = torch.tensor([3, -1, 10, 2 ** 31 - 1, -2 ** 31 + 1, 9], dtype=torch.int32, device="cuda")
    out = P.coop_embed(table, ids)
    assert out.sum(1).tolist() == [64, 0, 0, 0, 0, 64] and status_is(-2) and status_is(0)
    out = P.coop_embed(table, ids[:2], pad=-1)
    assert out.sum(1).tolist() == [64, 0] and status_is(0)
    grad = P.coop_embed_grad(torch.ones((6, 64), device="cuda"), ids, 10)
    assert grad.sum(1).tolist() == [0, 0, 0, 64] + [0] * 5 + [64] and status_is(-2) and status_is(0)
    rows, grad = P.coop_embed_grad_rows(torch.ones((6, 64), device="cuda"), ids, 10, pad=-1)
    assert rows.tolist() == [3, 9] and grad.shape == (2, 64) and status_is(-2)


@gpu
def test_embed_offsets_beyond_32_bits():
    n, dim = 70000, 40000                      # 5.6 GB of table: rows begin beyond 2^32 bytes and 2^31 elements
    table = torch.zeros((n, dim), dtype=torch.float16, device="cuda")
    at = [0, 1, 53686, 53688, 69999]
    for k, r in enumerate(at):
        table[r] = k + 1
    ids = torch.tensor(at, dtype=torch.int32, device="cuda")
    out = P.coop_embed(table, ids)
    assert torch.equal(out, table[ids.long()])
    p = torch.zeros(1, device="cuda")
    del table, out
    grad = P.coop_embed_grad(torch.ones((5, dim), dtype=torch.float16, device="cuda"), ids, n, dtype=torch.float16)
    assert float(grad.sum(dtype=torch.float64)) == 5.0 * dim and bool((grad[ids.long()] == 1).all()) and p.item() == 0


# ---- its gradient ---------------------------------------------------------------------------------------------------------
def plain_embed_grad(dout, ids, n_rows, factor, live):
    x, at = (dout.double() * factor[:, None])[live].cpu(), ids.long()[live].cpu()     # (on the host: 100,000 atomics on one row take many seconds)
    grad = torch.zeros((n_rows, dout.shape[1]), dtype=torch.float64).index_add_(0, at, x)
    size = torch.zeros_like(grad).index_add_(0, at, x.abs())
    count = torch.zeros(n_rows, dtype=torch.float64).index_add_(0, at, torch.ones(at.shape[0], dtype=torch.float64))
    return grad.cuda(), size.cuda(), count.cuda()


ID_SETS = {
    "spread": lambda g, n, v: torch.randint(0, v, (n,), generator=g, device="cuda"),
    "one": lambda g, n, v: torch.full((n,), v - 1, device="cuda"),
    "two": lambda g, n, v: torch.randint(0, 2, (n,), generator=g, device="cuda") * (v - 1),
    "hub": lambda g, n, v: torch.where(torch.rand(n, generator=g, device="cuda") < 0.7, v // 2, torch.randint(0, v, (n,), generator=g, device="cuda")),
    "pads": lambda g, n, v: torch.where(torch.rand(n, generator=g, device="cuda") < 0.5, -7, torch.randint(0, v, (n,), generator=g, device="cuda")),
    "all pads": lambda g, n, v: torch.full((n,), -7, device="cuda"),
    "each once": lambda g, n, v: torch.randperm(v, generator=g, device="cuda")[:n] if n <= v else torch.arange(n, device="cuda") % v,
}


@gpu
@pytest.mark.parametrize("ids_of", list(ID_SETS))
@pytest.mark.parametrize("n,n_rows,dim", [(0, 5, 3), (1, 1, 1), (1, 300, 64), (31, 40, 5), (32, 2, 8), (33, 255, 4), (4097, 256, 75), (5000, 70000, 64),
                                          (20011, 33, 130), (700, 3000, 1030), (100000, 17000000, 4)])
def test_embed_grad(ids_of, n, n_rows, dim):
    g = rng(n + n_rows + dim)
    dtype, out_dtype = TYPES[(n + dim) % 3], TYPES[(n_rows + dim) % 3]
    dout = unaligned(normal(g, n, dim, dtype=dtype))
    ids = ID_SETS[ids_of](g, n, n_rows).to(torch.int32)
    scale = torch.rand(n, generator=g, device="cuda") + 0.5
    want, size, count = plain_embed_grad(dout, ids, n_rows, scale.double() * 1.7, ids >= 0)
    bound = size * (count[:, None] + 4) * U + (want.abs() + size * (count[:, None] + 4) * U) * HALF[out_dtype] + TINY[out_dtype]
    got = P.coop_embed_grad(dout, ids, n_rows, scale=scale, alpha=1.7, pad=-7, dtype=out_dtype)
    within(got, want, bound)
    rows, part = P.coop_embed_grad_rows(dout, ids, n_rows, scale=scale, alpha=1.7, pad=-7, dtype=out_dtype)
    assert torch.equal(rows.long(), count.nonzero()[:, 0])
    assert torch.equal(part, got[rows.long()])          # one order of the sums, either way
    rows2, part2, k = P.coop_embed_grad_rows(dout, ids, n_rows, scale=scale, alpha=1.7, pad=-7, dtype=out_dtype, wait=False)
    assert int(k) == rows.numel() and torch.equal(rows2[:int(k)], rows) and torch.equal(part2[:int(k)], part)
    assert status_is(0)


# around the numbers of tokens at which the sort changes its way, the last of them past 512 tiles of 8,192
@gpu
@pytest.mark.parametrize("ids_of", ["spread", "hub", "pads", "each once"])
@pytest.mark.parametrize("n,n_rows,dim", [(511, 100000, 2), (512, 300, 3), (513, 300, 2), (8192, 9000, 2), (8193, 400000, 1), (4194305, 5000000, 1)])
def test_embed_grad_orders(ids_of, n, n_rows, dim):
    g = rng(n)
    ids = ID_SETS[ids_of](g, n, n_rows).to(torch.int32)
    dout = torch.randint(-8, 9, (n, dim), generator=g, device="cuda").float()       # small whole numbers: the sums are exact
    live = (ids >= 0).cpu().numpy()
    at, x = ids.cpu().numpy()[live], dout.double().cpu().numpy()[live]              # (on the host: millions of atomics on one row take minutes)
    want = torch.from_numpy(np.stack([np.bincount(at, x[:, d], n_rows) for d in range(dim)], 1)).cuda()
    assert torch.equal(P.coop_embed_grad(dout, ids, n_rows, pad=-7).double(), want)
    rows, part = P.coop_embed_grad_rows(dout, ids, n_rows, pad=-7)
    assert torch.equal(rows.long(), torch.unique(ids[ids >= 0]).long()) and torch.equal(part.double(), want[rows.long()])
    assert status_is(0)


@gpu
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("out_dtype", TYPES, ids=IDS)
def test_embed_grad_types_and_adjoint(dtype, out_dtype):
    """<dout, embed(E)> = <grad, E>, whatever the rows: the gradient is the lookup's adjoint."""
    g = rng(5)
    n, n_rows, dim = 3000, 500, 40
    ids = ID_SETS["hub"](g, n, n_rows).to(torch.int32)
    dout, table = normal(g, n, dim, dtype=dtype), normal(g, n_rows, dim)
    grad = P.coop_embed_grad(dout, ids, n_rows, alpha=2.0, dtype=out_dtype)
    want, size, count = plain_embed_grad(dout, ids, n_rows, torch.full((n,), 2.0, dtype=torch.float64, device="cuda"), ids >= 0)
    bound = size * (count[:, None] + 4) * U + want.abs() * 2 * HALF[out_dtype] + TINY[out_dtype]
    within(grad, want, bound)
    left = (dout.double() * P.coop_embed(table, ids, alpha=2.0).double()).sum()
    right = (grad.double() * table.double()).sum()
    assert abs(left - right) <= (bound * table.double().abs()).sum() + 2 * U * (dout.double().abs() * table.double()[ids.long()].abs() * 2).sum()


# ---- layer norm -----------------------------------------------------------------------------------------------------------
def plain_norm(x, w, b, eps):
    x, w, b = x.double(), w.double(), b.double()
    mean = x.mean(1)
    var = ((x - mean[:, None]) ** 2).mean(1)
    rstd = 1 / torch.sqrt(var + eps)
    return (x - mean[:, None]) * rstd[:, None] * w + b, mean, rstd


NORM_SIZES = [(0, 4), (1, 1), (5, 2), (3, 3), (70, 4), (33, 7), (257, 8), (1000, 64), (515, 75), (300, 100), (129, 128), (77, 513), (64, 602),
              (40, 1030), (31, 2048), (17, 2500), (9, 8191), (5, 16384), (3, 20001), (2, 32768)]


@gpu
@pytest.mark.parametrize("rows,dim", NORM_SIZES)
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_layer_norm(rows, dim, dtype):
    g = rng(rows + dim)
    x = unaligned((normal(g, rows, dim) * 2 + normal(g, rows, 1) * 3).to(dtype))
    dy = unaligned(normal(g, rows, dim, dtype=dtype))
    for wtype in {torch.float32, dtype}:
        w, b = unaligned((1 + normal(g, dim, scale=0.2)).to(wtype)), unaligned(normal(g, dim, dtype=wtype, scale=0.2))
        y, mean, rstd = P.coop_layer_norm(x, w, b, eps=1e-5)
        want, m, r = plain_norm(x, w, b, 1e-5)
        if rows == 0:
            assert y.shape == (0, dim)
            dx, dw, db = P.coop_layer_norm_grad(dy, x, mean, rstd, w)
            assert dx.shape == (0, dim) and not dw.any() and not db.any()
            continue
        top = x.double().abs().amax(1)
        em = (dim + 2) * U * top                                       # of the mean: a sum of dim terms
        within(mean, m, em)
        # of x - mean, relative to 1 / rstd; of the variance, twice that times the largest |x - mean| rstd, and its own sum
        ec = (em + 2 * U * top) * r
        er = r * ((dim + 8) * U + 2 * ec * (2 * top * r))
        within(rstd, r, er)
        hat = ((x.double() - m[:, None]) * r[:, None])
        eh = ec[:, None] + hat.abs() * (er / r)[:, None] + 2 * U * hat.abs()
        within(y, want, eh * w.double().abs() + (want.abs() + (hat * w.double()).abs()) * 2 * U + want.abs() * HALF[dtype] + TINY[dtype])
        # gradient, for the statistics as they are
        dx, dw, db = P.coop_layer_norm_grad(dy, x, mean, rstd, w)
        md, rd = mean.double(), rstd.double()
        hat = (x.double() - md[:, None]) * rd[:, None]
        d = dy.double() * w.double()
        s1, s2 = d.mean(1, keepdim=True), (d * hat).mean(1, keepdim=True)
        want = (d - s1 - hat * s2) * rd[:, None]
        eh = (x.double().abs() + md.abs()[:, None]) * rd[:, None] * 2 * U + hat.abs() * 2 * U
        e1 = (dim + 3) * U * d.abs().mean(1, keepdim=True)
        e2 = ((dim + 4) * U * (d * hat).abs() + d.abs() * eh).mean(1, keepdim=True)
        e = (3 * U * d.abs() + e1 + s1.abs() * 2 * U + hat.abs() * e2 + eh * s2.abs() + 3 * U * (hat * s2).abs()) * rd[:, None]
        within(dx, want, e + want.abs() * (HALF[dtype] + 4 * U) + TINY[dtype])
        within(dw, (dy.double() * hat).sum(0), ((rows + 2) * U * (dy.double() * hat).abs() + dy.double().abs() * eh).sum(0))
        within(db, dy.double().sum(0), (rows + 2) * U * dy.double().abs().sum(0))


@gpu
def test_layer_norm_without_weights_in_place_and_degenerate_rows():
    g = rng(1)
    x = normal(g, 300, 96)
    x[3] = 5.0                                  # no variance: y = 0, rstd = 1 / sqrt(eps)
    x[4, 7] = float("nan")
    x[5, 9] = float("inf")
    y, mean, rstd = P.coop_layer_norm(x, eps=1e-3)
    want, _, _ = plain_norm(x, torch.ones(96, device="cuda"), torch.zeros(96, device="cuda"), 1e-3)
    assert not y[3].any() and abs(float(rstd[3]) - 1e-3 ** -0.5) < 1e-4
    assert torch.isnan(y[4]).all() and torch.isnan(y[5]).any()
    fine = [i for i in range(300) if i not in (4, 5)]
    assert (y[fine].double() - want[fine]).abs().max() < 1e-4
    dy = normal(g, 300, 96)
    dx, dw, db = P.coop_layer_norm_grad(dy, x, mean, rstd)
    assert torch.isfinite(dx[fine]).all() and torch.isnan(dw).any() and torch.isfinite(db).all()
    only, none, none2 = P.coop_layer_norm_grad(dy, x, mean, rstd, want_weight=False)
    assert none is None and none2 is None and torch.equal(torch.nan_to_num(only), torch.nan_to_num(dx))
    copy, dcopy = x.clone(), dy.clone()
    assert torch.equal(torch.nan_to_num(P.coop_layer_norm(copy, eps=1e-3, out=copy)[0]), torch.nan_to_num(y))
    P.coop_layer_norm_grad(dcopy, x, mean, rstd, out=dcopy)
    assert torch.equal(torch.nan_to_num(dcopy), torch.nan_to_num(dx))


@gpu
def test_layer_norm_grad_against_differences():
    g = rng(2)
    x, dy, w, b = normal(g, 40, 75), normal(g, 40, 75), 1 + normal(g, 75, scale=0.3), normal(g, 75)
    _, mean, rstd = P.coop_layer_norm(x, w, b)
    grads = P.coop_layer_norm_grad(dy, x, mean, rstd, w)
    for k, t in enumerate((x, w, b)):
        way = normal(g, *t.shape).double()
        loss = []
        for sign in (1, -1):
            args = [x.double(), w.double(), b.double()]
            args[k] = args[k] + sign * 1e-5 * way
            loss.append((plain_norm(*args, 1e-5)[0] * dy.double()).sum())
        slope = (loss[0] - loss[1]) / 2e-5
        got = (grads[k].double() * way).sum()
        # the gradient's own error (bounded above by the test of the formula), and the differences' 1e-10 of curvature
        assert abs(got - slope) <= 200 * U * (grads[k].double().abs() * way.abs()).sum() + 1e-4 * 40 * 75 * U * 100 + 1e-6 * abs(slope)


# ---- cross entropy -----------------------------------------------------------------------------------------------------------
def plain_xent(h, w, t, alpha, ignore=-1):
    z = alpha * (h.double() @ w.double().t())
    lse = torch.logsumexp(z, 1)
    live = t != ignore
    zt = z.gather(1, t.long().clamp(min=0)[:, None])[:, 0]
    return torch.where(live, lse - zt, 0.0), lse, z


def xent_bounds(h, w, z, lse, alpha):
    """Bounds of the errors of a row's logits and of its lse: the products' sums, the scale, exponentials and sums."""
    terms = h.double().abs() @ w.double().abs().t() * abs(alpha)
    ez = ((h.shape[1] + 4) * U * terms + 4 * U * z.abs()).amax(1)
    length = w.shape[0] + 64
    return ez, ez + (length + 16) * U + 4 * U * (lse.abs() + z.abs().amax(1))


XENT_SIZES = [(1, 1, 1), (1, 5, 16), (2, 300, 3), (24, 1000, 128), (32, 257, 64), (33, 256, 64), (70, 999, 75), (256, 512, 128), (257, 513, 136), (300, 1030, 300),
              (5, 3001, 1024), (600, 40, 200), (300, 1030, 100), (65, 64, 32), (64, 65, 20), (513, 20000, 24)]


@gpu
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("n,vocab,dim", XENT_SIZES)
def test_softmax_xent(dtype, n, vocab, dim):
    check_xent(dtype, n, vocab, dim, 0.8)


# products in tiles of 256 rows; a vocabulary in three pieces; one split with several stages of rows; more rows than one block looks through
# for the largest coefficient, of a few classes; rows that end in each quarter of a stage
@gpu
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("n,vocab,dim", [(4097, 4100, 200), (16384, 20000, 136), (300, 140000, 40), (200, 131100, 128), (40000, 47, 24), (33000, 70, 200), (1200001, 300, 136),
                                         (16, 70, 8), (17, 81, 24), (48, 113, 72), (63, 127, 120)])
def test_softmax_xent_of_many_and_of_few(dtype, n, vocab, dim):
    check_xent(dtype, n, vocab, dim, 0.8)


@gpu
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("alpha", [-0.7, 0.0])
@pytest.mark.parametrize("n,vocab,dim", [(20, 700, 100), (300, 700, 100), (300, 700, 200)])
def test_softmax_xent_scale(dtype, alpha, n, vocab, dim):
    check_xent(dtype, n, vocab, dim, alpha)


def check_xent(dtype, n, vocab, dim, alpha):
    g = rng(n + vocab + dim)
    h, w = normal(g, n, dim, dtype=dtype), normal(g, vocab, dim, dtype=dtype, scale=2 * dim ** -0.5)
    if n % 2:
        h, w = unaligned(h), unaligned(w)
    t = torch.randint(0, vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
    t[torch.rand(n, generator=g, device="cuda") < 0.2] = -1
    t[:1] = vocab - 1
    loss, lse = P.coop_softmax_xent(h, w, t, alpha=alpha)
    want, want_lse, z = plain_xent(h, w, t, alpha)
    ez, el = xent_bounds(h, w, z, want_lse, alpha)
    within(lse, want_lse, el)
    within(loss, want, el + ez + 4 * U * want.abs())
    # gradient, at the lse that came back, from dloss of all sizes
    dloss = torch.randn(n, generator=g, device="cuda") * torch.exp2(torch.randint(-6, 3, (n,), generator=g, device="cuda").float())
    dh, dw = P.coop_softmax_xent_grad(h, w, t, lse, dloss, alpha=alpha)
    c = torch.where(t >= 0, dloss.double() * alpha, 0.0)
    p = torch.exp(z - lse.double()[:, None])
    hot = torch.zeros_like(p).scatter_(1, t.long().clamp(min=0)[:, None], 1.0)
    G = (p - hot) * c[:, None]
    # p through errors of the exponent and of the exponential, then G's own rounding
    ep = p * (ez + 4 * U * (lse.double().abs() + z.abs().amax(1)) + 4 * U)[:, None] * c.abs()[:, None]
    eG = ep + (G.abs() + ep) * (HALF[dtype] + 4 * U)
    if dtype == torch.float16:      # numbers below 2^-14 of the lifted ones are spaced 2^-24 apart
        eG = eG + (c.abs().max() * 2.0 ** -13) * 2.0 ** -25
    W, H = w.double(), h.double()
    for got, want, err, size, terms in ((dh, G @ W, eG @ W.abs(), G.abs() @ W.abs(), vocab), (dw, G.t() @ H, eG.t() @ H.abs(), G.abs().t() @ H.abs(), n)):
        e = err + (terms + 256 + 16) * U * (size + err)
        within(got, want, e + (want.abs() + e) * HALF[dtype] + TINY[dtype])
    only = P.coop_softmax_xent_grad(h, w, t, lse, dloss, alpha=alpha, want_weight=False)
    assert only[1] is None and torch.equal(only[0], dh)
    only = P.coop_softmax_xent_grad(h, w, t, lse, dloss, alpha=alpha, want_hidden=False)
    assert only[0] is None and torch.equal(only[1], dw)
    assert status_is(0)


@gpu
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_softmax_xent_grad_against_differences(dtype):
    g = rng(9)
    n, vocab, dim = 60, 700, 72
    h, w = normal(g, n, dim, dtype=dtype), normal(g, vocab, dim, dtype=dtype, scale=0.2)
    t = torch.randint(-1, vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
    dloss = torch.rand(n, generator=g, device="cuda") + 0.5
    _, lse = P.coop_softmax_xent(h, w, t)
    grads = P.coop_softmax_xent_grad(h, w, t, lse, dloss)
    for k, x in enumerate((h, w)):
        way = normal(g, *x.shape).double()
        loss = []
        for sign in (1, -1):
            args = [h.double(), w.double()]
            args[k] = args[k] + sign * 1e-5 * way
            loss.append((plain_xent(*args, t, 1.0)[0] * dloss.double()).sum())
        slope, got = (loss[0] - loss[1]) / 2e-5, (grads[k].double() * way).sum()
        # every element of a gradient is off by at most a rounding of G's terms and one of its own: G's terms are at most dloss,
        # two of each row (the target's and the others' sum) as long as the other operand's largest number
        size = 2 * dloss.double().abs().sum() * (w if k == 0 else h).double().abs().max() * way.abs().max() * dim
        assert abs(got - slope) <= (HALF[dtype] + 400 * U) * size * 2 + 1e-6 * abs(slope)


@gpu
@pytest.mark.parametrize("dim,dtype", [(64, torch.bfloat16), (200, torch.bfloat16), (100, torch.float16), (64, torch.float32)])
def test_softmax_xent_rows_without_targets_and_bad_targets(dim, dtype):
    g = rng(3)
    n, vocab = 300, 600
    h, w = normal(g, n, dim, dtype=dtype), normal(g, vocab, dim, dtype=dtype)
    t = torch.randint(0, vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
    t[10], t[11], t[12] = -1, vocab, -5
    h[10] = float("nan")                         # a masked row's values reach nothing
    h[13] = float("inf")                         # a live row's do
    loss, lse = P.coop_softmax_xent(h, w, t)
    assert status_is(-2) and loss[10] == 0 and loss[11] == 0 and loss[12] == 0 and torch.isnan(loss[13])
    assert torch.isfinite(torch.cat([loss[:13], loss[14:], lse[:10], lse[14:]])).all()
    t[13] = -1
    dloss = torch.ones(n, device="cuda")
    dloss[10:14] = float("nan")
    dh, dw = P.coop_softmax_xent_grad(h, w, t, lse, dloss)
    assert status_is(-2) and not dh[10:14].any() and torch.isfinite(dh).all() and torch.isfinite(dw).all()
    h[10], h[13] = 0.0, 0.0
    dh2, dw2 = P.coop_softmax_xent_grad(h, w, t, lse, dloss)
    assert torch.equal(dh, dh2) and torch.equal(dw, dw2) and status_is(-2)
    t[:] = -1
    loss, lse = P.coop_softmax_xent(h, w, t)
    dh, dw = P.coop_softmax_xent_grad(h, w, t, lse, torch.ones(n, device="cuda"))
    assert not loss.any() and not dh.any() and not dw.any() and torch.isfinite(lse).all() and status_is(0)
    empty = h[:0]
    loss, lse = P.coop_softmax_xent(empty, w, t[:0])
    dh, dw = P.coop_softmax_xent_grad(empty, w, t[:0], lse, lse)
    assert loss.numel() == 0 and dh.shape == (0, dim) and dw.shape == w.shape and not dw.any()


@gpu
def test_softmax_xent_large_logits():
    """Logits of thousands: the maximum is subtracted before anything is raised to a power; a row of equal logits."""
    h = torch.zeros((3, 64), device="cuda")
    w = torch.zeros((1000, 64), device="cuda")
    h[0, 0], h[1, 0] = 3000.0, -3000.0
    w[:, 0] = torch.arange(1000, device="cuda") / 1000.0
    t = torch.tensor([999, 0, 5], dtype=torch.int32, device="cuda")
    loss, lse = P.coop_softmax_xent(h, w, t)
    want, want_lse, z = plain_xent(h, w, t, 1.0)
    ez, el = xent_bounds(h, w, z, want_lse, 1.0)
    within(lse, want_lse, el)
    within(loss, want, el + ez)
    assert abs(float(loss[2]) - np.log(1000)) < 1e-5


# ---- AdamW ----------------------------------------------------------------------------------------------------------------
HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1)


def plain_adamw(p, g, m, v, step, lr, beta1, beta2, eps, weight_decay):
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    hat = (m / (1 - beta1 ** step)) / (torch.sqrt(v / (1 - beta2 ** step)) + eps)
    return p * (1 - lr * weight_decay) - lr * hat, m, v, lr * hat


@gpu
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("grad_dtype", TYPES, ids=IDS)
def test_adamw_many_tensors(dtype, grad_dtype):
    g = rng(4)
    sizes = [1, 0, 2, 3, 4, 5, 63, 64, 255, 256, 257, 1000, 4096, 4097, 70001] + [17 + i for i in range(60)]
    params = [unaligned(normal(g, s, dtype=dtype)) for s in sizes]
    grads = [unaligned(normal(g, s, dtype=grad_dtype)) for s in sizes]
    copies = [torch.empty(s, dtype=torch.bfloat16, device="cuda") for s in sizes]
    old = [p.double() for p in params]
    clip = torch.tensor([0.37], device="cuda")
    opt = P.AdamW(params, grads, copies=copies)
    state = [(torch.zeros_like(p), torch.zeros_like(p)) for p in old]
    for step in (1, 2, 3):
        opt.step(step, grad_scale=clip, **HYPER)
        for i, p in enumerate(params):
            want, m, v, move = plain_adamw(old[i], grads[i].double() * clip.double(), *state[i], step, **HYPER)
            # the moments: a rounding for each product and sum, of terms that do not cancel below their own size
            em, ev = 8 * U * step * (m.abs() + grads[i].double().abs()), 8 * U * step * v
            within(opt.state["m"][i], m, em)
            within(opt.state["v"][i], v, ev)
            e = 3 * U * want.abs() + HYPER["lr"] * (em / (1 - HYPER["beta1"] ** step) / torch.sqrt(v / (1 - HYPER["beta2"] ** step)).clamp(min=1e-30)) + move.abs() * 32 * U
            within(p, want, e + want.abs() * HALF[dtype] + TINY[dtype] + U * old[i].abs())
            within(copies[i], want, e + want.abs() * 1.01 * HALF[torch.bfloat16] + U * old[i].abs() + want.abs() * HALF[dtype])
            old[i], state[i] = p.double(), (opt.state["m"][i].double(), opt.state["v"][i].double())


def decoded(opt, i, name, rows, dim):
    x = opt.state[name][i].view(rows, dim).double()
    s = opt.state[name + "_scale"][i].view(rows, -1).double()
    return x * s.repeat_interleave(256, 1)[:, :dim], s


def gap(y):
    """the distance between 8-bit floats at y"""
    return torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)


@gpu
@pytest.mark.parametrize("rows,dim,by_rows", [(1, 1, False), (1, 7, False), (1, 256, False), (1, 100003, False), (50, 100, True), (33, 75, True), (9, 1031, True), (4, 256, True)])
def test_adamw_8_bit_moments(rows, dim, by_rows):
    g = rng(rows + dim)
    p = unaligned(normal(g, rows, dim))
    grads = unaligned(normal(g, rows, dim) * torch.exp2(torch.randint(-8, 3, (rows, dim), generator=g, device="cuda").float()))
    opt = P.AdamW([p], [grads], bits=8, by_rows=by_rows)
    m, r = torch.zeros((rows, dim), dtype=torch.float64, device="cuda"), torch.zeros((rows, dim), dtype=torch.float64, device="cuda")
    shape = (rows, dim) if by_rows else (1, rows * dim)
    m, r = m.view(shape), r.view(shape)
    for step in (1, 2, 3):
        old = p.double().view(shape)
        opt.step(step, seed=77, **HYPER)
        want, m, v, move = plain_adamw(old, grads.double().view(shape), m, r * r, step, **HYPER)
        within(p.view(shape), want, 4 * U * (want.abs() + old.abs()) + 32 * U * move.abs() + 32 * U * HYPER["lr"])
        for name, x in (("m", m), ("v", torch.sqrt(v))):
            got, scale = decoded(opt, 0, name, *shape)
            blocks = torch.nn.functional.pad(x.abs(), (0, -shape[1] % 256)).view(shape[0], -1, 256)
            within(scale, blocks.amax(2) / 448, 16 * U * blocks.amax(2) / 448)
            s = scale.repeat_interleave(256, 1)[:, :shape[1]]
            y, code = x / s, got / s
            # rounded to one of the two 8-bit floats beside it
            assert ((code - y).abs() <= gap(y) * (1 + 1e-4) + 64 * U * 448).all()
            assert (torch.sign(code) * torch.sign(y) >= 0).all()
            if name == "v":
                assert ((got > 0) == (x > 0)).all()
            # with the value as the mean: a gap times a number in [-1, 1] of mean zero and variance at most a quarter each
            off = ((code - y) / gap(y))[y.abs() < 447]
            if name == "m" or y.min() > 2.0 ** -9:
                assert abs(off.sum()) <= 6 * (0.25 * off.numel()) ** 0.5 + 1
        m, r = decoded(opt, 0, "m", *shape)[0], decoded(opt, 0, "v", *shape)[0]


@gpu
def test_adamw_8_bit_many_tensors():
    """More tensors than one launch takes; the parameter follows the moments before they are rounded."""
    g = rng(14)
    sizes = [1, 0, 255, 256, 257, 3000] + [100 + 13 * i for i in range(70)]
    params, grads = [normal(g, s) for s in sizes], [normal(g, s) for s in sizes]
    opt = P.AdamW(params, grads, bits=8)
    for step in (1, 2):
        old, state = [p.double() for p in params], [(decoded(opt, i, "m", 1, s)[0][0], decoded(opt, i, "v", 1, s)[0][0]) if s else None for i, s in enumerate(sizes)]
        opt.step(step, seed=3, **HYPER)
        for i, s in enumerate(sizes):
            if s == 0:
                continue
            want, m, v, move = plain_adamw(old[i], grads[i].double(), state[i][0], state[i][1] ** 2, step, **HYPER)
            within(params[i], want, 4 * U * (want.abs() + old[i].abs()) + 32 * U * move.abs() + 32 * U * HYPER["lr"])
            for name, x in (("m", m), ("v", torch.sqrt(v))):
                got, scale = decoded(opt, i, name, 1, s)
                scale = scale.repeat_interleave(256, 1)[0, :s]
                assert ((got[0] / scale - x / scale).abs() <= gap(x / scale) * (1 + 1e-4) + 64 * U * 448).all()


@gpu
def test_adamw_8_bit_is_a_function_of_its_arguments():
    g = rng(8)
    p, grad = normal(g, 5000), normal(g, 5000)
    runs = {}
    for name, seed in (("a", 1), ("again", 1), ("b", 2)):
        q = p.clone()
        opt = P.AdamW([q], [grad], bits=8)
        for step in (1, 2):
            opt.step(step, seed=seed, **HYPER)
        runs[name] = (q, opt.state["m"][0].float(), opt.state["v"][0].float())
    assert all(torch.equal(x, y) for x, y in zip(runs["a"], runs["again"]))
    assert not torch.equal(runs["a"][1], runs["b"][1]) and not torch.equal(runs["a"][2], runs["b"][2])


@gpu
@pytest.mark.parametrize("bits", [8, 32])
def test_adamw_decays_and_follows_in_8_bits(bits):
    """A gradient that stops: the moments fade, the parameter does not run away.  One that grows: v follows it."""
    p, grad = torch.zeros(4096, device="cuda"), torch.ones(4096, device="cuda")
    opt = P.AdamW([p], [grad], bits=bits)
    value = lambda x: (opt.state[x][0].float() * (opt.state[x + "_scale"][0].repeat_interleave(256) if bits == 8 else 1)).double()  # noqa: E731
    hyper = dict(HYPER, weight_decay=0.0)
    for step in range(1, 201):
        if step == 101:
            grad.fill_(3.0)
        opt.step(step, seed=5, **hyper)
        if step in (100, 200):
            v = value("v") if bits == 32 else value("v") ** 2
            want = 1 - 0.99 ** 100 if step == 100 else 9 * (1 - 0.99 ** 100) + (1 - 0.99 ** 100) * 0.99 ** 100
            assert abs(float(v.mean()) / want - 1) < 0.1
    before = p.clone()
    grad.zero_()
    for step in range(201, 601):
        opt.step(step, seed=5, **hyper)
    assert float((value("m").abs()).max()) < 1e-3 and float((p - before).abs().max()) < 0.2


@gpu
@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("n_rows,dim,k", [(1, 1, 1), (40, 100, 13), (1000, 300, 999), (100, 64, 0), (70, 3, 70)])
def test_adamw_touched_rows(bits, n_rows, dim, k):
    """The listed rows change as all would, no other row is written, and the count on the device decides how many are listed."""
    g = rng(n_rows + dim)
    table = normal(g, n_rows, dim)
    full, part = table.clone(), table.clone()
    rows = torch.randperm(n_rows, generator=g, device="cuda")[:k].sort().values.to(torch.int32)
    grad = normal(g, k, dim)
    dense = torch.zeros((n_rows, dim), device="cuda")
    dense[rows.long()] = grad
    a, b = P.AdamW([full], [dense], bits=bits, by_rows=True), P.AdamW([part], bits=bits, by_rows=True)
    more = torch.cat([rows, torch.full((3,), -9, dtype=torch.int32, device="cuda")])
    more_grad = torch.cat([grad, torch.ones((3, dim), device="cuda")])
    count = torch.tensor([k], dtype=torch.int32, device="cuda")
    for step in (1, 2):
        a.step(step, seed=3, **HYPER)
        b.step(step, seed=3, rows={0: (rows, grad, None)} if step == 1 else {0: (more, more_grad, count)}, **HYPER)
    at = rows.long()
    assert torch.equal(part[at], full[at]) and status_is(0)
    rest = torch.ones(n_rows, dtype=torch.bool, device="cuda")
    rest[at] = False
    assert torch.equal(part[rest], table[rest])
    for x in a.state:
        s, t = (o.state[x][0].view(n_rows, -1).float() for o in (a, b))
        assert torch.equal(s[at], t[at]) and not t[rest].any()
    b.step(3, rows={0: (torch.tensor([n_rows, -1], dtype=torch.int32, device="cuda"), torch.ones((2, dim), device="cuda"), None)}, **HYPER)
    assert status_is(-2) and torch.equal(part[rest], table[rest])


@gpu
@pytest.mark.parametrize("bits", [8, 32])
def test_adamw_not_finite(bits):
    p, grad = torch.ones(1000, device="cuda"), torch.ones(1000, device="cuda")
    grad[300] = float("nan")
    opt = P.AdamW([p], [grad], bits=bits)
    opt.step(1, **HYPER)
    assert torch.isnan(p[300]) and torch.isfinite(p[:256]).all() and torch.isfinite(torch.cat([p[256:300], p[301:]])).all()
    opt.step(2, **HYPER)
    alone = torch.isnan(p)
    assert alone[300] and not alone[:256].any() and not alone[512:].any() and (bits == 8 or alone.sum() == 1)


# ---- streams and graphs ------------------------------------------------------------------------------------------------------
def everything(table, ids, w, t, x, gamma, opt, dloss, step, stream=None):
    h = P.coop_embed(table, ids, alpha=2.0, stream=stream)
    y, mean, rstd = P.coop_layer_norm(h, gamma, stream=stream)
    loss, lse = P.coop_softmax_xent(y, w, t, stream=stream)
    dy, dw = P.coop_softmax_xent_grad(y, w, t, lse, dloss, stream=stream)
    dx, dgamma, dbeta = P.coop_layer_norm_grad(dy, h, mean, rstd, gamma, stream=stream)
    rows = P.coop_embed_grad_rows(dx, ids, table.shape[0], alpha=2.0, wait=False, stream=stream)
    dense = P.coop_embed_grad(dx, ids, table.shape[0], alpha=2.0, stream=stream)
    opt.step(step, rows={0: rows}, stream=stream, **HYPER)
    return loss, lse, dy, dw, dx, dgamma, dbeta, dense


def inputs(seed):
    g = rng(seed)
    table = normal(g, 3000, 72)
    ids = ID_SETS["hub"](g, 4500, 3000).to(torch.int32)
    w = normal(g, 700, 72, scale=0.3)
    t = torch.randint(-1, 700, (4500,), generator=g, device="cuda", dtype=torch.int32)
    return table, ids, w, t, None, 1 + normal(g, 72, scale=0.1), P.AdamW([table], bits=8, by_rows=True), torch.rand(4500, generator=g, device="cuda")


@gpu
def test_same_bits_on_another_stream_and_in_a_graph():
    a = inputs(1)
    want = everything(*a, 1)
    b = inputs(1)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = everything(*b, 1, stream=side)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, got)) and torch.equal(a[0], b[0])
    # captured once, replayed several times between other work: each replay is the next step of the same arguments
    c, d = inputs(1), inputs(1)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        everything(*inputs(1), 1)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = everything(*c, 1)
    for _ in range(4):
        graph.replay()
        torch.cuda.synchronize()
        want = everything(*d, 1)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(want, out)) and torch.equal(c[0], d[0])
        torch.ones(1 << 20, device="cuda").sum()
    assert status_is(0)


@gpu
def test_workspaces_are_the_callers():
    """A workspace that is given is used as it comes, whatever it holds."""
    g = rng(6)
    ids = ID_SETS["hub"](g, 5000, 900).to(torch.int32)
    dout = normal(g, 5000, 24)
    L = learn.lib()
    want = P.coop_embed_grad(dout, ids, 900)
    ws = torch.full((L.coop_embed_grad_workspace_bytes(5000, 24),), 255, dtype=torch.uint8, device="cuda")
    assert torch.equal(P.coop_embed_grad(dout, ids, 900, workspace=ws), want)
    h, w = normal(g, 100, 40, dtype=torch.float16), normal(g, 500, 40, dtype=torch.float16)
    t = torch.randint(0, 500, (100,), generator=g, device="cuda", dtype=torch.int32)
    loss, lse = P.coop_softmax_xent(h, w, t)
    ws = torch.full((L.coop_softmax_xent_workspace_bytes(100, 500, 40, P.COOP_F16, 1, 1),), 255, dtype=torch.uint8, device="cuda")
    again = P.coop_softmax_xent(h, w, t, workspace=ws)
    assert torch.equal(again[0], loss) and torch.equal(again[1], lse)
    want = P.coop_softmax_xent_grad(h, w, t, lse, loss)
    ws.fill_(255)
    assert all(torch.equal(x, y) for x, y in zip(want, P.coop_softmax_xent_grad(h, w, t, lse, loss, workspace=ws)))
    with pytest.raises(P.CoopError):
        P.coop_softmax_xent_grad(h, w, t, lse, loss, workspace=ws[:1024])


# ---- offsets beyond 32 bits -----------------------------------------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("n,dim,dtype", [(40, 128, torch.bfloat16), (40, 136, torch.float16), (3, 136, torch.bfloat16)])
def test_softmax_xent_offsets_beyond_32_bits(n, dim, dtype):
    torch.cuda.empty_cache()
    check_xent(dtype, n, 17000001, dim, 0.8)                     # 4.3 GB of weight, and of its gradient


@gpu
def test_layer_norm_offsets_beyond_32_bits():
    torch.cuda.empty_cache()
    rows, dim, k = 70001, 32768, 7                               # 2.3e9 elements
    g = rng(21)
    x, dy = (torch.zeros((rows, dim), dtype=torch.float16, device="cuda") for _ in range(2))
    x[-k:], dy[-k:] = normal(g, k, dim, dtype=torch.float16), normal(g, k, dim, dtype=torch.float16)
    y, mean, rstd = P.coop_layer_norm(x)
    few, few_mean, few_rstd = P.coop_layer_norm(x[-k:].contiguous())
    assert torch.equal(y[-k:], few) and torch.equal(mean[-k:], few_mean) and torch.equal(rstd[-k:], few_rstd) and not y[:-k].any()
    dx, dw, db = P.coop_layer_norm_grad(dy, x, mean, rstd)
    few, few_dw, few_db = P.coop_layer_norm_grad(dy[-k:].contiguous(), x[-k:].contiguous(), few_mean, few_rstd)
    assert torch.equal(dx[-k:], few) and not dx[:-k].any()
    # sums of 7 numbers, in another order
    size = (dy[-k:].double().abs() * (1 + y[-k:].double().abs())).sum(0) * 16 * U
    within(dw, few_dw, size)
    within(db, few_db, size)


@gpu
@pytest.mark.parametrize("bits", [8, 32])
def test_adamw_offsets_beyond_32_bits(bits):
    torch.cuda.empty_cache()
    n = 2 ** 31 + 4099
    spots = [slice(0, 2048), slice(2 ** 31 - 1024, 2 ** 31 + 1024), slice(n - 1027, n)]
    p, grad = torch.ones(n, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g = rng(22)
    for s in spots:
        grad[s] = normal(g, s.stop - s.start, dtype=torch.bfloat16)
    opt = P.AdamW([p], [grad], bits=bits)
    opt.step(1, **HYPER)
    for s in spots:
        want, m, v, move = plain_adamw(torch.ones(s.stop - s.start, dtype=torch.float64, device="cuda"), grad[s].double(), 0.0, 0.0, 1, **HYPER)
        within(p[s], want, 64 * U + want.abs() * HALF[torch.bfloat16])
        if bits == 32:
            within(opt.state["m"][0][s], m, 8 * U * m.abs())
            within(opt.state["v"][0][s], v, 8 * U * v)
        else:
            got = opt.state["m"][0][s].float() * opt.state["m_scale"][0][s.start // 256:-(-s.stop // 256)].repeat_interleave(256)[:s.stop - s.start]
            within(got, m, m.abs() * 2.0 ** -3 * 1.01 + opt.state["m_scale"][0].max() * 2.0 ** -9 * 1.01)
    del p, grad, opt
    table = torch.zeros((60000, 40000), dtype=torch.bfloat16, device="cuda")
    rows = torch.tensor([0, 53687, 53688, 59999], dtype=torch.int32, device="cuda")
    opt = P.AdamW([table], bits=bits, by_rows=True)
    grads = normal(g, 4, 40000)
    opt.step(1, rows={0: (rows, grads, None)}, **HYPER)
    want = plain_adamw(torch.zeros_like(grads.double()), grads.double(), 0.0, 0.0, 1, **HYPER)[0]
    within(table[rows.long()], want, 64 * U * HYPER["lr"] + want.abs() * HALF[torch.bfloat16])
    assert int((table != 0).any(1).sum()) == 4


# ---- together ----------------------------------------------------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("bits,dim", [(8, 128), (32, 75)])
def test_vertex_embeddings_learn(bits, dim):
    """Trained rows tell a neighbour better than the neighbours' frequencies do halfway from none to all of their information."""
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "vertex_embeddings.py")
    spec = importlib.util.spec_from_file_location("vertex_embeddings", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    indptr, indices = synth.rmat_csr(scale=12, n_edges=65536)
    model, losses = example.train(indptr, indices, dim=dim, batch=512, steps=120, bits=bits, log=None)
    degrees = np.diff(indptr.numpy())                             # a vertex's neighbours are drawn min(10, degree) at a time
    share = np.bincount(indices.numpy(), np.repeat(np.minimum(10, degrees) / np.maximum(degrees, 1), degrees), 4096)
    share /= share.sum()
    entropy = -(share[share > 0] * np.log(share[share > 0])).sum()
    assert abs(losses[0] - np.log(4096)) < 1e-4                  # output weights of zero: all vertices alike
    assert np.mean(losses[-10:]) < (np.log(4096) + entropy) / 2
    assert torch.equal(model.out16, model.out.to(torch.bfloat16))
    _, again = example.train(indptr, indices, dim=dim, batch=512, steps=120, bits=bits, log=None)
    assert again == losses                                       # the same bits on every run


# ---- refusals ----------------------------------------------------------------------------------------------------------------
def test_refusals_of_the_c_abi():
    """What the host can see is refused before anything is launched."""
    L = learn.lib()
    A, N = 0x1000, None
    assert L.coop_embed(A, 10, 4, 3, A, 5, N, 1.0, 0, A, 0, N) == -4            # unknown dtype
    assert L.coop_embed(A, 10, 4, 0, A, 5, N, 1.0, 0, A, 9, N) == -4
    assert L.coop_embed(A, 10, 0, 0, A, 5, N, 1.0, 0, A, 0, N) == -4            # dim < 1
    assert L.coop_embed(A, 0, 4, 0, A, 5, N, 1.0, 0, A, 0, N) == -4             # ids, but no rows
    assert L.coop_embed(N, 10, 4, 0, A, 5, N, 1.0, 0, A, 0, N) == -1
    assert L.coop_embed(A + 2, 10, 4, 0, A, 5, N, 1.0, 0, A, 0, N) == -4        # fp32 on a 2-byte boundary
    assert L.coop_embed(N, 10, 4, 0, N, 0, N, 1.0, 0, N, 0, N) == 0             # nothing to do
    need = L.coop_embed_grad_workspace_bytes(100, 8)
    assert need > 0 and L.coop_embed_grad_workspace_bytes(-1, 8) == 0 and L.coop_embed_grad_workspace_bytes(1 << 31, 8) == 0
    assert L.coop_embed_grad(A, 0, A, 100, N, 1.0, 0, 10, 8, A, 0, A, need - 1, N) == -4       # workspace too small
    assert L.coop_embed_grad(A, 0, A, 100, N, 1.0, 0, 10, 8, A, 0, A + 8, need, N) == -4       # or not aligned
    assert L.coop_embed_grad(A, 0, A, 100, N, 1.0, 0, 1 << 31, 8, A, 0, A, need, N) == -4
    assert L.coop_embed_grad(A, 0, A, 100, N, 1.0, 0, 10, 8, A, 0, N, need, N) == -1
    assert L.coop_embed_grad_rows(A, 0, A, 100, N, 1.0, 0, 10, 8, A, A, 0, N, A, need, N) == -1  # no place for the count
    assert L.coop_layer_norm(A, 5, 0, 0, N, N, 0, 1e-5, A, A, A, N) == -4
    assert L.coop_layer_norm(A, 5, 8, 0, A, N, 1, 1e-5, A, A, A, N) == -4                      # fp16 weights of fp32 rows
    assert L.coop_layer_norm(A, 5, 40000, 0, N, N, 0, 1e-5, A, A, A, N) == -4                  # wider than is supported
    assert L.coop_layer_norm(A, 5, 8, 0, N, N, 0, -1.0, A, A, A, N) == -4
    assert L.coop_layer_norm(A, 5, 8, 0, N, N, 0, 1e-5, A, N, A, N) == -1
    assert L.coop_layer_norm(N, 0, 8, 0, N, N, 0, 1e-5, N, N, N, N) == 0
    assert L.coop_layer_norm_grad(A, A, 5, 8, 0, A, A, N, 0, A, A, N, N, 0, N) == -1           # a weight's gradient, no workspace
    assert L.coop_layer_norm_grad(A, A, 5, 8, 0, A, A, N, 0, A, A, N, A, 8, N) == -4
    need = L.coop_softmax_xent_workspace_bytes(10, 100, 8, 2, 1, 1)
    assert need > 0 and L.coop_softmax_xent_workspace_bytes(10, 0, 8, 2, 1, 1) == 0 and L.coop_softmax_xent_workspace_bytes(10, 100, 8, 5, 1, 1) == 0
    assert L.coop_softmax_xent(A, 10, A, 0, 8, 2, A, 1.0, -1, A, A, A, need, N) == -4          # no vocabulary
    assert L.coop_softmax_xent(A, 10, A, 100, 8, 2, N, 1.0, -1, A, A, A, need, N) == -1
    assert L.coop_softmax_xent(A, 10, A, 100, 8, 2, A, 1.0, -1, A, A, A, 16, N) == -4
    assert L.coop_softmax_xent(A, 1 << 24, A, 100, 8, 2, A, 1.0, -1, A, A, A, need, N) == -4
    assert L.coop_softmax_xent_grad(A, 10, A, 100, 8, 2, A, 1.0, -1, N, A, A, A, A, need, N) == -1
    assert L.coop_softmax_xent_grad(A, 10, A, 100, 8, 2, A, 1.0, -1, A, A, A, A, A, need - 1, N) == -4
    assert L.coop_softmax_xent_grad(A, 10, A, 100, 8, 2, A, 1.0, -1, A, A, N, N, A, need, N) == 0   # nothing asked for
    t = (learn._CAdamWTensor * 1)()
    call = lambda bits=32, step=1, b1=0.9, n=1, ts=t: L.coop_adamw(ts, n, bits, 1e-3, b1, 0.99, 1e-8, 0.0, step, 0, N, N)  # noqa: E731
    assert call(n=0) == 0 and call(bits=16) == -4 and call(step=0) == -4 and call(b1=1.0) == -4 and call(ts=None) == -1
    t[0].n_rows, t[0].dim, t[0].param, t[0].grad, t[0].m, t[0].v = 1, 8, A, A, A, A
    assert call(bits=8) == -1                                                                  # 8 bits without scales
    t[0].param_dtype = 5
    assert call() == -4
    t[0].param_dtype, t[0].n_list_dev = 0, A
    assert call() == -4                                                                        # a count without a list
    t[0].n_list_dev, t[0].m = None, A + 1
    assert call() == -4
    t[0].m, t[0].n_rows, t[0].dim = A, 1 << 30, 1 << 40
    assert call() == -4


@gpu
def test_refusals_of_the_binding():
    x = torch.zeros((8, 6), device="cuda")
    ids = torch.zeros(8, dtype=torch.int32, device="cuda")
    for call in (lambda: P.coop_embed(x[:, ::2], ids), lambda: P.coop_embed(x, ids.long()), lambda: P.coop_embed(x.double(), ids),
                 lambda: P.coop_embed(x, ids, scale=torch.zeros(7, device="cuda")), lambda: P.coop_embed_grad(x[:7], ids, 5),
                 lambda: P.coop_embed_grad_rows(x, ids.cpu(), 5), lambda: P.coop_layer_norm(x, torch.zeros(5, device="cuda")),
                 lambda: P.coop_layer_norm(x, torch.zeros(6, device="cuda"), torch.zeros(6, device="cuda").half()),
                 lambda: P.coop_layer_norm_grad(x.half(), x, x[:, 0].clone(), x[:, 0].clone()),
                 lambda: P.coop_softmax_xent(x, x[:, :4].contiguous(), ids), lambda: P.coop_softmax_xent(x, x.half(), ids),
                 lambda: P.coop_softmax_xent(x, x, ids[:3]), lambda: P.coop_softmax_xent_grad(x, x, ids, x[0], x[0]),
                 lambda: P.AdamW([x], [x[:4]]), lambda: P.AdamW([x[0, 0]], bits=4), lambda: P.AdamW([x]).step(1, 1e-3),
                 lambda: P.AdamW([x], bits=8).step(1, 1e-3, rows={0: (ids[:2], x[:2], None)}),
                 lambda: P.AdamW([x], by_rows=True).step(1, 1e-3, rows={0: (ids[:2], x[:3], None)})):
        with pytest.raises(AssertionError):
            call()
    with pytest.raises(P.CoopError) as e:
        P.coop_layer_norm(torch.zeros((1, 40000), device="cuda"))
    assert e.value.code == -4
    with pytest.raises(P.CoopError):
        P.AdamW([x], [x.clone()]).step(0, 1e-3)


class OnDevice:
    """A tensor of the host that says it is the device's: what a refusal leaves behind can be looked at without a GPU."""

    def __init__(self, t):
        self.t, self.is_cuda = t, True

    def __getattr__(self, name):
        return getattr(self.t, name)


def host_adamw(params, bits=32, **kw):
    n = [p.numel() for p in params]
    state = {"m": [OnDevice(torch.zeros(k)) for k in n], "v": [OnDevice(torch.zeros(k)) for k in n]}
    return P.AdamW([OnDevice(p) for p in params], bits=bits, state=state, **kw)


def test_a_refused_step_leaves_the_plan_as_it_was():
    """Whatever is wrong with a step's rows, the next step's tensors, addresses and sizes are those of before."""
    x, y = torch.zeros((8, 6)), torch.zeros((5, 4))
    opt = host_adamw([x, y], grads=[OnDevice(torch.zeros((8, 6))), OnDevice(torch.zeros((5, 4)))], by_rows=True)
    before = bytes(opt._c)
    ids, g = OnDevice(torch.zeros(2, dtype=torch.int32)), OnDevice(torch.zeros((2, 6)))
    g4, count = OnDevice(torch.zeros((2, 4))), OnDevice(torch.zeros(1, dtype=torch.int32))
    wide = OnDevice(torch.zeros(2, dtype=torch.int64))
    for rows, kw in (({0: (wide, g, None)}, {}), ({0: (ids, g4, None)}, {}), ({0: (ids, g, wide)}, {}), ({0: (ids, g, count), 1: (ids, g, None)}, {}),
                     ({0: (ids, g, count), 1: (wide, g4, None)}, {}), ({0: (ids, g, None)}, {"grad_scale": wide}), ({0: (ids, g, None)}, {"grad_scale": ids})):
        with pytest.raises(AssertionError):
            opt.step(1, 1e-3, rows=rows, **kw)
        assert bytes(opt._c) == before
    with pytest.raises(P.CoopError):         # (by the library, before it launches anything)
        opt.step(0, 1e-3, rows={0: (ids, g, count), 1: (ids, g4, None)}, stream=types.SimpleNamespace(cuda_stream=None))
    assert bytes(opt._c) == before


def test_refused_gradients_leave_the_ones_that_are_kept():
    """set_grads takes all of its gradients or none: the plan's addresses are those of the tensors that the optimizer keeps."""
    x, y = torch.zeros((8, 6)), torch.zeros((5, 4))
    kept = [OnDevice(torch.zeros((8, 6))), OnDevice(torch.zeros((5, 4)))]
    opt = host_adamw([x, y], grads=kept)
    before = bytes(opt._c)
    for bad in (torch.zeros((5, 5)), torch.zeros((5, 4), dtype=torch.float64), torch.zeros((4, 5)).t()):
        with pytest.raises(AssertionError):
            opt.set_grads([OnDevice(torch.zeros((8, 6))), OnDevice(bad)])
        assert bytes(opt._c) == before and all(a is b for a, b in zip(opt.grads, kept))
    opt.set_grads([None, kept[1]])
    assert opt._c[0].grad is None and opt._c[1].grad == kept[1].data_ptr()


def test_the_memory_that_the_plan_points_to_stays():
    """... when a parameter gets other memory (as .data = does) and the moments are replaced in their lists."""
    class Memory(np.ndarray):
        pass
    arrays = [np.zeros((8, 6), dtype=np.float32).view(Memory) for _ in range(4)]
    p, copy, m, v = (OnDevice(torch.from_numpy(a)) for a in arrays)
    opt = P.AdamW([p], copies=[copy], state={"m": [m], "v": [v]})
    alive = [weakref.ref(a) for a in arrays]
    p.t.data = torch.zeros((8, 6))
    opt.state["m"][0] = opt.state["v"][0] = opt.copies[0] = None
    del arrays, p, copy, m, v
    gc.collect()
    assert all(a() is not None for a in alive)
    del opt
    gc.collect()
    assert not any(a() is not None for a in alive)


def test_adamw_most_rows():
    """A tensor has at most 2^27 blocks of 256 elements of a row, short rows being less than one.  (A second tensor without addresses:
    what is let through is refused as well, by another name, and nothing is launched.)"""
    L, A = learn.lib(), 0x1000
    t = (learn._CAdamWTensor * 2)()
    t[1].n_rows, t[1].dim = 1, 1
    for x in ("param", "grad", "m", "v", "m_scale", "v_scale"):
        setattr(t[0], x, A)
    for bits in (8, 32):
        for dim, most in ((1, 1 << 30), (32, 1 << 30), (33, 1 << 29), (64, 1 << 29), (65, 1 << 28), (128, 1 << 28), (129, 1 << 27), (256, 1 << 27),
                          (257, 1 << 26), (100000, (1 << 27) // 391), (1 << 35, 1)):
            for rows, code in ((most, -1), (most + 1, -4)):
                for listed in (None, A):
                    t[0].dim, t[0].n_rows, t[0].n_list, t[0].rows = dim, (1 << 31) - 1 if listed and dim < 1 << 20 else rows, rows if listed else 0, listed
                    assert L.coop_adamw(t, 2, bits, 1e-3, 0.9, 0.99, 1e-8, 0.0, 1, 0, None, None) == code, (dim, rows, listed)
    t[0].rows, t[0].n_list, t[0].n_rows, t[0].dim = None, 0, 1, (1 << 35) + 1
    assert L.coop_adamw(t, 2, 32, 1e-3, 0.9, 0.99, 1e-8, 0.0, 1, 0, None, None) == -4


@gpu
@pytest.mark.parametrize("bits", [8, 32])
def test_adamw_more_short_rows_than_whole_blocks(bits):
    """More than 2^27 rows, eight to a wave: those at either end and around 2^27 change as they would alone."""
    torch.cuda.empty_cache()
    n, dim = 2 ** 27 + 2 ** 20 + 5, 8
    spots = [slice(0, 300), slice(2 ** 27 - 150, 2 ** 27 + 150), slice(n - 300, n)]
    g = rng(23)
    p, grad = torch.ones((n, dim), dtype=torch.bfloat16, device="cuda"), torch.zeros((n, dim), dtype=torch.bfloat16, device="cuda")
    for s in spots:
        grad[s] = normal(g, s.stop - s.start, dim, dtype=torch.bfloat16)
    opt = P.AdamW([p], [grad], bits=bits, by_rows=True)
    opt.step(1, **HYPER)
    for s in spots:
        want, m, v, move = plain_adamw(torch.ones((s.stop - s.start, dim), dtype=torch.float64, device="cuda"), grad[s].double(), 0.0, 0.0, 1, **HYPER)
        within(p[s], want, 64 * U + want.abs() * HALF[torch.bfloat16])
        got = opt.state["m"][0].view(n, dim)[s].float()
        if bits == 32:
            within(got, m, 8 * U * m.abs())
        else:
            scale = opt.state["m_scale"][0][s].double()
            within(scale, m.abs().amax(1) / 448, 16 * U * m.abs().amax(1) / 448)
            within(got * scale[:, None], m, m.abs() * 2.0 ** -3 * 1.01 + scale[:, None] * 2.0 ** -9 * 1.01)
    still = torch.cat([p[300:2 ** 20], p[2 ** 27 + 150:2 ** 27 + 2 ** 20 - 300]])
    assert bool((still == still[0, 0]).all()) and not bool(opt.state["m"][0].view(torch.uint8).view(n, -1)[300:2 ** 20].any())


# rows that stay in registers; few rows; tiles of 128; tiles of 256; a vocabulary in three pieces
@gpu
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("n,vocab,dim", [(24, 20000, 120), (300, 20000, 128), (24, 20000, 136), (300, 20000, 136), (4097, 4100, 200), (16384, 20000, 136)])
def test_softmax_xent_grad_of_rows_that_count_little(dtype, n, vocab, dim):
    """A row's gradient is as exact as its own dloss allows, however much larger another row's is: the bound is the row's own."""
    g = rng(n + dim)
    h, w = normal(g, n, dim, dtype=dtype), normal(g, vocab, dim, dtype=dtype, scale=2 * dim ** -0.5)
    t = torch.randint(0, vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
    # dloss from 2^11 down to 2^-11 (what fp16 holds both gradients of), and a row of none
    dloss = torch.exp2(11.0 - 22.0 * torch.rand(n, generator=g, device="cuda")) * torch.where(torch.rand(n, generator=g, device="cuda") < 0.5, -1.0, 1.0)
    dloss[0], dloss[1] = 2.0 ** 11, 0.0
    _, lse = P.coop_softmax_xent(h, w, t)
    dh, dw = P.coop_softmax_xent_grad(h, w, t, lse, dloss)
    z = h.double() @ w.double().t()
    ez, _ = xent_bounds(h, w, z, lse.double(), 1.0)
    c = dloss.double()
    off = 4 * U * (lse.double().abs() + z.abs().amax(1)) + 4 * U
    G = torch.exp(z.sub_(lse.double()[:, None]))
    ep = G * (ez + off)[:, None]
    G.scatter_add_(1, t.long()[:, None], torch.full((n, 1), -1.0, dtype=torch.float64, device="cuda"))
    # G's rounding, relative to the row: 2^-25 of 2^13 times what the row's coefficient is lifted to, at least 2^-10 of the largest
    eG = ep + (G.abs() + ep) * (HALF[dtype] + 4 * U) + (2.0 ** -28 if dtype == torch.float16 else 0.0)
    W = w.double()
    e = eG @ W.abs()
    e += (vocab + 272) * U * (G.abs() @ W.abs() + e)
    want = (G @ W) * c[:, None]
    e *= c.abs()[:, None]
    within(dh, want, e + (want.abs() + e) * HALF[dtype] + TINY[dtype])
    # dW's sums over the rows have one scale: that of the largest coefficient
    eG = eG * c.abs()[:, None]
    if dtype == torch.float16:
        eG = eG + 1.5 * c.abs().max() * 2.0 ** -38
    G = G * c[:, None]
    H = h.double()
    want, e, size = G.t().contiguous() @ H, eG.t().contiguous() @ H.abs(), G.abs().t().contiguous() @ H.abs()
    e += (n + 272) * U * (size + e)
    within(dw, want, e + (want.abs() + e) * HALF[dtype] + TINY[dtype])
    assert bool(torch.isfinite(dh).all()) and not dh[1].any()
    assert torch.equal(P.coop_softmax_xent_grad(h, w, t, lse, dloss, want_weight=False)[0], dh)
    assert torch.equal(P.coop_softmax_xent_grad(h, w, t, lse, dloss, want_hidden=False)[1], dw)


@gpu
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("n,dim", [(60, 72), (60, 136), (20, 136)])
def test_softmax_xent_grad_along_the_gradient(dtype, n, dim):
    """The loss' slope along the gradient's own direction, where it is the gradient's length: by differences in 64 bits, and by what came
    back, whose errors are bounded element by element and together are less than a fiftieth of the slope."""
    g = rng(dim + n)
    vocab, step = 700, 1e-4
    h, w = normal(g, n, dim, dtype=dtype), normal(g, vocab, dim, dtype=dtype, scale=0.2)
    t = torch.randint(-1, vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
    dloss = torch.rand(n, generator=g, device="cuda") + 0.5
    loss, lse = P.coop_softmax_xent(h, w, t)
    grads = P.coop_softmax_xent_grad(h, w, t, lse, dloss)
    _, want_lse, z = plain_xent(h, w, t, 1.0)
    ez, el = xent_bounds(h, w, z, want_lse, 1.0)
    H, W, c = h.double(), w.double(), torch.where(t >= 0, dloss.double(), 0.0)
    p = torch.exp(z - want_lse[:, None])
    G = p.scatter_add(1, t.long().clamp(min=0)[:, None], torch.full((n, 1), -1.0, dtype=torch.float64, device="cuda")) * c[:, None]
    ep = p * ((ez + el + 4 * U * (want_lse.abs() + z.abs().amax(1)) + 4 * U) * c)[:, None]
    eG = ep + (G.abs() + ep) * (HALF[dtype] + 4 * U) + (c.max() * 2.0 ** -38 if dtype == torch.float16 else 0.0)
    for k, (want, e, size, terms) in enumerate(((G @ W, eG @ W.abs(), G.abs() @ W.abs(), vocab),
                                                (G.t().contiguous() @ H, eG.t().contiguous() @ H.abs(), G.abs().t().contiguous() @ H.abs(), n))):
        e = e + (terms + 272) * U * (size + e)
        e = e + (want.abs() + e) * HALF[dtype] + TINY[dtype]
        way = want / want.norm()
        losses = []
        for sign in (1, -1):
            args = [H, W]
            args[k] = args[k] + sign * step * way
            losses.append((plain_xent(*args, t, 1.0)[0] * dloss.double()).sum())
        slope, got, bound = (losses[0] - losses[1]) / (2 * step), (grads[k].double() * way).sum(), (e * way.abs()).sum()
        assert float(slope) > 0 and float(bound) < float(slope) / 50
        assert abs(float(got - slope)) <= float(bound) + 1e-6 * float(slope)       # (the differences: step^2 of the third derivative)


@gpu
def test_the_least_id_is_reported_where_there_is_no_padding():
    """COOP_NO_PAD is the least int32, which as an id is as wrong as any other negative one."""
    least = torch.full((600,), -2 ** 31, dtype=torch.int32, device="cuda")
    least[5] = 3
    table, x = torch.ones((10, 8), device="cuda"), torch.ones((600, 8), device="cuda")
    for ids in (least[4:6].contiguous(), least):                 # (the sort of few tokens, and of more)
        for call in (lambda: P.coop_embed(table, ids), lambda: P.coop_embed_grad(x[:ids.numel()], ids, 10),
                     lambda: P.coop_embed_grad_rows(x[:ids.numel()], ids, 10)[1]):
            assert float(call().sum()) == 8 and status_is(-2) and status_is(0)
        assert float(P.coop_embed(table, ids, pad=-1).sum()) == 8 and status_is(-2)
    least[:5] = least[6:] = -1
    assert float(P.coop_embed(table, least, pad=-1).sum()) == 8 and status_is(0)


def test_embed_grad_widest_rows_refused():
    """As many column tiles as a grid has rows, and no more: refused before anything is launched.  (Without tokens: what is let through is
    refused as well, by another name.)"""
    L, A, most = learn.lib(), 0x1000, 16776960
    assert L.coop_embed_grad_workspace_bytes(100, most) > 0 and L.coop_embed_grad_workspace_bytes(100, most + 1) == 0
    for dim, code in ((most, -1), (most + 1, -4), (2 ** 31 - 1, -4)):
        assert L.coop_embed_grad(None, 0, A, 100, None, 1.0, 0, 10, dim, A, 0, A, 1 << 40, None) == code
        assert L.coop_embed_grad_rows(None, 0, A, 100, None, 1.0, 0, 10, dim, A, A, 0, A, A, 1 << 40, None) == code


@gpu
def test_embed_widest_rows():
    torch.cuda.empty_cache()
    dim, ids = 16776960, torch.tensor([2, 0, 2], dtype=torch.int32, device="cuda")
    dout = torch.arange(dim, device="cuda").remainder(1000).float() * torch.tensor([[1.0], [2.0], [3.0]], device="cuda")
    grad = P.coop_embed_grad(dout, ids, 3)
    assert torch.equal(grad[0], dout[1]) and not grad[1].any() and torch.equal(grad[2], dout[0] * 4)
    del dout, grad
    dim = 2 ** 31 - 5                          # 4.3 GB, the last items' numbers close to 2^31
    table = torch.zeros((1, dim), dtype=torch.float16, device="cuda")
    table[0, ::1001] = 1.0
    table[0, -1] = 2.0
    assert torch.equal(P.coop_embed(table, torch.zeros(1, dtype=torch.int32, device="cuda")), table) and status_is(0)


@gpu
@pytest.mark.parametrize("rows,dim", [(5000, 3), (3000, 75), (2500, 100), (2100, 602), (1100, 1500), (700, 8191), (300, 20001), (550, 32768)])
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_layer_norm_in_place(rows, dim, dtype):
    """y in the place of x, dx in that of dy: the same bits, in every layout of a row, with more rows than groups that share them."""
    g = rng(dim)
    x, dy, w, b = normal(g, rows, dim, dtype=dtype), normal(g, rows, dim, dtype=dtype), 1 + normal(g, dim, scale=0.2), normal(g, dim)
    y, mean, rstd = P.coop_layer_norm(x, w, b)
    dx, dw, db = P.coop_layer_norm_grad(dy, x, mean, rstd, w)
    got, dgot = unaligned(x), unaligned(dy)
    assert all(torch.equal(s, t) for s, t in zip(P.coop_layer_norm(got, w, b, out=got), (y, mean, rstd)))
    assert all(torch.equal(s, t) for s, t in zip(P.coop_layer_norm_grad(dgot, x, mean, rstd, w, out=dgot), (dx, dw, db)))


def test_softmax_xent_grad_workspace_is_what_is_said():
    """... of its size, in coop.h: over rows, vocabularies, widths and types, the sum of what it is said to hold is enough and not far more."""
    L, MB = learn.lib(), 1 << 20
    for n in (1, 24, 32, 33, 300, 4096, 8192, 100000, 500000, 1000000, (1 << 20) - 1, 1 << 20, (1 << 24) - 1):
        for vocab in (1, 170, 20000, 131072, 17000001):
            for dim in (1, 75, 128, 136, 602, 1024, 4096):
                for dtype, es in ((0, 4), (1, 2), (2, 2)):
                    for aligned in (0, 1):
                        width = -(-dim * es // 16) * 16 // es
                        narrow = es == 2 and width <= 128
                        rows = 32 if n <= 32 and not narrow else -(-n // 256) * 256
                        copies = rows * width * es + (vocab * width * es if width != dim or not aligned else 0)
                        sums = max(64 * MB, rows * width * 4) + 64 * MB
                        g = 0 if narrow else max(512 * MB, 512 * rows) + 256 * rows
                        need = L.coop_softmax_xent_workspace_bytes(n, vocab, dim, dtype, aligned, 1)
                        assert 0 < need <= copies + sums + g + 16 * rows + 8192, (n, vocab, dim, dtype, aligned)


def test_memory_of_a_call_is_that_of_its_stream(monkeypatch):
    """Results and workspaces come from torch while the stream that writes them is the current one, and torch is told that the stream which
    was current uses the results."""
    now, made = ["main"], []

    class Current:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            now.append(self.stream)

        def __exit__(self, *error):
            now.pop()

    class Buffer:
        def __init__(self, *shape, **kw):
            self.of, self.used_on = now[-1], []
            made.append(self)

        def data_ptr(self):
            return 0x1000

        def record_stream(self, stream):
            self.used_on.append(stream)

    monkeypatch.setattr(learn.torch, "empty", Buffer)
    monkeypatch.setattr(learn.torch.cuda, "stream", Current)
    monkeypatch.setattr(learn.torch.cuda, "current_stream", lambda device=None: now[-1])
    for module in (learn, learn.binding):
        monkeypatch.setattr(module, "_torch_stream", lambda stream: stream, raising=False)
    learn._new((3, 4), torch.float32, "cuda", None)
    learn._new((3, 4), torch.float32, "cuda", "side")
    learn._workspace(1024, None, "cuda", "side")
    assert [(b.of, b.used_on) for b in made] == [("main", []), ("side", ["main"]), ("side", [])] and now == ["main"]


@gpu
def test_memory_that_the_current_stream_still_uses_is_not_written():
    """Work that waits on torch's current stream, over memory that has been given back, does not meet a call's on another stream."""
    g = rng(31)
    table, ids = normal(g, 3000, 256), torch.randint(0, 3000, (20000,), generator=g, device="cuda", dtype=torch.int32)
    want = P.coop_embed(table, ids)
    side = torch.cuda.Stream()
    old = torch.empty_like(want)
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)        # (some ten milliseconds)
    old.fill_(7.0)
    del old
    got = P.coop_embed(table, ids, stream=side)
    grad = P.coop_embed_grad(want, ids, 3000, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(grad, P.coop_embed_grad(want, ids, 3000))


def test_norm_weights_of_unknown_types_are_refused_like_other_arguments():
    x, w = torch.zeros((2, 4)), torch.zeros(4)
    assert learn._weight_dtype(x) == learn._weight_dtype(x, w, w) == P.COOP_F32 and learn._weight_dtype(x, w.half()) == P.COOP_F16
    for weights in ((w.double(),), (w.int(), w.int()), (w, w.half())):
        with pytest.raises(AssertionError):
            learn._weight_dtype(x, *weights)
