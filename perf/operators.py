"""What a program that learns vertex embeddings from sampled blocks does with them, as cases that can be timed and compared.

Four operators: the rows of a table looked up with a scale, and their gradient with the tokens sorted (`embed`); layer
norm with its gradient (`norm`); softmax cross entropy over a large vocabulary (the vertices of a graph, or tokens) without
the logits kept, with its gradient (`xent`); and an AdamW step over many tensors, or over the touched rows of a table, with
moments in 32 or in 8 bits (`adamw`).

A case is a dict of sizes and types; `prepare` makes what the program has in hand, `run` is one pass: the plain form in
elementary torch operations in 32 bits, or, where `own` is true, the calls of this repository's package.  `exact` is the
definition in 64 bits.
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
PAD = -1        # the id of a place that holds no token, and the target of a row without one
BLOCK = 256     # elements that share a scale in an 8-bit moment

# What a case says where it does not say otherwise.
DEFAULTS = {
    "embed": dict(way="forward", n=1024, vocab=100000, dim=128, type="f32", out="f32", ids="zipf", distinct=0, scaled=False, alpha=1.0, pads=0.0),
    "norm": dict(rows=1024, dim=128, type="f32", weights="f32", train=True),
    "xent": dict(n=1024, vocab=50021, dim=128, type="bf16", train=True, ignored=0.0, alpha=1.0),
    "adamw": dict(tensors=1, total=1 << 20, type="f32", grads="f32", copies="", bits=32, packed=False, vocab=0, dim=0, rows=0,
                  clipped=False),
}


def _case(name, op, **kw):
    return dict(DEFAULTS[op], name=name, op=op, **kw)


def listed():
    return [
        # The embeddings of a handful of vertices that are scored on request, from the products-shaped graph's table: latency.
        _case("embed_few", "embed", n=24, vocab=2450000, dim=100, ids="distinct"),
        # The input rows of a minibatch of the papers100M configuration at its stated batch, from a learned fp16 table of a
        # quarter of its vertices, each row with a weight of its own.
        _case("embed_frontier", "embed", n=2592327, vocab=27764989, dim=128, type="f16", out="f16", ids="distinct", scaled=True),
        # Back through the edges of a sampled block: a million tokens, every source vertex at least once and the hubs thousands
        # of times, and only the rows that were touched come back, as an optimiser of a table that large wants them.
        _case("embed_grad_edges", "embed", way="rows", n=1019311, vocab=2450000, dim=128, type="bf16", out="f32", ids="edges",
              distinct=572596),
        # The gradient of a whole small table, everything odd: 150-byte rows, places without a token, a scale per token.
        _case("embed_grad_ragged", "embed", way="dense", n=65537, vocab=50021, dim=75, type="f16", out="f32", scaled=True,
              alpha=8.66, pads=0.1),
        # The norm of the handful's rows.
        _case("norm_few", "norm", rows=24, dim=100, train=False),
        # Norm and gradient of the vertices of a minibatch's second layer, 256-byte rows.
        _case("norm_frontier", "norm", rows=572596, dim=128, type="bf16"),
        # Scoring a handful of targets among the vertices of the reddit-shaped graph: the weight is read once.
        _case("xent_few", "xent", n=24, vocab=232965, dim=128, train=False),
        # A training step on the reddit-shaped graph at its stated batch: predict a sampled neighbour among all vertices.
        # The inner dimension is short, so exponentials weigh as much as products.
        _case("xent_vertices", "xent", n=8192, vocab=232965, dim=128, ignored=0.05),
        # A vocabulary and a width of a language model's head: products are nearly all there is.
        _case("xent_tokens", "xent", n=8192, vocab=131072, dim=1024, ignored=0.1),
        # Nothing divides anything, and 32-bit products.
        _case("xent_ragged", "xent", n=1021, vocab=50021, dim=100, type="f32", ignored=0.1, alpha=0.7),
        # A model's parameters of all sizes, gradients in 16 bits, a 16-bit copy for the next pass, the gradient's norm clipped.
        _case("adamw_many", "adamw", tensors=300, total=100000000, grads="bf16", copies="bf16", clipped=True),
        # The touched rows of the products-shaped graph's table, moments in 8 bits.
        _case("adamw_rows", "adamw", bits=8, vocab=2450000, dim=100, rows=500000),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    dims = [1, 64, 75, 100, 128, 256, 602, 768, 1024]
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(["embed", "embed", "norm", "xent", "xent", "adamw"])
        c = dict(DEFAULTS[op], op=op)
        if op == "embed":
            c.update(way=rng.choice(["forward", "rows", "dense"]), n=_log_uniform(rng, 1, 3000000), vocab=_log_uniform(rng, 2, 20000000),
                     dim=rng.choice(dims + [rng.randint(2, 1024)]), type=rng.choice(list(TYPES)), out=rng.choice(list(TYPES)),
                     ids=rng.choice(["zipf", "uniform"]), scaled=rng.random() < 0.5, alpha=rng.choice([1.0, 11.3]))
            c["pads"] = rng.choice([0.0, 0.0, 0.2, 0.9]) if c["n"] >= 64 else 0.0
            if c["way"] == "rows":
                c.update(ids="edges", distinct=_log_uniform(rng, 1, min(c["vocab"], max(1, c["n"] // 8 if c["pads"] else c["n"]))))
            size = c["vocab"] * c["dim"] * (4 if c["way"] == "dense" else BYTES[c["type"]] if c["way"] == "forward" else 0)
            if size > 8e9:
                continue
        elif op == "norm":
            c.update(rows=_log_uniform(rng, 1, 600000), dim=rng.choice(dims + [4096, rng.randint(1, 9000)]), type=rng.choice(list(TYPES)),
                     train=rng.random() < 0.7)
            c["weights"] = rng.choice(["f32", c["type"]])
        elif op == "xent":
            c.update(n=_log_uniform(rng, 1, 16384), vocab=_log_uniform(rng, 64, 250000), dim=rng.choice(dims + [rng.randint(1, 1100)]),
                     type=rng.choice(["bf16", "bf16", "f16", "f32"]), train=rng.random() < 0.7, ignored=rng.choice([0.0, 0.1, 1.0]),
                     alpha=rng.choice([1.0, 0.5]))
        elif rng.random() < 0.5:
            n = _log_uniform(rng, 1, 400)
            c.update(tensors=n, total=max(_log_uniform(rng, 1000, 100000000), 16 * n), type=rng.choice(list(TYPES)), grads=rng.choice(list(TYPES)),
                     bits=rng.choice([8, 32]), packed=rng.random() < 0.4, clipped=rng.random() < 0.5)
            c["copies"] = rng.choice(["", "f16", "bf16"]) if c["type"] == "f32" else ""
        else:
            c.update(vocab=_log_uniform(rng, 100, 4000000), dim=rng.choice(dims + [rng.randint(2, 1024)]), grads=rng.choice(list(TYPES)), bits=rng.choice([8, 32]))
            c["rows"] = min(c["vocab"], _log_uniform(rng, 1, 1000000))
            if c["vocab"] * c["dim"] > 4e8:
                continue
        if _cost(c) <= most:
            return c


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 5e12, w["flops"] / (5e13 if case.get("type") == "f32" else 5e14))


def _expected_rows(c):
    """How many different ids the tokens are expected to have."""
    n, v = c["n"] * (1 - c["pads"]), c["vocab"]
    if c["ids"] == "distinct":
        return n
    if c["ids"] == "edges":
        return c["distinct"]
    if c["ids"] == "uniform":
        return v * -math.expm1(-n / v)
    rank = np.unique(np.geomspace(1, v + 1, 400).astype(np.int64))
    p = np.diff(np.log(rank)) / math.log(v + 1) / np.diff(rank)     # of one id of the class
    return float((np.diff(rank) * -np.expm1(-n * p)).sum())


def work(case):
    """What a pass cannot do without: every input read once, every output written once, the products that the outputs take."""
    c = case
    if c["op"] == "embed":
        n, rows, size, out = c["n"], _expected_rows(c), BYTES[c["type"]], BYTES[c["out"]]
        tokens = n * (4 + (4 if c["scaled"] else 0))
        if c["way"] == "forward":
            return {"bytes": tokens + c["dim"] * (rows * size + n * out), "flops": n * c["dim"]}
        live = n * (1 - c["pads"])
        written = c["vocab"] * c["dim"] * out if c["way"] == "dense" else rows * (4 + c["dim"] * out)
        return {"bytes": tokens + live * c["dim"] * size + written, "flops": 2 * live * c["dim"]}
    if c["op"] == "norm":
        x, stats = c["rows"] * c["dim"] * BYTES[c["type"]], 8 * c["rows"]
        if not c["train"]:
            return {"bytes": 2 * x + stats + 2 * c["dim"] * BYTES[c["weights"]], "flops": 8 * c["rows"] * c["dim"]}
        # (backward: the gradient and the input in, the input's gradient out, and the weights')
        return {"bytes": 5 * x + 2 * stats + c["dim"] * (3 * BYTES[c["weights"]] + 8), "flops": 20 * c["rows"] * c["dim"]}
    if c["op"] == "xent":
        size = BYTES[c["type"]]
        operands = (c["n"] + c["vocab"]) * c["dim"] * size
        product = 2 * c["n"] * c["vocab"] * c["dim"]
        # (trained: the logits once, the hidden states' gradient and the weight's)
        return {"bytes": operands * (2 if c["train"] else 1) + c["n"] * (16 if c["train"] else 12), "flops": product * (3 if c["train"] else 1)}
    count = c["rows"] * c["dim"] if c["rows"] else c["total"]
    each = 2 * BYTES[c["type"]] + BYTES[c["grads"]] + (16 if c["bits"] == 32 else 4 + 16 / BLOCK) + (2 if c["copies"] else 0)
    return {"bytes": count * each + 4 * c["rows"], "flops": 15 * count}


# ---- state -------------------------------------------------------------------------------------------------------------
def _normal(g, *shape, scale=1.0, dtype=torch.float32):
    return torch.empty(shape, device=DEVICE).normal_(0.0, scale, generator=g).to(dtype)


def _ids(g, c):
    n, v = c["n"], c["vocab"]
    if c["ids"] == "distinct":      # what a sampled frontier is: no vertex twice, no order
        first = int(torch.randint(v, (1,), generator=g, device=DEVICE))
        return ((torch.arange(n, device=DEVICE) * 805459861 + first) % v).to(torch.int32)
    k = c["distinct"] if c["ids"] == "edges" else v
    u = torch.rand(n, generator=g, device=DEVICE, dtype=torch.float64)
    rank = ((u * k).long() if c["ids"] == "uniform" else torch.exp(u * math.log(k + 1)).long() - 1).clamp(0, k - 1)
    pads = torch.rand(n, generator=g, device=DEVICE) < c["pads"]
    if c["ids"] == "edges":     # `distinct` different ones, each at least once
        once = torch.randperm(n, generator=g, device=DEVICE)[:k]
        rank[once], pads[once] = torch.arange(k, device=DEVICE), False
    ids = (rank * 805459861 + int(torch.randint(v, (1,), generator=g, device=DEVICE))) % v  # the frequent ones lie anywhere
    ids[pads] = PAD
    return ids.to(torch.int32)


def tensor_sizes(case):
    """The elements of each of a model's tensors: a third of them short (norms, biases), the others spread over three decades."""
    k = case["tensors"]
    w = [1.0 if i % 3 == 0 else 10.0 ** (1 + 3 * ((i * 0.6180339887) % 1.0)) for i in range(k)]
    return [max(1, int(case["total"] * x / sum(w))) for x in w]


def _flat(case):
    """(sizes, where each tensor begins in its flat buffer, the buffer's length)"""
    sizes = tensor_sizes(case)
    step = 1 if case["packed"] else 64
    at = np.concatenate([[0], np.cumsum([-(-s // step) * step for s in sizes])])
    return sizes, [int(a) for a in at[:-1]], int(at[-1])


def _views(flat, sizes, at):
    return [flat[a:a + s] for s, a in zip(sizes, at)]


def _blocks(n):
    return -(-n // BLOCK)


def prepare(case, seed):
    c = dict(DEFAULTS[case["op"]], **case)
    g = torch.Generator(device=DEVICE).manual_seed(int(seed))
    s = {"case": c}
    dtype = TYPES[c["type"]]
    if c["op"] == "embed":
        s["ids"] = _ids(g, c)
        s["scale"] = torch.rand(c["n"], generator=g, device=DEVICE) + 0.5 if c["scaled"] else None
        if c["way"] == "forward":
            s["table"] = torch.empty((c["vocab"], c["dim"]), device=DEVICE, dtype=dtype).normal_(0.0, 1.0, generator=g)
        else:
            s["dout"] = _normal(g, c["n"], c["dim"], dtype=dtype)
    elif c["op"] == "norm":
        w = TYPES[c["weights"]]
        s["x"] = (_normal(g, c["rows"], c["dim"]) * (0.1 + torch.rand((c["rows"], 1), generator=g, device=DEVICE))
                  + _normal(g, c["rows"], 1)).to(dtype)
        s["weight"], s["bias"] = (1 + _normal(g, c["dim"], scale=0.1)).to(w), _normal(g, c["dim"], scale=0.1, dtype=w)
        s["eps"] = 1e-5
        if c["train"]:
            s["dy"] = _normal(g, c["rows"], c["dim"], dtype=dtype)
    elif c["op"] == "xent":
        w = _normal(g, c["vocab"], c["dim"], scale=1.5 / math.sqrt(c["dim"]), dtype=dtype)
        t = torch.randint(c["vocab"], (c["n"],), generator=g, device=DEVICE)
        s["hidden"] = (_normal(g, c["n"], c["dim"]) + 2.0 * w[t].float()).to(dtype)   # a model that has learnt something
        t[torch.rand(c["n"], generator=g, device=DEVICE) < c["ignored"]] = PAD
        s["weight"], s["targets"] = w, t.to(torch.int32)
        # the gradient of the mean over the rows that have a target; fp16 is trained with the loss scaled up
        s["dloss"] = torch.full((c["n"],), 4096.0 if c["type"] == "f16" else 1.0, device=DEVICE) / (t != PAD).sum().clamp(min=1)
    else:
        s["step"], s["hyper"] = 100, dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01)
        s["clip"] = torch.rand(1, generator=g, device=DEVICE) if c["clipped"] else None
        if c["rows"]:
            sizes, at, n, scales = [c["vocab"] * c["dim"]], [0], c["vocab"] * c["dim"], c["vocab"] * _blocks(c["dim"])
            s["shape"] = (c["vocab"], c["dim"])
            order = (torch.arange(c["rows"], device=DEVICE) * 805459861 + int(seed) % 9973) % c["vocab"]
            s["rows"] = order.sort().values.to(torch.int32)
            s["grad"] = _normal(g, c["rows"], c["dim"], scale=1e-3, dtype=TYPES[c["grads"]])
        else:
            sizes, at, n = _flat(c)
            scales = sum(_blocks(k) for k in sizes)
            s["grad"] = _normal(g, n, scale=1e-3, dtype=TYPES[c["grads"]])
        s["sizes"], s["at"] = sizes, at
        s["param"] = _normal(g, n, scale=0.05, dtype=dtype)
        s["copy"] = torch.zeros(n, device=DEVICE, dtype=TYPES[c["copies"]]) if c["copies"] else None
        m, r = _normal(g, n, scale=3e-4), _normal(g, n, scale=1e-3).abs()
        if c["bits"] == 32:
            s["m"], s["v"] = m, r * r
        else:   # 8-bit floats of the first moment and of the second one's root, over a scale for each block
            s["m"], s["v"] = ((x * (100.0 / 3e-4)).clamp(-448, 448).to(torch.float8_e4m3fn) for x in (m, r))
            s["m_scale"], s["v_scale"] = (torch.rand(scales, generator=g, device=DEVICE) * 1e-6 + 2e-6 for _ in range(2))
        if own:
            s["plan"] = _plan(s)
    return s


def _plan(s):
    import paper_2310_12403_amd as P
    c = s["case"]
    if c["rows"]:
        params, grads, copies = [s["param"].view(s["shape"])], None, None
    else:
        params, grads = _views(s["param"], s["sizes"], s["at"]), _views(s["grad"], s["sizes"], s["at"])
        copies = _views(s["copy"], s["sizes"], s["at"]) if c["copies"] else None
    state = {"m": _views(s["m"], s["sizes"], s["at"]), "v": _views(s["v"], s["sizes"], s["at"])}
    if c["bits"] == 8:
        n = [_blocks(k) for k in s["sizes"]] if not c["rows"] else [s["m_scale"].numel()]
        first = [sum(n[:i]) for i in range(len(n))]
        state["m_scale"], state["v_scale"] = _views(s["m_scale"], n, first), _views(s["v_scale"], n, first)
    return P.AdamW(params, grads, bits=c["bits"], by_rows=bool(c["rows"]), copies=copies, state=state)


# ---- one pass ------------------------------------------------------------------------------------------------------------
def run(state):
    return {"embed": _embed, "norm": _norm, "xent": _xent, "adamw": _adamw}[state["case"]["op"]](state)


def _embed(s):
    c = s["case"]
    if own:
        import paper_2310_12403_amd as P
        kw = dict(scale=s["scale"], alpha=c["alpha"], pad=PAD, dtype=TYPES[c["out"]])
        if c["way"] == "forward":
            return P.coop_embed(s["table"], s["ids"], **kw)
        if c["way"] == "dense":
            return P.coop_embed_grad(s["dout"], s["ids"], c["vocab"], **kw)
        return P.coop_embed_grad_rows(s["dout"], s["ids"], c["vocab"], **kw)
    out, ids = TYPES[c["out"]], s["ids"].long()
    live = ids != PAD
    factor = (s["scale"] * c["alpha"] if c["scaled"] else torch.full_like(ids, c["alpha"], dtype=torch.float32))[:, None]
    if c["way"] == "forward":
        x = s["table"][ids.clamp(min=0)].float() * factor
        return torch.where(live[:, None], x, 0.0).to(out)
    x, ids = (s["dout"].float() * factor)[live], ids[live]
    if c["way"] == "dense":
        return torch.zeros((c["vocab"], c["dim"]), device=DEVICE).index_add_(0, ids, x).to(out)
    hit = torch.zeros(c["vocab"], dtype=torch.bool, device=DEVICE)
    hit[ids] = True
    rows = hit.nonzero()[:, 0]
    place = torch.cumsum(hit, 0) - 1
    grad = torch.zeros((rows.numel(), c["dim"]), device=DEVICE).index_add_(0, place[ids], x)
    return rows.to(torch.int32), grad.to(out)


def _norm(s):
    train = s["case"]["train"]
    if own:
        import paper_2310_12403_amd as P
        y, mean, rstd = P.coop_layer_norm(s["x"], s["weight"], s["bias"], eps=s["eps"])
        if not train:
            return y, mean, rstd
        return (y, mean, rstd) + tuple(P.coop_layer_norm_grad(s["dy"], s["x"], mean, rstd, s["weight"]))
    x, w, b = s["x"].float(), s["weight"].float(), s["bias"].float()
    mean = x.mean(1)
    x = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((x * x).mean(1) + s["eps"])
    x = x * rstd[:, None]
    y = (x * w + b).to(s["x"].dtype)
    if not train:
        return y, mean, rstd
    dy = s["dy"].float()
    d = dy * w
    dx = (d - d.mean(1)[:, None] - x * (d * x).mean(1)[:, None]) * rstd[:, None]
    return y, mean, rstd, dx.to(s["x"].dtype), (dy * x).sum(0), dy.sum(0)


def _xent(s):
    c = s["case"]
    if own:
        import paper_2310_12403_amd as P
        loss, lse = P.coop_softmax_xent(s["hidden"], s["weight"], s["targets"], alpha=c["alpha"], ignore=PAD)
        if not c["train"]:
            return loss, lse
        return (loss, lse) + tuple(P.coop_softmax_xent_grad(s["hidden"], s["weight"], s["targets"], lse, s["dloss"], alpha=c["alpha"], ignore=PAD))
    h, w, t = s["hidden"].float(), s["weight"].float(), s["targets"].long()
    live, row = t != PAD, torch.arange(c["n"], device=DEVICE)
    t = t.clamp(min=0)
    z = (h @ w.t()) * c["alpha"]
    top = z.max(1).values
    lse = torch.log(torch.exp(z - top[:, None]).sum(1)) + top
    loss = torch.where(live, lse - z[row, t], 0.0)
    if not c["train"]:
        return loss, lse
    p = torch.exp(z - lse[:, None])
    p[row, t] -= 1.0
    p = p * torch.where(live, s["dloss"] * c["alpha"], 0.0)[:, None]
    return loss, lse, (p @ w).to(s["hidden"].dtype), (p.t() @ h).to(s["weight"].dtype)


# The 32-bit mixer and the key words (Philox4x32-10) by which an 8-bit moment is rounded at random.
def _mix(x):
    x = x ^ (x >> 16)
    x = (x * 0x7FEB352D) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0x846CA68B) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _philox_round(c, k):
    p, q = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
    return ((q >> 32) ^ c[1] ^ k[0], q & 0xFFFFFFFF, (p >> 32) ^ c[3] ^ k[1], p & 0xFFFFFFFF)


def _keys(seed, step, tensor):
    c, k = (step & 0xFFFFFFFF, step >> 32, tensor, 0x4144414D), (seed & 0xFFFFFFFF, seed >> 32)
    for _ in range(10):
        c = _philox_round(c, k)
        k = ((k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF)
    return c


def _random(element, seed, step, tensor):
    k = _keys(seed, step, tensor)
    u = _mix(_mix((element & 0xFFFFFFFF) ^ k[0]) ^ k[1] ^ _mix((element >> 32) ^ k[2])) ^ k[3]
    return ((u & 0xFFFF) << 4) + 8, ((u >> 16) << 4) + 8


def _by_blocks(x, rows, dim):
    """[rows, dim] as [rows, blocks, BLOCK], zeros behind a row's end"""
    pad = torch.zeros((rows, _blocks(dim) * BLOCK), dtype=x.dtype, device=DEVICE)
    pad[:, :dim] = x.reshape(rows, dim)
    return pad.view(rows, _blocks(dim), BLOCK)


def _encode(x, noise, floor):
    """(8-bit floats, scales) of x [rows, blocks, BLOCK]: rounded up or down at random, so that the mean is x"""
    scale = x.abs().amax(2) * (1.0 / 448.0)
    y = x / scale[:, :, None]
    bits = (y.abs() * 2.0 ** -120).view(torch.int32)
    code = ((bits + noise) >> 20).clamp(max=0x7E)
    code = torch.where(x == 0, 0, torch.where((x != 0) & (code == 0), floor, code))
    code = torch.where(scale[:, :, None] == 0, 0, code)
    code = code | ((x < 0).int() << 7)
    return code.to(torch.uint8).view(torch.float8_e4m3fn), scale


def _update(p, g, m, v, h, step, clip):
    """One AdamW step, elementwise: the new parameter and moments."""
    if clip is not None:
        g = g * clip
    m = m * h["beta1"] + g * (1 - h["beta1"])
    v = v * h["beta2"] + (g * g) * (1 - h["beta2"])
    root = torch.sqrt(v)
    rate, undo = h["lr"] / (1 - h["beta1"] ** step), 1 / math.sqrt(1 - h["beta2"] ** step)
    p = p * (1 - h["lr"] * h["weight_decay"]) - (m / (root * undo + h["eps"])) * rate
    return p, m, v, root


def _moments(m, v, m_scale, v_scale, rows, dim):
    """The 32-bit moments that 8-bit ones stand for, by blocks."""
    m, v = (_by_blocks(x.float(), rows, dim) * s.view(rows, _blocks(dim), 1) for x, s in ((m, m_scale), (v, v_scale)))
    return m, v * v


def _step_tensor(s, i, p, g, rows, dim, m, v, m_scale, v_scale, first):
    """The new (parameter, m, v, scales) of one tensor or of a table's touched rows; `first`: each row's first element's number."""
    h, step = s["hyper"], s["step"]
    if m_scale is None:
        p, m, v, _ = _update(p.float(), g.float(), m, v, h, step, s["clip"])
        return p, m, v, None, None
    m, v = _moments(m, v, m_scale, v_scale, rows, dim)
    p, m, v, root = _update(_by_blocks(p.float(), rows, dim), _by_blocks(g.float(), rows, dim), m, v, h, step, s["clip"])
    element = first.view(rows, 1, 1) + torch.arange(_blocks(dim) * BLOCK, device=DEVICE).view(1, -1, BLOCK)
    noise = _random(element, s.get("seed", 0), step, i)
    m, m_scale = _encode(m, noise[0].int(), 0)
    v, v_scale = _encode(root, noise[1].int(), 1)
    cut = [x.view(rows, -1)[:, :dim] for x in (p, m, v)]
    return cut[0], cut[1], cut[2], m_scale, v_scale


def _put(to, x):
    """x into the buffer it belongs to, rounded to its type"""
    if to is not None:
        to.copy_(x.reshape(to.shape).to(to.dtype))


def _adamw(s):
    c = s["case"]
    s["step"] += 1
    if own:
        rows = {0: (s["rows"], s["grad"], None)} if c["rows"] else None
        s["plan"].step(step=s["step"], seed=s.get("seed", 0), rows=rows, grad_scale=s["clip"], **s["hyper"])
    elif c["rows"]:
        at, dim, k = s["rows"].long(), c["dim"], c["rows"]
        table = {x: s[x].view(s["shape"]) for x in ("param", "m", "v")}
        bytes_of = {x: t.view(torch.uint8) if t.dtype.itemsize == 1 else t for x, t in table.items()}
        scales = {x: s[x].view(c["vocab"], -1) if c["bits"] == 8 else None for x in ("m_scale", "v_scale")}
        old = [bytes_of[x][at].view(table[x].dtype) for x in ("param", "m", "v")]
        p, m, v, ms, vs = _step_tensor(s, 0, old[0], s["grad"], k, dim, old[1], old[2],
                                       *(scales[x][at] if c["bits"] == 8 else None for x in ("m_scale", "v_scale")),
                                       at * (_blocks(dim) * BLOCK))
        bytes_of["param"][at] = p.reshape(k, dim).to(s["param"].dtype)
        bytes_of["m"][at], bytes_of["v"][at] = (x.contiguous().view(torch.uint8) if c["bits"] == 8 else x for x in (m, v))
        if c["bits"] == 8:
            scales["m_scale"][at], scales["v_scale"][at] = ms, vs
    else:
        views = {x: _views(s[x], s["sizes"], s["at"]) for x in ("param", "grad", "m", "v")}
        copies = _views(s["copy"], s["sizes"], s["at"]) if c["copies"] else [None] * len(s["sizes"])
        n = [_blocks(k) for k in s["sizes"]]
        first = np.concatenate([[0], np.cumsum(n)]).tolist()
        scales = [_views(s[x], n, first) if c["bits"] == 8 else [None] * len(n) for x in ("m_scale", "v_scale")]
        zero = torch.zeros(1, dtype=torch.int64, device=DEVICE)
        [_step_in_place(s, i, views, copies, scales, zero) for i in range(len(n))]
    return [s[x] for x in ("param", "m", "v", "m_scale", "v_scale", "copy") if s.get(x) is not None]


def _step_in_place(s, i, views, copies, scales, zero):
    p, g, m, v = (views[x][i] for x in ("param", "grad", "m", "v"))
    new = _step_tensor(s, i, p, g, 1, p.numel(), m, v, scales[0][i], scales[1][i], zero)
    for to, x in zip((p, m, v, scales[0][i], scales[1][i], copies[i]), (*new, new[0])):
        _put(to, x)


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"embed": _exact_embed, "norm": _exact_norm, "xent": _exact_xent, "adamw": _exact_adamw}[s["case"]["op"]](s)


def _exact_embed(s):
    c = s["case"]
    ids = s["ids"].long()
    factor = c["alpha"] * (torch.ones(c["n"], device=DEVICE) if s["scale"] is None else s["scale"]).double()
    factor[ids == PAD] = 0.0
    if c["way"] == "forward":
        return s["table"][ids.clamp(min=0)].double() * factor.view(-1, 1)
    # the tokens in the order of their ids, running sums, and the differences between the ends of the ids' stretches
    order = torch.argsort(ids, stable=True)
    order = order[int((ids == PAD).sum()):]
    sums = torch.cumsum(s["dout"][order].double() * factor[order].view(-1, 1), 0)
    rows, counts = torch.unique_consecutive(ids[order], return_counts=True)
    sums = sums[torch.cumsum(counts, 0) - 1]
    sums[1:] -= sums[:-1].clone()
    if c["way"] == "rows":
        return rows.to(torch.int32), sums
    table = torch.zeros((c["vocab"], c["dim"]), dtype=torch.float64, device=DEVICE)
    table[rows] = sums
    return table


def _exact_norm(s):
    x = s["x"].double()
    var, mean = torch.var_mean(x, 1, correction=0)
    rstd = torch.rsqrt(var + s["eps"])
    hat = (x - mean.view(-1, 1)) * rstd.view(-1, 1)
    y = torch.addcmul(s["bias"].double(), hat, s["weight"].double())
    if not s["case"]["train"]:
        return y, mean, rstd
    dy = s["dy"].double()
    # dx = rstd (I - 1 1' / D - hat hat' / D) (w dy)
    back = dy * s["weight"].double()
    dim = x.shape[1]
    dx = back - (back.sum(1, keepdim=True) + hat * (back * hat).sum(1, keepdim=True)) / dim
    return y, mean, rstd, dx * rstd.view(-1, 1), (dy * hat).sum(0), dy.sum(0)


def _exact_xent(s):
    c = s["case"]
    h, w, t = s["hidden"].double(), s["weight"].double(), s["targets"].long()
    z = c["alpha"] * (h @ w.t())
    lse = torch.logsumexp(z, 1)
    has = (t >= 0).double()
    loss = has * (lse - z.gather(1, t.clamp(min=0).view(-1, 1)).view(-1))
    if not c["train"]:
        return loss, lse
    z.sub_(lse.view(-1, 1)).exp_()
    z.scatter_add_(1, t.clamp(min=0).view(-1, 1), torch.full((c["n"], 1), -1.0, dtype=torch.float64, device=DEVICE))
    z.mul_((has * s["dloss"].double() * c["alpha"]).view(-1, 1))
    return loss, lse, z @ w, z.t().contiguous() @ h


def _exact_adamw(s):
    """As in 32 bits, in 64; where the moments are in 8 bits, their values differ wherever the two fall on either side of the
    random bound between two codes, a few in a million."""
    c, h, step = s["case"], s["hyper"], s["step"] + 1
    wide = {}
    if c["rows"]:
        pieces = [(s["rows"].long(), c["vocab"], c["dim"], 0, 0)]
    else:
        scale_at = np.concatenate([[0], np.cumsum([_blocks(k) for k in s["sizes"]])]).tolist()
        pieces = [(None, 1, k, a, b) for k, a, b in zip(s["sizes"], s["at"], scale_at)]
    for x in ("param", "m", "v", "m_scale", "v_scale", "copy"):
        wide[x] = s[x].to(torch.float64) if s.get(x) is not None else None
    for i, (at, rows, dim, first, first_scale) in enumerate(pieces):
        n, nb = rows * dim, _blocks(dim)
        take = (lambda t: t) if at is None else (lambda t: t[at])  # noqa: E731
        old = {x: take(wide[x][first:first + n].view(rows, dim)) for x in ("param", "m", "v")}
        g = (s["grad"] if at is not None else s["grad"][first:first + n]).double().view(-1, dim)
        if s["clip"] is not None:
            g = g * s["clip"].double()
        m, v = old["m"], old["v"]
        if c["bits"] == 8:
            wide_scale = {x: wide[x][first_scale:first_scale + rows * nb].view(rows, nb) for x in ("m_scale", "v_scale")}
            m = m * take(wide_scale["m_scale"]).repeat_interleave(BLOCK, 1)[:, :dim]
            v = (v * take(wide_scale["v_scale"]).repeat_interleave(BLOCK, 1)[:, :dim]) ** 2
        m = h["beta1"] * m + (1 - h["beta1"]) * g
        v = h["beta2"] * v + (1 - h["beta2"]) * g ** 2
        hat_m, hat_v = m / (1 - h["beta1"] ** step), v / (1 - h["beta2"] ** step)
        p = old["param"] - h["lr"] * (h["weight_decay"] * old["param"] + hat_m / (hat_v.sqrt() + h["eps"]))
        new = {"param": p, "m": m, "v": v}
        if c["bits"] == 8:
            row = torch.arange(rows, device=DEVICE) if at is None else at
            element = row.view(-1, 1) * (nb * BLOCK) + torch.arange(dim, device=DEVICE)
            for x, noise in zip(("m", "v"), _random(element, s.get("seed", 0), step, i)):
                value = m if x == "m" else v.sqrt()
                padded = torch.nn.functional.pad(value.abs(), (0, nb * BLOCK - dim)).view(-1, nb, BLOCK)
                scale = padded.amax(2) / 448.0
                y = value.abs() / scale.repeat_interleave(BLOCK, 1)[:, :dim]
                # the step between neighbouring 8-bit floats at y: 2^(exponent - 3), from 2^-9 on
                gap = torch.exp2(torch.floor(torch.log2(y.clamp(min=2.0 ** -6))) - 3)
                code = (torch.floor(y / gap + noise.double() / 2 ** 20) * gap).clamp(max=448.0)
                if x == "v":
                    code = torch.where((code == 0) & (y > 0), 2.0 ** -9, code)
                new[x] = torch.nan_to_num(code) * torch.sign(value)
                if at is None:
                    wide_scale[x + "_scale"].copy_(scale)
                else:
                    wide_scale[x + "_scale"][at] = scale
        for x, t in new.items():
            to = wide[x][first:first + n].view(rows, dim)
            if at is None:
                to.copy_(t)
            else:
                to[at] = t
        if wide["copy"] is not None:
            wide["copy"][first:first + n] = new["param"].view(-1)
    return [wide[x] for x in ("param", "m", "v", "m_scale", "v_scale", "copy") if wide[x] is not None]
