"""The work whose speed counts for the operators around a student's blocks:
embedding lookup of category columns with its gradient, counter-based dropout,
layer norm, and the product in 8-bit floating point with scales per block of
128, as cases that can be prepared, run and checked.

Together they are what a student on a table with category columns is made of:
its input (lookup, dropout), its residual stream (dropout added to it, layer
norm) and its wide layers served in 8 bits.  Sizes follow the repository's
workloads (widths 256..2048, batches 256..2048, 20011 validation rows, 37
serving rows) and plain generic ones.
"""
import math

import numpy as np
import torch

own = False
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
BLOCK = 128      # of a scale
F8_MAX = 448.0   # the largest e4m3 number


# ------------------------------------------------------------------ the cases
def _embed(name, **kw):
    # n ids into a table [vocab, d] of type table, looked up into type out; train: the table's gradient in fp32 too;
    # pad: spare elements at the end of every row of the table and of dy
    c = dict(name=name, op="embed", n=1, vocab=1000, d=64, table="fp32", out="bf16", ids="int32", scale=1.0, train=False, pad=0)
    c.update(kw)
    return c


def _dropout(name, **kw):
    # train: the gradient of x too; residual: a stream that the result is added to
    c = dict(name=name, op="dropout", rows=1, d=1024, dtype="bf16", p=0.1, residual=True, train=True, pad=0)
    c.update(kw)
    return c


def _norm(name, **kw):
    c = dict(name=name, op="norm", rows=1, d=1024, dtype="bf16", residual=True, bias=True, train=False, pad=0)
    c.update(kw)
    return c


def _f8(name, **kw):
    # out: "product" (x quantised, then its product with n rows of weights), "values" (quantised only, rows of block
    # rows sharing a scale)
    c = dict(name=name, op="f8", rows=1, k=1024, n=1000, dtype="bf16", bias=True, out="product", block=1, pad=0)
    c.update(kw)
    return c


def listed():
    return [
        # one row's category columns at serving time: latency
        _embed("embed_token", n=13),
        # a training batch of 24 category columns, frequent values far more often than rare ones
        _embed("embed_train", n=2048 * 24, vocab=20011, d=128, scale=8.0, train=True),
        # columns of few values: thousands of rows of dy for each row of the gradient
        _embed("embed_few", n=20011 * 7, vocab=300, d=33, table="fp32", out="fp32", ids="int64", train=True, pad=3),
        # a long batch over a large table
        _embed("embed_large", n=20011 * 40, vocab=1000003, d=64, train=True),
        # a training step's residual stream
        _dropout("dropout_train", rows=8192, d=2048),
        # a small batch in 32 bits on odd sizes, rows that start at odd addresses
        _dropout("dropout_odd", rows=500, d=389, dtype="fp32", p=0.35, residual=False, pad=3),
        # one row: latency
        _norm("norm_token"),
        # a training step's norm: residual added, all gradients
        _norm("norm_train", rows=8192, d=2048, train=True),
        # a wide odd row in 32 bits
        _norm("norm_odd", rows=2003, d=5001, dtype="fp32", train=True, residual=False),
        # a serving call of one row: the weights' bytes
        _f8("f8_token", k=2048, n=4096),
        # a batch of requests, no multiple of any tile or block, 32-bit results
        _f8("f8_requests", rows=500, k=2001, n=1003, dtype="fp32", pad=3),
        # a validation pass's wide layer
        _f8("f8_table", rows=8192, k=4096, n=4096),
    ]


def _log_int(rng, lo, hi):
    v = min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.999)) - 0.5 / hi)))))
    return v


def _size(rng, lo, hi):
    """A length of the range: odd, a multiple of 8 or a multiple of 64."""
    v = _log_int(rng, lo, hi)
    step = rng.choice([1, 1, 8, 64, 64])
    return max(lo, v // step * step)


def draw(rng):
    """One more case: its operator, types and options at random, sizes spread
    over their logarithm, odd ones among them."""
    while True:
        op = rng.choice(["embed", "embed", "embed", "dropout", "norm", "norm", "f8", "f8", "f8"])
        types, pads = ["bf16", "bf16", "fp32"], [0, 0, 8, 3]
        if op == "embed":
            c = _embed("", n=_log_int(rng, 1, 800440), vocab=_log_int(rng, 2, 1000003), d=_size(rng, 1, 1024),
                       table=rng.choice(["fp32", "bf16"]), out=rng.choice(types), ids=rng.choice(["int32", "int64"]),
                       scale=rng.choice([1.0, 8.0, 0.3]), train=rng.random() < 0.7, pad=rng.choice(pads))
        elif op == "dropout":
            c = _dropout("", rows=_log_int(rng, 1, 20011), d=_size(rng, 1, 8192), dtype=rng.choice(types),
                         p=rng.choice([0.0, 0.1, 0.25, 0.5, 0.9]), residual=rng.random() < 0.5, train=rng.random() < 0.7,
                         pad=rng.choice(pads))
        elif op == "norm":
            c = _norm("", rows=_log_int(rng, 1, 20011), d=_size(rng, 16, 8192), dtype=rng.choice(types),
                      residual=rng.random() < 0.7, bias=rng.random() < 0.8, train=rng.random() < 0.6, pad=rng.choice(pads))
        else:
            c = _f8("", rows=_log_int(rng, 1, 20011), k=_size(rng, 16, 8192), n=_size(rng, 10, 8192), dtype=rng.choice(types),
                    bias=rng.random() < 0.5, pad=rng.choice(pads))
            if rng.random() < 0.25:
                c.update(out="values", block=rng.choice([1, BLOCK]), bias=False)
        del c["name"]
        w = work(c)
        if w["bytes"] <= 5e8 and w["flops"] <= 2.7e11:
            return c


def _seen(n, vocab):
    """Rows of the table that n ids are expected to meet."""
    at = torch.linspace(0, 1, vocab + 1, dtype=torch.float64) ** (1 / 3)
    return float((1 - (1 - 0.97 * (at[1:] - at[:-1])) ** n).sum())


def work(c):
    size = {"bf16": 2.0, "fp32": 4.0}
    if c["op"] == "embed":
        n, d = float(c["n"]), float(c["d"])
        id_bytes = 8 if c["ids"] == "int64" else 4
        rows = _seen(c["n"], c["vocab"])
        b = n * id_bytes + rows * d * size[c["table"]] + n * d * size[c["out"]]
        if c["train"]:   # dy read, the whole gradient written
            b += n * d * size[c["out"]] + c["vocab"] * d * 4
        return {"bytes": b, "flops": n * d * (2 if c["train"] else 1)}
    e, r = size[c["dtype"]], float(c["rows"])
    if c["op"] == "dropout":
        passes = (3 if c["residual"] else 2) + (2 if c["train"] else 0)
        return {"bytes": passes * r * c["d"] * e, "flops": r * c["d"] * (4 if c["train"] else 2)}
    if c["op"] == "norm":
        d = float(c["d"])
        b = r * d * e * (4 if c["residual"] else 2) + (8 if c["bias"] else 4) * d
        if c["train"]:   # dy, the stored sum and its own gradient read, dx and both weights' gradients written
            b += r * d * e * (4 if c["residual"] else 3) + (12 if c["bias"] else 8) * d
        return {"bytes": b, "flops": r * d * (20 if c["train"] else 8)}
    k, n = float(c["k"]), float(c["n"])
    blocks = math.ceil(k / BLOCK)
    if c["out"] == "values":
        return {"bytes": r * k * (e + 1) + 4 * math.ceil(r / c["block"]) * blocks, "flops": 2 * r * k}
    return {"bytes": r * k * e + n * k + 4 * math.ceil(n / BLOCK) * blocks + (4 * n if c["bias"] else 0) + r * n * e,
            "flops": 2 * r * k * n}


# -------------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1000003 + 29) & 0x7FFFFFFFFFFF)
    return g


def _rand(g, rows, cols, dtype, scale=1.0, pad=0):
    """Normal values; pad: spare elements between the rows."""
    t = torch.randn(rows, cols + pad, generator=g, device=DEV) * scale
    return t.to(dtype)[:, :cols]


def _quantised_weights(w):
    """e4m3 weights with a scale for each block of 128 x 128, as a program stores them."""
    n, k = w.shape
    bn, bk = -(-n // BLOCK), -(-k // BLOCK)
    full = torch.zeros(bn * BLOCK, bk * BLOCK, device=DEV)
    full[:n, :k] = w
    full = full.view(bn, BLOCK, bk, BLOCK)
    s = full.abs().amax((1, 3)) / F8_MAX
    q = (full / s[:, None, :, None]).clamp(-F8_MAX, F8_MAX).to(torch.float8_e4m3fn)
    return q.view(bn * BLOCK, bk * BLOCK)[:n, :k].contiguous(), s


def prepare(case, seed):
    c, g = case, _gen(seed)
    s = {"c": c}
    if c["op"] == "embed":
        n, v, d = c["n"], c["vocab"], c["d"]
        # frequent values first, as a vocabulary is numbered; some entries are missing (-1)
        ids = (v * torch.rand(n, generator=g, device=DEV, dtype=torch.float64) ** 3).long().clamp(max=v - 1)
        ids = torch.where(torch.rand(n, generator=g, device=DEV) < 0.03, -1, ids)
        s["ids"] = ids.to(torch.int32 if c["ids"] == "int32" else torch.int64)
        s["table"] = _rand(g, v, d, TYPES[c["table"]], 1 / math.sqrt(d), c["pad"])
        if c["train"]:
            s["dy"] = _rand(g, n, d, TYPES[c["out"]], 1e-3, c["pad"])
        return s
    T = TYPES[c["dtype"]]
    if c["op"] == "dropout":
        s["x"] = _rand(g, c["rows"], c["d"], T, 1.0, c["pad"])
        s["res"] = _rand(g, c["rows"], c["d"], T, 3.0, c["pad"]) if c["residual"] else None
        s["dy"] = _rand(g, c["rows"], c["d"], T, 1.0 / c["rows"], c["pad"]) if c["train"] else None
        s["seed"], s["step"], s["site"] = (0x9E3779B97F4A7C15 * (int(seed) + 1)) & 0xFFFFFFFFFFFFFFFF, 1000 + int(seed) % 1000, 5
    elif c["op"] == "norm":
        # a residual stream that grew and drifted from zero, a block's output beside it
        s["x"] = _rand(g, c["rows"], c["d"], T, 1.0, c["pad"])
        s["res"] = None
        if c["residual"]:
            s["res"] = (_rand(g, c["rows"], c["d"] + c["pad"], torch.float32, 3.0) + 0.5).to(T)[:, : c["d"]]
        s["w"] = 1 + 0.2 * torch.randn(c["d"], generator=g, device=DEV)
        s["b"] = 0.1 * torch.randn(c["d"], generator=g, device=DEV) if c["bias"] else None
        if c["train"]:
            s["dy"] = _rand(g, c["rows"], c["d"], T, 1.0 / c["rows"], c["pad"])
            s["dsum"] = _rand(g, c["rows"], c["d"], T, 1.0 / c["rows"], c["pad"]) if c["residual"] else None
    else:
        # activations some of whose channels are far larger than the rest
        x = torch.randn(c["rows"], c["k"] + c["pad"], generator=g, device=DEV)
        x *= torch.where(torch.rand(c["k"] + c["pad"], generator=g, device=DEV) < 0.01, 20.0, 1.0)
        s["x"] = x.to(T)[:, : c["k"]]
        if c["out"] == "product":
            w = torch.randn(c["n"], c["k"], generator=g, device=DEV) / math.sqrt(c["k"])
            s["w"], s["ws"] = _quantised_weights(w)
            s["b"] = 0.1 * torch.randn(c["n"], generator=g, device=DEV) if c["bias"] else None
    return s


# ------------------------------------------------- the operators' plain forms
def _plain_embed(s):
    c = s["c"]
    there = s["ids"] >= 0
    at = s["ids"].clamp(min=0).long()
    y = torch.where(there[:, None], s["table"][at].float() * c["scale"], 0.0).to(TYPES[c["out"]])
    if not c["train"]:
        return [y]
    g = torch.zeros(c["vocab"], c["d"], device=DEV)
    g.index_add_(0, at, torch.where(there[:, None], s["dy"].float(), 0.0))
    return [y, g * c["scale"]]


def _high(m, v):
    """The upper 32 bits of the product of two 32-bit numbers."""
    return ((m >> 16) * v + ((m & 0xFFFF) * v >> 16)) >> 16


def _kept(seed, step, site, rows, d, p):
    """Philox4x32-10 at counter (row, column / 4, step, site): an element is
    kept where its word is not below floor(p 2^32)."""
    c0 = torch.arange(rows, device=DEV)[:, None]
    c1 = torch.arange((d + 3) // 4, device=DEV)[None, :]
    c = [c0, c1, torch.full_like(c0, step), torch.full_like(c0, site)]
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    low = 0xFFFFFFFF
    for _ in range(10):
        c = [_high(0xCD9E8D57, c[2]) ^ c[1] ^ k0, 0xCD9E8D57 * c[2] & low,
             _high(0xD2511F53, c[0]) ^ c[3] ^ k1, 0xD2511F53 * c[0] & low]
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack(torch.broadcast_tensors(*c), -1).reshape(rows, -1)[:, :d]
    return words >= math.floor(float(np.float32(p)) * 2 ** 32)


def _plain_dropout(s):
    c = s["c"]
    T = TYPES[c["dtype"]]
    keep = _kept(s["seed"], s["step"], s["site"], c["rows"], c["d"], c["p"])
    up = 1 / (1 - float(np.float32(c["p"])))
    y = torch.where(keep, s["x"].float() * up, 0.0)
    out = [(y if s["res"] is None else y + s["res"].float()).to(T)]
    return out + [torch.where(keep, s["dy"].float() * up, 0.0).to(T)] if c["train"] else out


EPS = 1e-5


def _plain_norm(s):
    c = s["c"]
    T = TYPES[c["dtype"]]
    # the norm of the sum as it is stored
    v = s["x"] if s["res"] is None else (s["x"].float() + s["res"].float()).to(T)
    out = [] if s["res"] is None else [v]
    v = v.float()
    mid = v - v.mean(1, keepdim=True)
    r = 1 / torch.sqrt((mid * mid).mean(1, keepdim=True) + EPS)
    h = mid * r
    y = h * s["w"]
    out.append((y if s["b"] is None else y + s["b"]).to(T))
    if c["train"]:
        dy = s["dy"].float()
        t = dy * s["w"]
        dx = r * (t - t.mean(1, keepdim=True) - h * (t * h).mean(1, keepdim=True))
        out.append((dx if s["dsum"] is None else dx + s["dsum"].float()).to(T))
        out.append((dy * h).sum(0))
        if s["b"] is not None:
            out.append(dy.sum(0))
    return out


def _spread(scale, block, rows, k):
    """A scale for each element of its block."""
    s = scale.repeat_interleave(BLOCK, 1)[:, :k]
    return s if block == 1 else s.repeat_interleave(block, 0)[:rows]


def _plain_quantise(x, block):
    """The e4m3 numbers nearest to x / scale: quotients in 64 bits, because
    those of 32 meet the borders between two numbers."""
    rows, k = x.shape
    br, bk = -(-rows // block), -(-k // BLOCK)
    full = torch.zeros(br * block, bk * BLOCK, device=DEV)
    full[:rows, :k] = x
    scale = (full.view(br, block, bk, BLOCK).abs().amax((1, 3)).double() / F8_MAX).float()
    each = _spread(scale, block, rows, k).double()
    t = torch.where(each > 0, x.double() / each, 0.0)
    # four significant bits, or steps of 2^-9 below 2^-6
    unit = torch.ldexp(torch.ones_like(t), torch.frexp(t).exponent.clamp(min=-5) - 4)
    return (torch.round(t / unit) * unit).clamp(-F8_MAX, F8_MAX).to(torch.float8_e4m3fn), scale


def _values(q, scale, block, T):
    """What 8-bit values stand for."""
    return (q.float() * _spread(scale, block, *q.shape)).to(T)


def _plain_f8(s):
    c = s["c"]
    T = TYPES[c["dtype"]]
    q, scale = _plain_quantise(s["x"], c["block"])
    if c["out"] == "values":
        return [_values(q, scale, c["block"], T), scale]
    y = _values(q, scale, 1, torch.float32) @ _values(s["w"], s["ws"], BLOCK, torch.float32).T
    return [(y if s["b"] is None else y + s["b"]).to(T)]


# -------------------------------------------------------------------- a pass
def _own(s):
    import paper_2607_05380_gb300 as tp
    c = s["c"]
    if c["op"] == "embed":
        y = tp.embed(s["ids"], s["table"], c["scale"], dtype=TYPES[c["out"]])
        return [y, tp.embed_backward(s["dy"], s["ids"], c["vocab"], c["scale"])] if c["train"] else [y]
    if c["op"] == "dropout":
        y = tp.dropout(s["x"], c["p"], s["seed"], s["step"], s["site"], residual=s["res"])
        return [y, tp.dropout_backward(s["dy"], c["p"], s["seed"], s["step"], s["site"])] if c["train"] else [y]
    if c["op"] == "norm":
        if not c["train"]:
            y, v = tp.layer_norm(s["x"], s["w"], s["b"], s["res"], eps=EPS)
            return [y] if s["res"] is None else [v, y]
        y, v, stats = tp.layer_norm(s["x"], s["w"], s["b"], s["res"], eps=EPS, save=True)
        grads = tp.layer_norm_backward(s["dy"], v, s["w"], stats, s["dsum"])
        return ([y] if s["res"] is None else [v, y]) + list(grads if s["b"] is not None else grads[:2])
    q, scale = tp.quantise_f8(s["x"], c["block"])
    if c["out"] == "values":
        return [_values(q, scale, c["block"], TYPES[c["dtype"]]), scale]
    return [tp.product_f8(q, scale, s["w"], s["ws"], s["b"], dtype=TYPES[c["dtype"]])]


def run(state):
    if own:
        return _own(state)
    return {"embed": _plain_embed, "dropout": _plain_dropout, "norm": _plain_norm, "f8": _plain_f8}[state["c"]["op"]](state)


# ------------------------------------------------------- the definitions, fp64
def _exact_embed(s):
    c = s["c"]
    ids = s["ids"].long()
    ids = torch.where(ids < 0, c["vocab"], ids)   # a row of zeros below the table
    table = torch.cat([s["table"].double(), torch.zeros(1, c["d"], device=DEV, dtype=torch.float64)])
    y = c["scale"] * table.index_select(0, ids)
    if not c["train"]:
        return [y]
    # sums of the runs of the sorted ids
    at = torch.argsort(ids, stable=True)
    seen, count = torch.unique_consecutive(ids[at], return_counts=True)
    out = table.zero_()
    out[seen] = torch.segment_reduce(s["dy"].double()[at], "sum", lengths=count, axis=0)
    return [y, c["scale"] * out[:-1]]


def _exact_dropout(s):
    c = s["c"]
    rows, d, p = c["rows"], c["d"], float(np.float32(c["p"]))
    row, col = np.meshgrid(np.arange(rows, dtype=np.uint64), np.arange((d + 3) // 4, dtype=np.uint64), indexing="ij")
    w = [row, col, np.full_like(row, s["step"]), np.full_like(row, s["site"])]
    key, low = np.array([s["seed"] & 0xFFFFFFFF, s["seed"] >> 32], np.uint64), np.uint64(0xFFFFFFFF)
    bump = np.array([0x9E3779B9, 0xBB67AE85], np.uint64)
    for _ in range(10):
        a, b = np.uint64(0xD2511F53) * w[0], np.uint64(0xCD9E8D57) * w[2]
        w = [(b >> np.uint64(32)) ^ w[1] ^ key[0], b & low, (a >> np.uint64(32)) ^ w[3] ^ key[1], a & low]
        key = (key + bump) & low
    keep = np.stack(w, -1).reshape(rows, -1)[:, :d] >= int(p * 4294967296.0)
    keep = torch.from_numpy(keep).to(DEV).double() / (1 - p)
    y = keep * s["x"].double()
    out = [y if s["res"] is None else y + s["res"].double()]
    return out + [keep * s["dy"].double()] if c["train"] else out


def _exact_norm(s):
    c = s["c"]
    v = s["x"].double()
    if s["res"] is not None:
        v = (v + s["res"].double()).to(s["x"].dtype).double()
    leaves = [v.clone().requires_grad_(True), s["w"].double().requires_grad_(True)]
    if s["b"] is not None:
        leaves.append(s["b"].double().requires_grad_(True))
    y = torch.nn.functional.layer_norm(leaves[0], (c["d"],), *leaves[1:], eps=EPS)
    out = [] if s["res"] is None else [v]
    out.append(y.detach())
    if c["train"]:
        grads = list(torch.autograd.grad(y, leaves, s["dy"].double()))
        if s["dsum"] is not None:
            grads[0] = grads[0] + s["dsum"].double()
        out += grads
    return out


def _exact_f8(s):
    c = s["c"]
    x = s["x"].double()
    rows, k = x.shape
    val, scales = torch.empty_like(x), []
    for k0 in range(0, k, BLOCK):
        part = x[:, k0: k0 + BLOCK]
        top = torch.stack([p.abs().max() for p in part.split(c["block"])]) if c["block"] > 1 else part.abs().max(1).values
        top = (top / F8_MAX).float()   # as it is stored
        scales.append(top.double())
        each = top.double().repeat_interleave(c["block"])[:rows, None]
        # to the nearest number of four significant bits, or of steps of 2^-9
        t = torch.where(each > 0, part / each, 0.0)
        step = torch.exp2(torch.floor(torch.log2(t.abs().clamp(min=2.0 ** -6))) - 3)
        val[:, k0: k0 + BLOCK] = torch.round(t / step) * step * each
    if c["out"] == "values":
        return [val, torch.stack(scales, 1)]
    y = torch.zeros(rows, c["n"], dtype=torch.float64, device=DEV)
    for i in range(0, c["n"], BLOCK):
        w = s["w"][i: i + BLOCK].double() * s["ws"][i // BLOCK].double().repeat_interleave(BLOCK)[:k]
        y[:, i: i + BLOCK] = val @ w.T
    return [y if s["b"] is None else y + s["b"].double()]


def exact(case, seed):
    if case["op"] == "f8" and case["out"] == "product" and work(case)["flops"] > 1e12:
        return None
    s = prepare(case, seed)
    return {"embed": _exact_embed, "dropout": _exact_dropout, "norm": _exact_norm, "f8": _exact_f8}[case["op"]](s)
