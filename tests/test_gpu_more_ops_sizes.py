"""Embedding, dropout, layer norm and 8-bit floating point products at the sizes
where a launch goes round its loops again, takes another kernel or shares its
work out differently, with outputs left out, and past 2^31 elements."""
import ctypes
import math
import os
import re

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_gpu_f8 import _check, _operands, _product64, _quantise64  # noqa: E402
from test_gpu_more_ops import (BF, E24, EPS, F32, SEED, TYPES, U, _embed64, _embed_grad64, _gen, _ids, _keep64, _norm64,  # noqa: E402,F401
                               _norm_grad64, _rand, _within, tp)

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------- embedding
# digits of 8, 9 and 10 bits, one to four passes, tiles of two, four and eight rounds
@pytest.mark.parametrize("table_t,out_t", [(F32, BF), (BF, F32)])
@pytest.mark.parametrize("n,vocab,d", [(70001, 300, 3), (70001, 100003, 3), (66000, 1 << 21, 1), (320001, 1 << 20, 2), (400003, 700, 16),
                                       (800440, 1000003, 8), (1300001, 1000003, 1), (1300001, 200, 8), (2500003, 3000, 4),
                                       (200003, 4, 16), (311296, 511, 8), (311297, 512, 8), (1245184, 1023, 4), (1245185, 1024, 4)])
def test_embed_sorts(tp, table_t, out_t, n, vocab, d):  # noqa: F811
    g = _gen(n + vocab + d)
    ids = _ids(g, n, vocab, (torch.int32, torch.int64)[n % 2])
    dy = _rand(g, n, d, out_t)
    dt = tp.embed_backward(dy, ids, vocab, -2.0, dtype=table_t)
    _within(dt, *_embed_grad64(dy, ids, vocab, -2.0, table_t), "dtable")
    assert torch.equal(dt, tp.embed_backward(dy, ids, vocab, -2.0, dtype=table_t))


@pytest.mark.parametrize("n", [200, 3000, 50000, 70000])
def test_embed_largest_vocabulary(tp, n):  # noqa: F811
    """A table of nearly 2^31 rows: the longest keys, tokens on its first and last rows."""
    vocab = (1 << 31) - 4096
    g = _gen(n)
    ids = torch.randint(0, vocab, (n,), generator=g, device="cuda")
    ids[::5], ids[1::7], ids[2::11] = 0, vocab - 1, -1
    ids[3::13], ids[4::17] = vocab, 1 << 40
    dy = _rand(g, n, 1, F32)
    dt = tp.embed_backward(dy, ids, vocab, dtype=BF)
    ok = (ids >= 0) & (ids < vocab)
    at, back = torch.unique(ids[ok], return_inverse=True)
    ref, mag = (torch.zeros(len(at), 1, dtype=torch.float64, device="cuda").index_add_(0, back, v) for v in (dy[ok].double(), dy[ok].double().abs()))
    _within(dt[at], ref, 2.0 ** -16 * mag + U[BF] * ref.abs(), "dtable")
    assert int(torch.count_nonzero(dt)) <= len(at)      # (and nothing anywhere else)


# ------------------------------------------------------------------ dropout
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d,pad,off", [(60001, 24, 0, 0), (4001, 128, 0, 0), (30001, 64, 8, 0), (3001, 264, 0, 0), (2003, 2048, 0, 0),
                                            (400, 20000, 0, 0), (2001, 389, 0, 0), (3001, 389, 3, 0), (700, 2056, 0, 1), (12001, 5, 0, 0)])
def test_dropout_turns(tp, dtype, rows, d, pad, off):  # noqa: F811
    """More rows than run at once."""
    g = _gen(rows + d)
    x, res = _rand(g, rows, d, dtype, 1.0, pad, off), _rand(g, rows, d, dtype, 3.0, pad, off)
    keep = _keep64(np.arange(rows), d, 0.3, SEED, 9, 3)
    ref = torch.where(keep, x.double() / (1 - float(np.float32(0.3))), 0.0)
    _within(tp.dropout(x, 0.3, SEED, 9, 3), ref, (2 * E24 + U[dtype]) * 1.01 * ref.abs(), "y")
    total = ref + res.double()
    _within(tp.dropout(x, 0.3, SEED, 9, 3, residual=res), total,
            1.01 * (2 * E24 * ref.abs() + (E24 + U[dtype]) * (total.abs() + 2 * E24 * ref.abs())), "y + residual")
    total = x.double() + res.double()
    _within(tp.dropout(x, 0.0, SEED, residual=res), total, 1.01 * (E24 + U[dtype]) * total.abs(), "p = 0")


# --------------------------------------------------------------- layer norm
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d", [(6079, 33), (6083, 33), (6085, 255), (3041, 257), (2500, 389), (1600, 1001), (1601, 520), (20011, 8),
                                    (5001, 512), (3001, 1024), (1001, 5120), (700, 6144), (1300, 8192)])
def test_layer_norm_turns(tp, dtype, rows, d):  # noqa: F811
    """More rows than run at once, of one to twenty-four warps a row."""
    g = _gen(rows + d)
    x, res = _rand(g, rows, d, dtype), _rand(g, rows, d, dtype, 3.0)
    w, b = 1 + 0.2 * torch.randn(d, generator=g, device="cuda"), torch.randn(d, generator=g, device="cuda")
    dy, dsum = _rand(g, rows, d, dtype, 0.1), _rand(g, rows, d, dtype, 0.1)
    for rr, bb, ds in ((res, b, dsum), (None, None, None)):
        y, s, stats = tp.layer_norm(x, w, bb, rr, eps=EPS, save=True)
        ref = _norm64(x, w, bb, rr, dtype)
        assert torch.equal(s, ref[0])
        _within(y, ref[6], ref[7], "y")
        got = tp.layer_norm_backward(dy, s, w, stats, ds)
        for name, v, (val, tol) in zip(("dx", "dw", "db"), got, _norm_grad64(dy, w, ds, *ref[2:6], dtype)):
            _within(v, val, tol + 1e-30, name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d", [(5, 64), (300, 2048), (9, 16384), (5, 33), (6091, 33), (1301, 2501), (4103, 1501), (9, 9001)])
def test_layer_norm_outputs_left_out(tp, dtype, rows, d):  # noqa: F811
    """Any output of the library's calls may be NULL; the others are what they are with all."""
    L, prec, g = tp.load_library(), {BF: 0, F32: 1}[dtype], _gen(rows + d)
    x, res, dy, dsum = (_rand(g, rows, d, dtype) for _ in range(4))
    w, b = torch.randn(d, generator=g, device="cuda"), torch.randn(d, generator=g, device="cuda")
    y, s, stats = tp.layer_norm(x, w, b, res, eps=EPS, save=True)
    grads = tp.layer_norm_backward(dy, s, w, stats, dsum)
    p = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    st = torch.cuda.current_stream().cuda_stream
    for keep in range(1, 8):
        out = [torch.full_like(t, -7.0) if keep >> i & 1 else None for i, t in enumerate((s, y, stats))]
        assert L.pack_layer_norm(p(x), d, p(res), d, p(w), p(b), rows, d, EPS, prec, *map(p, out), st) == tp.TP_OK
        for got, want in zip(out, (s, y, stats)):
            assert got is None or torch.equal(got, want)
    n = ctypes.c_int64()
    assert L.pack_layer_norm_bytes(rows, d, ctypes.byref(n)) == tp.TP_OK
    work = torch.empty(n.value, dtype=torch.uint8, device="cuda")
    for keep in range(4):
        out = [torch.full_like(grads[0], -7.0), *(torch.full_like(t, -7.0) if keep >> i & 1 else None for i, t in enumerate(grads[1:]))]
        assert L.pack_layer_norm_backward(p(dy), d, p(s), d, p(w), p(stats), p(dsum), d, rows, d, prec, *map(p, out),
                                          p(work) if keep else None, n.value if keep else 0, st) == tp.TP_OK
        for got, want in zip(out, grads):
            assert got is None or torch.equal(got, want)


# ------------------------------------------------------- 8-bit floating point
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,k,pad,off", [(20011, 520, 0, 0), (20011, 96, 8, 0), (15000, 136, 0, 0), (700, 16384, 0, 0), (9000, 389, 0, 0),
                                            (3000, 2001, 3, 1), (1000, 2048, 0, 0)])
@pytest.mark.parametrize("block", [1, 128])
def test_quantise_turns(tp, dtype, rows, k, pad, off, block):  # noqa: F811
    """More blocks than run at once, with scales of all sizes."""
    g = _gen(rows + k)
    x = torch.randn(rows * (k + pad) + off, generator=g, device="cuda")
    x = (x * torch.exp2(torch.randint(-12, 5, x.shape, generator=g, device="cuda"))).to(dtype)[off:].view(rows, k + pad)[:, :k]
    q, scale = tp.quantise_f8(x, block)
    ref, ref_scale = _quantise64(x, block)
    assert torch.equal(scale, ref_scale) and torch.equal(q.double(), ref)


def _tiles(rows, k, n):
    """(rows, columns, CTAs sharing K, tiles, K blocks a CTA takes) of a tcgen05 product, by the library's own table of times."""
    src = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_05380_gb300", "csrc", "f8.cu")).read()
    table = re.search(r"kShapes\[\] = \{(.*?)\};", src, re.S).group(1)
    best, kb = None, -(-k // 128)
    for row in re.findall(r"\{([^{}]*)\}", table):
        r, c, split, t, t_full, fixed, epi = map(float, row.split(","))
        tiles, at_once = math.ceil(rows / r) * math.ceil(n / c), 152 // int(r / 128 * split)
        if split > 1 and (tiles > at_once or kb < split):
            continue
        waves = math.ceil(tiles / at_once)
        time = fixed + waves * math.ceil(kb / split) * (t_full if tiles > at_once else t) + (waves - 1) * epi
        if best is None or time < best[0]:
            best = time, (int(r), int(c), int(split)), tiles / at_once, kb // split
    return best[1:]


# The tile that each takes, how many waves of them and how many K blocks, six of which are in flight: rings go round, accumulators
# are used again, a CTA takes a second and third tile; with remainders in all three sizes.
PRODUCTS = [((8192, 4096, 4096), (256, 256, 1), 6, 32), ((3003, 2001, 3000), (256, 256, 1), 1, 16), ((9001, 1100, 2555), (256, 256, 1), 4, 9),
            ((5003, 1800, 2100), (128, 128, 1), 4, 15), ((2600, 3000, 2056), (128, 128, 1), 2, 24), ((1500, 2000, 1003), (128, 128, 1), 0, 16),
            ((500, 2001, 1003), (128, 64, 2), 0, 8), ((500, 2001, 2003), (128, 64, 1), 0, 16), ((290, 8000, 500), (128, 64, 4), 0, 15)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape,tile,waves,depth", PRODUCTS)
def test_product_turns(tp, dtype, shape, tile, waves, depth):  # noqa: F811
    took = _tiles(*shape)
    assert took[0] == tile and took[1] > waves and took[2] >= depth, took
    rows, k, n = shape
    q, s, w, ws, b = _operands(tp, rows, k, n, rows + k + n)
    y = tp.product_f8(q, s, w, ws, b, dtype=dtype)
    _check(y, *_product64(q, s, w, ws, b, dtype))
    for _ in range(3):
        assert torch.equal(y, tp.product_f8(q, s, w, ws, b, dtype=dtype))
    tp.ops_check()


# ------------------------------------------------------- past 2^31 elements
def _parts(rows, d):
    """The first rows, those around element 2^31 and the last ones."""
    mid = (1 << 31) // d
    return [slice(0, 40), slice(mid - 20, min(rows, mid + 20)), slice(rows - 40, rows)]


def _big(g, rows, d, dtype, scale=1.0):
    t = torch.empty(rows, d, dtype=dtype, device="cuda")
    for part in t.split(1 << 16):
        part.copy_(torch.randn(part.shape, generator=g, device="cuda") * scale)
    return t


@pytest.mark.parametrize("d", [512, 513])
def test_embed_many_elements(tp, d):  # noqa: F811
    n, vocab = 4200007, 1003
    g = _gen(d)
    ids = torch.arange(n, device="cuda") % (vocab - 3)
    ids[-3:] = torch.arange(vocab - 3, vocab, device="cuda")
    table, dy = _rand(g, vocab, d, F32), _big(g, n, d, BF)
    y = tp.embed(ids, table, 0.5, dtype=BF)
    for p in _parts(n, d):
        _within(y[p], *_embed64(ids[p], table, 0.5, BF), "y")
    del y
    dt = tp.embed_backward(dy, ids, vocab, 0.5)
    ref, mag = (torch.zeros(vocab, d, dtype=torch.float64, device="cuda") for _ in range(2))
    for i, v in zip(ids.split(1 << 18), dy.split(1 << 18)):
        ref.index_add_(0, i, v.double()), mag.index_add_(0, i, v.double().abs())
    _within(dt, ref / 2, 2.0 ** -16 * mag + 1.01 * 2 * E24 * ref.abs(), "dtable")
    assert torch.equal(dt[-3:], dy[-3:].float() * 0.5)


@pytest.mark.parametrize("d", [512, 513])
@pytest.mark.parametrize("n", [100, 5000, 70000])
def test_embed_large_table(tp, n, d):  # noqa: F811
    vocab = 4200007
    g = _gen(n + d)
    table, dy = _big(g, vocab, d, BF), _rand(g, n, d, F32)
    ids = torch.randint(0, vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
    ids[:3] = torch.tensor([vocab - 1, vocab - 2, (1 << 31) // d], device="cuda")
    ids[50:60] = vocab - 1
    _within(tp.embed(ids, table, 3.0, dtype=F32), *_embed64(ids, table[:, :], 3.0, F32), "y")
    del table
    dt = tp.embed_backward(dy, ids, vocab, 3.0, dtype=BF)
    at, back = torch.unique(ids.long(), return_inverse=True)
    ref, mag = (torch.zeros(len(at), d, dtype=torch.float64, device="cuda").index_add_(0, back, v) for v in (dy.double(), dy.double().abs()))
    _within(dt[at], 3 * ref, 3 * 2.0 ** -16 * mag + 1.01 * (U[BF] + E24) * 3 * ref.abs(), "dtable")
    none = torch.ones(vocab, dtype=torch.bool, device="cuda")
    none[at] = False
    for m, p in zip(none.split(1 << 18), dt.split(1 << 18)):
        assert not p[m].any()


@pytest.mark.parametrize("d", [2056, 2051])
def test_dropout_many_elements(tp, d):  # noqa: F811
    rows = (1 << 20) + 37
    g = _gen(d)
    x = _big(g, rows, d, BF)
    y = tp.dropout(x, 0.25, SEED, 1, 2, residual=x)
    for p in _parts(rows, d):
        keep = _keep64(np.arange(p.start, p.stop), d, 0.25, SEED, 1, 2)
        ref = x[p].double() * torch.where(keep, 1 + 1 / 0.75, 1.0)
        _within(y[p], ref, 1.02 * (4 * E24 + U[BF]) * ref.abs(), "y")


@pytest.mark.parametrize("d,dtype", [(8192, BF), (4097, BF), (4097, F32), (1000, BF), (389, F32)])
def test_layer_norm_many_elements(tp, d, dtype):  # noqa: F811
    rows = (1 << 31) // d + 77
    g = _gen(d)
    x, dy = _big(g, rows, d, dtype), _big(g, rows, d, dtype, 0.1)
    w, b = 1 + 0.2 * torch.randn(d, generator=g, device="cuda"), torch.randn(d, generator=g, device="cuda")
    y, s, stats = tp.layer_norm(x, w, b, x, eps=EPS, save=True)
    dx, dw, db = tp.layer_norm_backward(dy, s, w, stats)
    for p in _parts(rows, d):
        ref = _norm64(x[p], w, b, x[p], dtype)
        assert torch.equal(s[p], ref[0])
        _within(y[p], ref[6], ref[7], "y")
        _within(dx[p], *_norm_grad64(dy[p], w, None, *ref[2:6], dtype)[0], "dx")
    sums = [torch.zeros(d, dtype=torch.float64, device="cuda") for _ in range(4)]
    for v, t, m in zip(s.split(1 << 14), dy.split(1 << 14), stats.split(1 << 14)):
        h, t = (v.double() - m[:, :1].double()) * m[:, 1:].double(), t.double()
        for a, q in zip(sums, ((t * h).sum(0), (t * h).abs().sum(0), t.sum(0), t.abs().sum(0))):
            a += q
    chain = (rows / 128 + 128) * E24      # a block's rows one after another
    _within(dw, sums[0], 1.01 * (chain + 8 * E24) * sums[1], "dw")
    _within(db, sums[2], 1.01 * chain * sums[3], "db")


@pytest.mark.parametrize("d", [2056, 2051])
@pytest.mark.parametrize("block", [1, 128])
def test_quantise_many_elements(tp, d, block):  # noqa: F811
    rows = (1 << 20) + 128
    x = _big(_gen(d), rows, d, BF)
    q, scale = tp.quantise_f8(x, block)
    for p in _parts(rows, d):
        p = slice(p.start // block * block, -(-p.stop // block) * block)
        ref, ref_scale = _quantise64(x[p], block)
        assert torch.equal(scale[p.start // block: p.stop // block], ref_scale) and torch.equal(q[p].double(), ref)


@pytest.mark.parametrize("n,dtype", [(2056, BF), (2051, BF), (2051, F32)])
def test_product_many_elements(tp, n, dtype):  # noqa: F811
    rows = (1 << 20) + 37
    q, s, w, ws, b = _operands(tp, rows, 200, n, n)
    y = tp.product_f8(q, s, w, ws, b, dtype=dtype)
    for p in _parts(rows, n):
        _check(y[p], *_product64(q[p], s[p], w, ws, b, dtype))
    tp.ops_check()
