"""Embedding lookup, dropout and layer norm, with their gradients, against
their formulas in 64 bits over types, sizes, strides, masks and empty calls.

Bounds are derived, not fitted: ``U`` is half a step of the output type, one
rounding; ``C`` = 2^-18 bounds an fp32 sum whose longest chain is 64 additions
(2^-24 each) relative to the sum of its terms' magnitudes.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
U = {BF: 2.0 ** -8, F32: 2.0 ** -24}
C = 2.0 ** -18
E24 = 2.0 ** -24
TYPES = [BF, F32]


@pytest.fixture(scope="module")
def tp():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_05380_gb300 import build
    build.build()
    import paper_2607_05380_gb300 as tpm
    tpm.load_library()
    return tpm


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _rand(g, rows, cols, dtype, scale=1.0, pad=0, off=0):
    """Rows `pad` elements apart that start `off` elements into the memory."""
    t = torch.randn(rows * (cols + pad) + off, generator=g, device="cuda") * scale
    return t.to(dtype)[off:].view(rows, cols + pad)[:, :cols]


def _within(got, ref, tol, what):
    assert got.shape == ref.shape, what
    assert torch.isfinite(got).all(), what
    over = ((got.double() - ref).abs() - tol).max() if got.numel() else torch.tensor(-1.0)
    assert float(over) <= 0, (what, float(over), float((got.double() - ref).abs().max()))


# ---------------------------------------------------------------- embedding
def _embed64(ids, table, scale, out):
    scale = float(np.float32(scale))
    ok = (ids >= 0) & (ids < table.shape[0])
    y = torch.where(ok[..., None], table.double()[torch.where(ok, ids, 0).long()] * scale, 0.0)
    return y, (E24 + U[out]) * y.abs() * 1.01


def _embed_grad64(dy, ids, vocab, scale, out):
    """Values and bounds: chains of at most 64 additions on each of at most four levels, one rounding by the scale, one
    to the output's type."""
    scale = float(np.float32(scale))
    ok = (ids >= 0) & (ids < vocab)
    at, dy = torch.where(ok, ids, vocab).long(), dy.double()
    g, mag = (torch.zeros(vocab + 1, dy.shape[1], dtype=torch.float64, device="cuda") for _ in range(2))
    g.index_add_(0, at, dy), mag.index_add_(0, at, dy.abs())
    g, mag = g[:vocab] * scale, mag[:vocab] * abs(scale)
    return g, 4 * C * mag + (E24 + U[out]) * g.abs() * 1.01


EMBED = [(1, 1, 1), (1, 1000, 64), (7, 3, 5), (13, 1000, 8), (32, 2, 33), (100, 70, 128), (4096, 4096, 16), (4097, 37, 24),
         (5000, 300, 33), (3000, 20011, 64), (9000, 1025, 40), (20011, 100003, 8), (50000, 5, 12), (70000, 2, 64),
         (40000, 1, 1), (777, 50, 1024), (300, 17, 1000), (65, 9, 4099), (16384, 1 << 20, 4),
         (1024, 1, 8), (1025, 1 << 21, 2), (16385, 700, 40), (32769, 1023, 16), (65536, 1024, 8), (65537, 40000, 8),
         (65000, 3, 264), (150000, 2047, 33), (256, 2000, 3), (257, 9, 7), (1000, 3000, 194), (2048, 5, 1),
         (20000, 49, 1), (13, 70001, 21), (200000, 6, 2), (5, 1000, 1021)]


def _ids(g, n, vocab, dtype, missing=0.1):
    v = (vocab * torch.rand(n, generator=g, device="cuda", dtype=torch.float64) ** 2).long().clamp(max=vocab - 1)
    r = torch.rand(n, generator=g, device="cuda")
    v = torch.where(r < missing, -1, v)
    v = torch.where((r >= missing) & (r < 1.2 * missing), vocab, v)     # one past the end
    return v.to(dtype)


@pytest.mark.parametrize("types", [(F32, BF), (BF, BF), (F32, F32), (BF, F32)])
@pytest.mark.parametrize("shape", EMBED)
def test_embed(tp, types, shape):
    n, vocab, d = shape
    table_t, out_t = types
    g = _gen(n + vocab + d)
    ids = _ids(g, n, vocab, (torch.int32, torch.int64)[n % 2])
    table, dy = _rand(g, vocab, d, table_t), _rand(g, n, d, out_t)
    scale = (1.0, 0.3, -8.0)[d % 3]
    y = tp.embed(ids, table, scale, dtype=out_t)
    assert y.dtype == out_t
    _within(y, *_embed64(ids, table, scale, out_t), "y")
    dt = tp.embed_backward(dy, ids, vocab, scale, dtype=table_t)
    assert dt.dtype == table_t
    _within(dt, *_embed_grad64(dy, ids, vocab, scale, table_t), "dtable")
    assert torch.equal(dt, tp.embed_backward(dy, ids, vocab, scale, dtype=table_t))


@pytest.mark.parametrize("types", [(F32, BF), (BF, BF), (F32, F32), (BF, F32)])
@pytest.mark.parametrize("n,d", [(8191, 33), (8192, 33), (8193, 1), (8200, 1025), (9001, 3), (40001, 129), (70003, 7)])
def test_embed_odd_widths(tp, types, n, d):
    """Rows of odd widths, many and not quite as many: a float32 product, rounded to the output's type."""
    g = _gen(n + d)
    ids = _ids(g, n, 500, torch.int32)
    table = _rand(g, 500, d, types[0])
    ok = (ids >= 0) & (ids < 500)
    want = torch.where(ok[:, None], table.float()[torch.where(ok, ids, 0).long()] * 0.3, 0.0).to(types[1])
    assert torch.equal(tp.embed(ids, table, 0.3, dtype=types[1]), want)


@pytest.mark.parametrize("pad,off", [(8, 0), (3, 0), (0, 1), (5, 3)])
def test_embed_strides(tp, pad, off):
    """Spaced rows, odd addresses and ids of more than one dimension give the same values."""
    g = _gen(pad + off)
    ids = _ids(g, 60 * 7, 90, torch.int64)
    for t in TYPES:
        table, dy = _rand(g, 90, 72, t, pad=pad, off=off), _rand(g, 420, 72, t, pad=pad, off=off)
        y = tp.embed(ids.view(60, 7), table)
        assert y.shape == (60, 7, 72) and y.dtype == t
        assert torch.equal(y.view(420, 72), tp.embed(ids, table.contiguous()))
        _within(tp.embed_backward(dy, ids.view(60, 7), 90), *_embed_grad64(dy, ids, 90, 1.0, F32), "dtable")
        packed = dy.contiguous().clone()
        assert torch.equal(tp.embed_backward(packed.view(60, 7, 72), ids.view(60, 7), 90), tp.embed_backward(packed, ids, 90))


@pytest.mark.parametrize("n", [5, 4096, 4097, 30000])
def test_embed_one_id(tp, n):
    """All tokens alike, all missing, all different."""
    g = _gen(n)
    dy = _rand(g, n, 48, F32)
    for ids in (torch.full((n,), 3), torch.full((n,), -1), torch.full((n,), 8), torch.arange(n)):
        ids = ids.cuda()
        vocab = max(8, n) if int(ids[-1]) == n - 1 else 8
        _within(tp.embed_backward(dy, ids, vocab), *_embed_grad64(dy, ids, vocab, 1.0, F32), "dtable")


def test_embed_special(tp):
    """NaN and infinities stay on the rows that hold them; ids far outside count as missing; no tokens."""
    g = _gen(1)
    table = _rand(g, 40, 16, F32)
    table[3], table[4] = float("nan"), float("inf")
    ids = torch.tensor([1, 3, 4, -1, 2 ** 40, -2 ** 40, 2 ** 32 + 1, 2], device="cuda")
    y = tp.embed(ids, table)
    assert torch.isnan(y[1]).all() and torch.isinf(y[2]).all() and (y[3:7] == 0).all()
    assert torch.equal(y[[0, 7]], table[[1, 2]])
    dy = torch.ones(8, 16, device="cuda")
    dy[3:7] = float("nan")   # of missing ids: not looked at
    dy[0, 0] = float("inf")
    dt = tp.embed_backward(dy, ids, 40)
    assert torch.isfinite(dt).sum() == 40 * 16 - 1 and dt[1, 0] == float("inf")
    assert float(dt[[2, 3, 4]].sum()) == 48 and float(dt.sum(1)[5:].abs().sum()) == 0
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    assert tp.embed(none, table).shape == (0, 16)
    assert torch.equal(tp.embed_backward(torch.empty(0, 16, device="cuda"), none, 7), torch.zeros(7, 16, device="cuda"))


# ------------------------------------------------------------------ dropout
def _keep64(rows, d, p, seed, step, site):
    """Philox4x32-10 by its definition, in 64-bit integers."""
    row, col = np.meshgrid(np.asarray(rows, np.uint64), np.arange((d + 3) // 4, dtype=np.uint64), indexing="ij")
    w = [row, col, np.full_like(row, step), np.full_like(row, site)]
    k0, k1, low, half = np.uint64(seed & 0xFFFFFFFF), np.uint64(seed >> 32), np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(10):
        a, b = np.uint64(0xD2511F53) * w[0], np.uint64(0xCD9E8D57) * w[2]
        w = [(b >> half) ^ w[1] ^ k0, b & low, (a >> half) ^ w[3] ^ k1, a & low]
        k0, k1 = (k0 + np.uint64(0x9E3779B9)) & low, (k1 + np.uint64(0xBB67AE85)) & low
    words = np.stack(w, -1).reshape(len(rows), -1)[:, :d]
    return torch.from_numpy(words >= int(float(np.float32(p)) * 2 ** 32)).cuda()


SEED = 0x123456789ABCDEF1


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d,pad,off", [(1, 1, 0, 0), (1, 8, 0, 0), (3, 5, 0, 0), (37, 33, 3, 1), (5, 64, 0, 0), (130, 128, 0, 1),
                                            (100, 389, 3, 0), (257, 1000, 8, 0), (64, 2048, 0, 0), (9, 2056, 0, 0),
                                            (2, 131072, 0, 0), (2000, 24, 0, 0)])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.999])
def test_dropout(tp, dtype, rows, d, pad, off, p):
    g = _gen(rows + d)
    x, res = _rand(g, rows, d, dtype, 1.0, pad, off), _rand(g, rows, d, dtype, 3.0, pad, off)
    keep = _keep64(np.arange(rows), d, p, SEED, 7 + d, 0xF0000005)
    up = 1 / (1 - float(np.float32(p)))
    ref = torch.where(keep, x.double() * up, 0.0)
    y = tp.dropout(x, p, SEED, 7 + d, 0xF0000005)
    _within(y, ref, (2 * E24 + U[dtype]) * 1.01 * ref.abs(), "y")   # the factor's rounding, the product's, the result's
    assert torch.equal(y, tp.dropout_backward(x, p, SEED, 7 + d, 0xF0000005))
    both = tp.dropout(x, p, SEED, 7 + d, 0xF0000005, residual=res)
    total = ref + res.double()
    _within(both, total, 1.01 * (2 * E24 * ref.abs() + (E24 + U[dtype]) * (total.abs() + 2 * E24 * ref.abs())), "y + residual")


def test_dropout_masks(tp):
    """Dropped places do not matter; other seeds, steps and sites, other masks; the rate."""
    x = torch.ones(400, 500, device="cuda")
    base = tp.dropout(x, 0.3, 5, 1, 2)
    assert abs(float((base == 0).float().mean()) - 0.3) < 6 * (0.21 / 200000) ** 0.5
    bad = torch.where(base == 0, float("nan"), x)
    assert torch.equal(tp.dropout(bad, 0.3, 5, 1, 2), base)
    for other in ((6, 1, 2), (5, 0, 2), (5, 1, 3), (5 + 2 ** 32, 1, 2)):
        assert float(((tp.dropout(x, 0.3, *other) == 0) != (base == 0)).float().mean()) > 0.3
    assert tp.dropout(x[:0], 0.3, 5).shape == (0, 500)


def test_dropout_is_the_packs(tp):
    """The rule of a pack's masks: site (member << 4) | layer."""
    pack = tp.Pack(8, 3, "multiclass", [2, 1], [64, 32], [0.25, 0.5], [1e-3, 1e-3], [0.0, 0.0], max_batch=32, seed=99)
    try:
        for member, layer, width, p in ((0, 0, 64, 0.25), (0, 1, 64, 0.25), (1, 0, 32, 0.5)):
            mask = torch.as_tensor(np.asarray(pack.debug_masks(member, layer, 11, 32)).reshape(32, width)).cuda()
            y = tp.dropout(torch.ones(32, width, device="cuda"), p, 99, 11, (member << 4) | layer)
            assert torch.equal(y != 0, mask != 0)
    finally:
        pack.close()


# --------------------------------------------------------------- layer norm
EPS = 1e-5


def _norm64(x, w, b, res, dtype):
    """s as it is stored, its mean, r, h and their error bounds, y and its bound."""
    s = x if res is None else (x.float() + res.float()).to(dtype)
    v, w = s.double(), w.double()
    mean = v.mean(1, keepdim=True)
    em = C * v.abs().mean(1, keepdim=True) + E24 * mean.abs()
    c = v - mean
    ec = em + E24 * (c.abs() + em)
    var = (c * c).mean(1, keepdim=True)
    ev = (2 * c.abs() * ec + ec * ec).mean(1, keepdim=True) + 2 * C * var
    r = 1 / torch.sqrt(var + EPS)
    er = 0.5 * ev / (var + EPS) + 8 * E24          # relative (the square root and the quotient round, too)
    h = c * r
    eh = (r * ec + h.abs() * er + E24 * h.abs()) * 1.01
    y = h * w + (0 if b is None else b.double())
    ey = eh * w.abs() + 2 * E24 * ((h * w).abs() + y.abs()) + U[dtype] * y.abs()
    return s, mean, r, er, h, eh, y, 1.02 * ey


def _norm_grad64(dy, w, dsum, r, er, h, eh, dtype):
    dy, w = dy.double(), w.double()
    t = dy * w
    m0, m1 = t.mean(1, keepdim=True), (t * h).mean(1, keepdim=True)
    e0 = 2 * C * t.abs().mean(1, keepdim=True)
    e1 = 2 * C * (t * h).abs().mean(1, keepdim=True) + (t.abs() * eh).mean(1, keepdim=True)
    q = t - m0 - h * m1
    eq = E24 * 4 * (t.abs() + m0.abs() + (h * m1).abs()) + e0 + h.abs() * e1 + eh * (m1.abs() + e1)
    dx = r * q + (0 if dsum is None else dsum.double())
    ex = r * eq * 1.01 + (er + 2 * E24) * (r * q).abs() + (U[dtype] + E24) * dx.abs()
    dw, db = (dy * h).sum(0), dy.sum(0)
    return [(dx, 1.02 * ex), (dw, 1.01 * ((dy.abs() * eh).sum(0) + 2 * C * (dy * h).abs().sum(0))), (db, 2 * C * dy.abs().sum(0))]


NORM_D = [1, 3, 8, 33, 64, 256, 257, 264, 512, 1000, 1024, 1032, 2048, 2049, 4096, 5001, 8192, 8200, 16384, 16383]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", NORM_D)
@pytest.mark.parametrize("rows", [1, 5, 67])
def test_layer_norm(tp, dtype, d, rows):
    g = _gen(rows + d)
    x, res = _rand(g, rows, d, dtype), _rand(g, rows, d, dtype, 3.0)
    w, b = 1 + 0.2 * torch.randn(d, generator=g, device="cuda"), torch.randn(d, generator=g, device="cuda")
    dy, dsum = _rand(g, rows, d, dtype, 0.1), _rand(g, rows, d, dtype, 0.1)
    for with_res in (True, False):
        rr, bb, ds = (res, b, dsum) if with_res else (None, None, None)
        y, s, stats = tp.layer_norm(x, w, bb, rr, eps=EPS, save=True)
        ref = _norm64(x, w, bb, rr, dtype)
        assert torch.equal(s, ref[0])
        _within(y, ref[6], ref[7], "y")
        plain = tp.layer_norm(x, w, bb, rr, eps=EPS)
        assert torch.equal(plain[0], y) and torch.equal(plain[1], s)
        got = tp.layer_norm_backward(dy, s, w, stats, ds)
        for name, v, (val, tol) in zip(("dx", "dw", "db"), got, _norm_grad64(dy, w, ds, *ref[2:6], dtype)):
            _within(v, val, tol + 1e-30, name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d", [(3000, 256), (2500, 1000), (1500, 2048), (700, 4100), (400, 9000)])
def test_layer_norm_many_rows(tp, dtype, rows, d):
    """More rows than the backward pass has blocks; rows far from zero."""
    g = _gen(rows)
    x = (_rand(g, rows, d, F32) + 100 * _rand(g, rows, 1, F32)).to(dtype)
    w, b = 1 + 0.2 * torch.randn(d, generator=g, device="cuda"), torch.randn(d, generator=g, device="cuda")
    dy = _rand(g, rows, d, dtype, 0.1)
    y, s, stats = tp.layer_norm(x, w, b, eps=EPS, save=True)
    ref = _norm64(x, w, b, None, dtype)
    _within(y, ref[6], ref[7], "y")
    for name, v, (val, tol) in zip(("dx", "dw", "db"), tp.layer_norm_backward(dy, s, w, stats),
                                   _norm_grad64(dy, w, None, *ref[2:6], dtype)):
        _within(v, val, tol, name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,off", [(8, 0), (3, 0), (0, 1), (5, 3)])
def test_layer_norm_strides(tp, dtype, pad, off):
    """Spaced rows and odd addresses: the same sums in another order."""
    g = _gen(pad)
    rows, d = 45, 520
    x, res, dy, dsum = (_rand(g, rows, d, dtype, pad=pad, off=off) for _ in range(4))
    w, b = (torch.randn(d + 1, generator=g, device="cuda")[off % 2: d + off % 2] for _ in range(2))
    y, s, stats = tp.layer_norm(x, w, b, res, eps=EPS, save=True)
    ref = _norm64(x, w, b, res, dtype)
    assert torch.equal(s, ref[0])
    _within(y, ref[6], ref[7], "y")
    wide = torch.empty(rows, d + pad, dtype=dtype, device="cuda")[:, :d].copy_(s)
    for name, v, (val, tol) in zip(("dx", "dw", "db"), tp.layer_norm_backward(dy, wide, w, stats, dsum),
                                   _norm_grad64(dy, w, dsum, *ref[2:6], dtype)):
        _within(v, val, tol, name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,pad,off,dsum_off", [
    (1025, 0, 0, 0), (2039, 0, 0, 0), (2041, 8, 0, 0), (2500, 16, 0, 0), (4087, 0, 0, 0), (4088, 0, 7, 7), (4089, 8, 0, 0),
    (5001, 0, 0, 0), (5111, 0, 0, 1), (5113, 24, 0, 0), (6135, 0, 0, 8), (6137, 0, 0, 0), (8183, 0, 0, 0), (8185, 0, 0, 0)])
@pytest.mark.parametrize("rows", [63, 1301, 4103])
def test_layer_norm_odd_widths(tp, dtype, d, pad, off, dsum_off, rows):
    """Rows that begin at every place of a 16-byte group: a store that left its row would spoil the next one."""
    g = _gen(d + rows)
    x, res, dy = (_rand(g, rows, d, dtype, pad=pad, off=off) for _ in range(3))
    dsum = _rand(g, rows, d, dtype, pad=pad, off=dsum_off)
    w, b = 1 + 0.2 * torch.randn(d, generator=g, device="cuda"), torch.randn(d, generator=g, device="cuda")
    for with_res in (True, False):
        rr, bb, ds = (res, b, dsum) if with_res else (None, None, None)
        y, s, stats = tp.layer_norm(x, w, bb, rr, eps=EPS, save=True)
        ref = _norm64(x, w, bb, rr, dtype)
        assert torch.equal(s, ref[0])
        _within(y, ref[6], ref[7], "y")
        keep = torch.zeros(rows * (d + pad) + 16, dtype=dtype, device="cuda")[off:][:rows * (d + pad)].view(rows, d + pad)[:, :d]
        keep.copy_(s)
        got = tp.layer_norm_backward(dy, keep, w, stats, ds)
        for name, v, (val, tol) in zip(("dx", "dw", "db"), got, _norm_grad64(dy, w, ds, *ref[2:6], dtype)):
            _within(v, val, tol + 1e-30, name)
        again = tp.layer_norm_backward(dy, keep, w, stats, ds)
        assert all(torch.equal(p, q) for p, q in zip(got, again))


def test_layer_norm_differences(tp):
    """The gradients against differences of the forward pass (fp32)."""
    g = _gen(2)
    rows, d = 3, 40
    x, dy = _rand(g, rows, d, F32), _rand(g, rows, d, F32)
    w, b = torch.randn(d, generator=g, device="cuda"), torch.randn(d, generator=g, device="cuda")
    _, s, stats = tp.layer_norm(x, w, b, eps=EPS, save=True)
    dx, dw, db = tp.layer_norm_backward(dy, s, w, stats)
    loss = lambda x, w, b: float((tp.layer_norm(x, w, b, eps=EPS)[0].double() * dy.double()).sum())  # noqa: E731
    step = 2.0 ** -7
    for name, grad, at in (("x", dx, 0), ("w", dw, 1), ("b", db, 2)):
        v = torch.randn(grad.shape, generator=g, device="cuda")
        up, down = [x, w, b], [x, w, b]
        up[at], down[at] = up[at] + step * v, down[at] - step * v
        diff = (loss(*up) - loss(*down)) / (2 * step)
        want = float((grad.double() * v.double()).sum())
        # the third derivative's part (step^2) and the outputs' rounding over the step
        assert abs(diff - want) <= 2e-3 * float((grad.double() * v.double()).abs().sum()), name


def test_layer_norm_special(tp):
    """Infinities and NaN stay in their rows; constant rows; no rows."""
    g = _gen(3)
    for d in (48, 1500):
        x = _rand(g, 6, d, F32)
        x[1, 5], x[2, 6] = float("nan"), float("inf")
        x[3] = 2.5
        w, b = torch.ones(d, device="cuda"), torch.zeros(d, device="cuda")
        y, s, stats = tp.layer_norm(x, w, b, save=True)
        assert torch.isnan(y[1]).all() and torch.isnan(y[2]).all()
        assert (y[3] == 0).all() and torch.isfinite(y[[0, 3, 4, 5]]).all()
        dx, dw, db = tp.layer_norm_backward(torch.ones_like(x), s, w, stats)
        assert torch.isfinite(dx[[0, 3, 4, 5]]).all() and torch.isnan(dx[1]).all()
        y, s, stats = tp.layer_norm(x[:0], w, b, save=True)
        assert y.shape == (0, d) and stats.shape == (0, 2)
        dx, dw, db = tp.layer_norm_backward(x[:0], s, w, stats)
        assert dx.shape == (0, d) and (dw == 0).all() and (db == 0).all()
