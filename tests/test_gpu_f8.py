"""Quantisation into e4m3 with scales per block of 128, and the product of such
operands, against their definitions in 64 bits.

The quantised values are compared bit for bit.  A product's bound: a K block's
128 products, exact each, are added with 2^-24 of the sum of their magnitudes
lost at most per addition of the tensor cores' tree (2^-17 in all), times two
scales (2^-23), added up over at most 64 blocks (2^-18), rounded once.
"""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32, F8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
U = {BF: 2.0 ** -8, F32: 2.0 ** -24}
BOUND = 2.0 ** -17 + 2.0 ** -23 + 2.0 ** -18
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


def _spread(scale, block, rows, k):
    s = scale.double().repeat_interleave(128, 1)[:, :k]
    return s if block == 1 else s.repeat_interleave(block, 0)[:rows]


def _quantise64(x, block):
    """By the definition: the e4m3 numbers 0, +-2^-9 m, +-2^(e-3) (8 + m), the nearest one, ties to even."""
    rows, k = x.shape
    br, bk = -(-rows // block), -(-k // 128)
    full = torch.zeros(br * block, bk * 128, dtype=torch.float64, device="cuda")
    full[:rows, :k] = x.double()
    scale = (full.view(br, block, bk, 128).abs().amax((1, 3)) / 448).float()
    each = _spread(scale, block, rows, k)
    t = torch.where(each > 0, x.double() / torch.where(each > 0, each, 1.0), 0.0)
    step = ((torch.frexp(t).exponent.long().clamp(min=-5) - 4 + 1023) << 52).view(torch.float64)   # 2^(e - 4)
    return (torch.round(t / step) * step).clamp(-448, 448), scale


def _values(q, scale, block):
    return q.double() * _spread(scale, block, *q.shape)


SHAPES = [(1, 1), (1, 128), (3, 8), (5, 130), (129, 256), (200, 1000), (64, 2001), (37, 127), (500, 129), (1, 4096), (1000, 64)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("pad,off", [(0, 0), (3, 1)])
def test_quantise(tp, dtype, block, shape, pad, off):
    rows, k = shape
    g = _gen(rows + k)
    for kind in ("normal", "ties", "wide"):
        x = torch.randn(rows * (k + pad) + off, generator=g, device="cuda")
        if kind == "ties":      # multiples of a 32nd up to 448, whose quotients by a scale of one lie on the borders
            x = torch.round(x * 2000).clamp(-448 * 32, 448 * 32) / 32
            x[off] = 448
        if kind == "wide":
            x = x * torch.exp2(torch.randint(-12, 5, x.shape, generator=g, device="cuda"))
        x = x.to(dtype)[off:].view(rows, k + pad)[:, :k]
        q, scale = tp.quantise_f8(x, block)
        ref, ref_scale = _quantise64(x, block)
        assert q.dtype == F8 and q.shape == x.shape and torch.equal(scale, ref_scale)
        assert torch.equal(q.double(), ref), kind


def test_quantise_special(tp):
    """Zero blocks, infinities, NaN, the largest and smallest numbers, each in its own block; no rows."""
    x = torch.zeros(6, 300, device="cuda")
    x[1, 5], x[1, 200], x[2, 0], x[3, 299] = float("inf"), 7.0, float("nan"), float("-inf")
    x[4, :4] = torch.tensor([3.4e38, -3.4e38, 1e38, 1e-38], device="cuda")
    x[4, 128:132] = torch.tensor([1e-37, -2e-37, 3e-38, 1e-39], device="cuda")
    x[4, 256:260] = torch.tensor([1e-44, 2e-45, 3e-45, 0.0], device="cuda")
    x[5, :3] = torch.tensor([2.0 ** -64, 2.0 ** -65, -2.0 ** -70], device="cuda")
    q, s = tp.quantise_f8(x)
    bad = torch.zeros(6, 3, dtype=torch.bool, device="cuda")
    bad[1, 0] = bad[2, 0] = bad[3, 2] = True
    assert torch.equal(torch.isnan(s), bad)
    assert float(q[1, :128].double().abs().sum()) == 0 and float(q[3, 256:].double().abs().sum()) == 0
    assert float(q[1, 200].double()) == 448 and float(s[0].sum()) == 0
    ok = ~bad.repeat_interleave(128, 1)[:, :300]
    ref, rs = _quantise64(torch.where(torch.isfinite(x), x, 0.0), 1)
    assert torch.equal(q.double()[ok], ref[ok]) and torch.equal(s[~bad], rs[~bad])
    q, s = tp.quantise_f8(x[:0])
    assert q.shape == (0, 300) and s.shape == (0, 3)


PRODUCT = [(1, 16, 16), (1, 1, 1), (2, 2048, 300), (7, 100, 130), (31, 300, 1000), (33, 2001, 257), (100, 128, 128), (128, 512, 384),
           (129, 640, 129), (300, 1000, 1000), (500, 2001, 1003), (513, 256, 2048), (1000, 130, 4096), (2048, 1024, 1024),
           (4100, 384, 520), (260, 4096, 64), (16, 8192, 40), (64, 1152, 8192), (20011, 128, 136)]


def _operands(tp, rows, k, n, seed, dtype=F32):
    g = _gen(seed)
    x = torch.randn(rows, k, generator=g, device="cuda")
    x *= torch.where(torch.rand(k, generator=g, device="cuda") < 0.05, 20.0, 1.0)
    w = torch.randn(n, k, generator=g, device="cuda") * torch.exp2(torch.randint(-3, 3, (n, 1), generator=g, device="cuda"))
    q, s = tp.quantise_f8(x.to(dtype))
    wq, ws = tp.quantise_f8(w, 128)
    return q, s, wq, ws, torch.randn(n, generator=g, device="cuda")


def _product64(q, s, w, ws, bias, dtype):
    x, v = _values(q, s, 1), _values(w, ws, 128)
    y = x @ v.T
    tol = BOUND * (x.abs() @ v.abs().T)
    if bias is not None:
        y = y + bias.double()
        tol = tol + 2.0 ** -24 * y.abs()
    return y, 1.02 * (tol + U[dtype] * y.abs()) + 1e-30


def _check(got, ref, tol):
    assert got.shape == ref.shape and torch.isfinite(got).all()
    over = ((got.double() - ref).abs() - tol).max()
    assert float(over) <= 0, (float(over), float((got.double() - ref).abs().max()))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", PRODUCT)
def test_product(tp, dtype, shape):
    rows, k, n = shape
    q, s, w, ws, b = _operands(tp, rows, k, n, rows + k + n)
    for bias in (b, None):
        y = tp.product_f8(q, s, w, ws, bias, dtype=dtype)
        assert y.dtype == dtype
        _check(y, *_product64(q, s, w, ws, bias, dtype))
    assert torch.equal(y, tp.product_f8(q, s, w, ws, None, dtype=dtype))
    tp.ops_check()


@pytest.mark.parametrize("rows", [1, 5, 40, 300])
@pytest.mark.parametrize("qpad,qoff,wpad,woff", [(3, 0, 0, 0), (0, 1, 0, 0), (0, 0, 5, 0), (0, 0, 0, 3), (7, 5, 16, 2), (16, 16, 32, 48)])
def test_product_addresses(tp, rows, qpad, qoff, wpad, woff):
    """Rows at any distance and address give the bits of aligned ones."""
    k, n = 400, 150
    q, s, w, ws, b = _operands(tp, rows, k, n, 3)
    ref = tp.product_f8(q.contiguous(), s, w.contiguous(), ws, b, dtype=F32)

    def moved(t, pad, off):
        r, c = t.shape
        m = torch.full((r * (c + pad) + off,), 0x7F, dtype=torch.uint8, device="cuda")   # NaN around the matrix
        v = m[off:].view(r, c + pad)[:, :c]
        v.copy_(t.view(torch.uint8) if t.is_contiguous() else t.contiguous().view(torch.uint8))
        return torch.as_strided(m.view(F8), (r, c), (c + pad, 1), off)
    got = tp.product_f8(moved(q, qpad, qoff), s, moved(w, wpad, woff), ws, b, dtype=F32)
    assert torch.equal(got, ref)


def test_product_special(tp):
    """NaN and zero scales act on their rows and columns alone; no rows."""
    q, s, w, ws, b = _operands(tp, 300, 300, 300, 9)
    s[7, 1], s[8] = float("nan"), 0.0
    y = tp.product_f8(q, s, w, ws, b, dtype=F32)
    assert torch.isnan(y[7]).all() and torch.equal(y[8], b)
    rest = [r for r in range(300) if r != 7]
    assert torch.isfinite(y[rest]).all()
    ws[1, 0] = float("nan")
    y = tp.product_f8(q, s, w, ws, b, dtype=F32)
    assert torch.isnan(y[:, 128:256]).all() and torch.isfinite(y[rest][:, :128]).all() and torch.isfinite(y[rest][:, 256:]).all()
    assert tp.product_f8(q[:0], s[:0], w, ws, b).shape == (0, 300)
