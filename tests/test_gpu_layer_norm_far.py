"""Layer norm of rows whose mean is far larger than their spread: constant rows
give the bias, and others lose no more than roundings of the size of their
spread.

The bounds follow the computation: u = s - q with the row's first element q, the
mean of u (C = 2^-18: the longest chain of a row's sum, 64 additions), the
centred values u - mean(u) and their squares.  The mean that is kept for the
backward pass is rounded to float32.
"""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_more_ops import BF, C, E24, EPS, F32, TYPES, U, _gen, _norm_grad64, _rand, _within, tp  # noqa: E402,F401

pytestmark = pytest.mark.gpu


def _far_rows(g, rows, d, dtype):
    """Constant rows, rows of small spread on both sides of zero, rows with one value apart."""
    v = torch.empty(rows, d, device="cuda")
    for k, (mean, spread) in enumerate(((1000.1, 0.0), (12345.6, 0.0), (1000.0, 0.01), (-30000.0, 0.1), (3.0, 1.0))):
        at = torch.arange(k, rows, 5, device="cuda")
        v[at] = mean + spread * torch.randn(len(at), d, generator=g, device="cuda")
    v[2::10, d // 2] += 0.4
    v[7::10, 0] += 50.0
    return v.to(dtype)


def _forward64(s, w, b, dtype):
    """Per row: the mean and the bound of the stored one; r and its relative bound; h; y and its bound."""
    v, w, b = s.double(), w.double(), b.double()
    mean = v.mean(1, keepdim=True)
    c, u = v - mean, (v - v[:, :1]).abs()
    em = 1.01 * (C + 2 * E24) * u.mean(1, keepdim=True)     # of mean(u): the differences' roundings, the sum's, the quotient's
    ec = E24 * u + em + E24 * (c.abs() + em)
    var = (c * c).mean(1, keepdim=True)
    off = (2 * c.abs() * ec + ec * ec).mean(1, keepdim=True)
    ev = 1.01 * (off + (C + 3 * E24) * (var + off))
    r = 1 / torch.sqrt(var + EPS)
    x = ev / (var + EPS)
    assert float(x.max()) < 0.5
    er = 1.01 * (1 / torch.sqrt(1 - x) - 1) + 4 * E24       # (of 1 / sqrt((var + eps)(1 + t)), |t| <= x)
    h = c * r
    eh = 1.02 * (r * ec + h.abs() * (er + 2 * E24))
    y = h * w + b
    ey = 1.01 * (eh * w.abs() + 2 * E24 * ((h * w).abs() + y.abs()) + U[dtype] * y.abs())
    return mean, 1.01 * (em + E24 * mean.abs()), r, er, c, h, y, ey


# widths of every kernel: by 16 bytes, by single elements, many of those, many packed bf16 rows of odd widths
SHAPES = [(10, 16), (13, 64), (12, 1000), (70, 2048), (11, 5000), (10, 8192), (10, 16384), (11, 33), (12, 389), (11, 1023), (10, 3001),
          (10, 8191), (10, 16383), (6091, 33), (3101, 389), (1301, 2501), (1301, 5001), (4103, 1501)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d", SHAPES)
def test_far_from_zero(tp, dtype, rows, d):  # noqa: F811
    g = _gen(rows + d)
    x = _far_rows(g, rows, d, dtype)
    w, b = 1 + 0.2 * torch.randn(d, generator=g, device="cuda"), torch.randn(d, generator=g, device="cuda")
    dy = _rand(g, rows, d, dtype, 0.1)
    y, s, stats = tp.layer_norm(x, w, b, eps=EPS, save=True)
    mean, mean_off, r, er, c, h, ref, tol = _forward64(s, w, b, dtype)
    _within(y, ref, tol, "y")
    _within(stats[:, :1], mean, mean_off, "mean")
    _within(stats[:, 1:], r, 1.01 * (er + E24) * r, "1 / deviation")
    eh = 1.02 * (r * (2 * E24 * c.abs() + mean_off) + h.abs() * (er + E24))    # the backward pass's, by the stored mean
    got = tp.layer_norm_backward(dy, s, w, stats)
    (dx, dx_tol), (dw, _), (db, _) = _norm_grad64(dy, w, None, r, er, h, eh, dtype)
    _within(got[0], dx, dx_tol + 1e-30, "dx")
    chain, mag = 2 * C + E24 * rows / 128, dy.double().abs()      # a block's rows one after another
    _within(got[1], dw, 1.01 * ((mag * eh).sum(0) + chain * (mag * (h.abs() + eh)).sum(0)) + 1e-30, "dw")
    _within(got[2], db, chain * mag.sum(0), "db")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d", SHAPES)
def test_constant_rows(tp, dtype, rows, d):  # noqa: F811
    """Exactly: the bias, the value, no gradient of the weights."""
    g = _gen(rows + d)
    value = (12345.6 * torch.randn(rows, 1, generator=g, device="cuda")).to(dtype)
    x = value.expand(rows, d).contiguous()
    w, b = torch.randn(d, generator=g, device="cuda"), torch.randn(d, generator=g, device="cuda")
    y, s, stats = tp.layer_norm(x, w, b, eps=EPS, save=True)
    assert torch.equal(y, b.to(dtype).expand(rows, d)) and torch.equal(stats[:, :1], value.float())
    assert not tp.layer_norm_backward(_rand(g, rows, d, dtype), s, w, stats)[1].any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d", SHAPES)
def test_sum_in_place(tp, dtype, rows, d):  # noqa: F811
    """The library's call may write the sum over x: every warp has read the row's first element before."""
    L, g = tp.load_library(), _gen(rows + d)
    x, res = _rand(g, rows, d, dtype), _rand(g, rows, d, dtype, 30.0)
    w = torch.randn(d, generator=g, device="cuda")
    y, s = tp.layer_norm(x, w, None, res)
    out = torch.empty_like(y)
    for _ in range(20):
        both = x.clone()
        assert L.pack_layer_norm(both.data_ptr(), d, res.data_ptr(), d, w.data_ptr(), None, rows, d, 1e-5, {BF: 0, F32: 1}[dtype],
                                 both.data_ptr(), out.data_ptr(), None, torch.cuda.current_stream().cuda_stream) == tp.TP_OK
        assert torch.equal(both, s) and torch.equal(out, y)


@pytest.mark.parametrize("d", [40, 389, 1000, 3001, 16384])
def test_far_residual(tp, d):  # noqa: F811
    """A residual stream that is large and all but constant."""
    g = _gen(d)
    x, res = _rand(g, 20, d, F32, 0.05), torch.full((20, d), 4321.7, device="cuda")
    w, b = 1 + 0.2 * torch.randn(d, generator=g, device="cuda"), torch.randn(d, generator=g, device="cuda")
    y, s, stats = tp.layer_norm(x, w, b, res, eps=EPS, save=True)
    assert torch.equal(s, x + res)
    mean, mean_off, r, er, c, h, ref, tol = _forward64(s, w, b, F32)
    _within(y, ref, tol, "y")
    _within(stats[:, :1], mean, mean_off, "mean")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d", [(7, 48), (7, 389), (6091, 33), (1301, 2501)])
def test_squares_overflow(tp, dtype, rows, d):  # noqa: F811
    """Where the squares of a row overflow, 1 / deviation is 0 and y the bias; other rows do not change."""
    g = _gen(d)
    x = _rand(g, rows, d, F32)
    x[:, 1::2] = -x[:, :d - 1:2]
    w, b = torch.ones(d, device="cuda"), torch.randn(d, generator=g, device="cuda")
    plain = tp.layer_norm(x.to(dtype), w, b)[0]
    x[3] *= 1e25
    y, _, stats = tp.layer_norm(x.to(dtype), w, b, save=True)
    assert float(stats[3, 1]) == 0 and torch.equal(y[3], b.to(dtype))
    rest = torch.arange(rows, device="cuda") != 3
    assert torch.equal(y[rest], plain[rest])
