"""The product in 8-bit floating point where the two scales' own product leaves
float32's normal numbers and the result does not.

The bound is that of the other products (test_gpu_f8.py), with one rounding
more for the scales' two steps; what is below the normal numbers may be off by
float32's smallest step for each of at most 64 blocks.
"""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_f8 import BOUND, F32, TYPES, U, _gen, _values, tp  # noqa: E402,F401

pytestmark = pytest.mark.gpu

# few rows by every number of them and alignment; the tensor cores' tiles with and without shared-out K
SHAPES = [(1, 128, 16), (5, 300, 150), (12, 2000, 300), (31, 300, 1000), (7, 101, 37), (128, 512, 384), (300, 1000, 1000),
          (500, 2001, 1003), (64, 1152, 8192), (2048, 1024, 1024), (1000, 130, 4096), (4100, 1800, 2100),
          (300, 8000, 300)]
LEAST = 2.0 ** -149


def _case(tp, rows, k, n):  # noqa: F811
    g = _gen(rows + k + n)
    q, s = tp.quantise_f8(torch.randn(rows, k, generator=g, device="cuda"))
    w, ws = tp.quantise_f8(torch.randn(n, k, generator=g, device="cuda"), 128)
    some = lambda t: 1 + torch.rand(t.shape, generator=g, device="cuda")  # noqa: E731
    return q, some(s), w, some(ws)


def _within(got, ref, tol):
    assert got.shape == ref.shape and torch.isfinite(got).all()
    over = ((got.double() - ref).abs() - tol).max()
    assert float(over) <= 0, (float(over), float((got.double() - ref).abs().max()))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_small_scales(tp, dtype, shape):  # noqa: F811
    """Rows and column blocks of tiny scales: their product has a few digits left, the result has all."""
    rows, k, n = shape
    q, s, w, ws = _case(tp, rows, k, n)
    s[::2] *= 2.0 ** -76
    ws[::2] *= 2.0 ** -69
    s[3::4] = 0.0
    y = tp.product_f8(q, s, w, ws, dtype=dtype)
    x, v = _values(q, s, 1), _values(w, ws, 128)
    ref = x @ v.T
    tol = (BOUND + 2.0 ** -23) * (x.abs() @ v.abs().T) + U[dtype] * ref.abs()
    # the blocks' least steps, and the output's: bf16's smallest numbers are 2^-133 apart
    _within(y, ref, 1.02 * tol + 64 * LEAST + (2.0 ** -134 if dtype != F32 else 0))
    assert not y[3::4].any()
    tp.ops_check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_large_scales(tp, dtype, shape):  # noqa: F811
    """Scales whose product is infinite: sums of nothing stay 0, small sums finite."""
    rows, k, n = shape
    q, s, w, ws = _case(tp, rows, k, n)
    # the smallest numbers, 2^-9 m with m below 2 and 4, of either sign, and rows and columns of zeros
    bits = lambda t, top: (torch.arange(t.shape[0] * t.shape[1], device="cuda").view(t.shape) % (2 * top) * 7 % (2 * top))  # noqa: E731
    q = torch.where(bits(q, 2) < 2, bits(q, 2), bits(q, 2) - 2 + 128).to(torch.uint8).view(q.dtype)
    w = torch.where(bits(w, 4) < 4, bits(w, 4), bits(w, 4) - 4 + 128).to(torch.uint8).view(w.dtype)
    q.view(torch.uint8)[1::3] = 0
    w.view(torch.uint8)[2::5] = 0
    s *= 2.0 ** 64
    ws *= 2.0 ** 63      # 1 to 4 times 2^127; a sum is below 4096 2^-18 3
    s[1::6] *= 2.0 ** 60
    y = tp.product_f8(q, s, w, ws, dtype=dtype)
    x, v = _values(q, s, 1), _values(w, ws, 128)
    ref = x @ v.T
    tol = (BOUND + 2.0 ** -23) * (x.abs() @ v.abs().T) + U[dtype] * ref.abs()
    assert float((x.abs() @ v.abs().T).max()) < 3.3e38
    _within(y, ref, 1.02 * tol)
    assert not y[1::3].any() and not y[:, 2::5].any()
    tp.ops_check()


@pytest.mark.parametrize("rows", [5, 300])
def test_scales_that_are_no_numbers(tp, rows):  # noqa: F811
    """A scale that is NaN or infinite acts as the formula says, beside tiny ones too."""
    q, s, w, ws = _case(tp, rows, 300, 300)
    s *= 2.0 ** -100
    ws *= 2.0 ** -40
    s[1, 0], s[2, 1] = float("nan"), float("inf")
    ws[1, 2] = 0.0
    y = tp.product_f8(q, s, w, ws, dtype=F32)
    assert torch.isnan(y[1]).all() and torch.isinf(y[2]).all()
    rest = [r for r in range(rows) if r not in (1, 2)]
    x, v = _values(q, s, 1)[rest], _values(w, ws, 128)
    ref, mag = x @ v.T, x.abs() @ v.abs().T
    _within(y[rest], ref, 1.02 * ((BOUND + 2.0 ** -23) * mag + U[F32] * ref.abs()) + 64 * LEAST)
