"""Student operators on both sides of the sizes at which a launch takes another
kernel or shares its work out differently, against the formulas in 64 bits."""
import math

import pytest

torch = pytest.importorskip("torch")

from test_gpu_ops import TYPES, _check_distill, _distill_case, _gated64, _gated_case, _gen, _within, tp  # noqa: E402,F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,rows,n,k", [(1, 24576, 10, 4), (1, 24577, 10, 4), (2, 12300, 2, 1), (3, 8200, 31, 8), (5, 5000, 32, 40), (3, 8200, 31, 128),
                                        (1, 4096, 200, 9), (1, 4097, 200, 9), (2, 2100, 129, 128), (2, 2049, 500, 33),
                                        (1, 4100, 512, 8), (1, 1024, 700, 5), (1, 1025, 700, 5), (2, 513, 1024, 128)])
def test_distill_rows(tp, dtype, m, rows, n, k):  # noqa: F811
    z, ids, top, labels = _distill_case(m, rows, n, k, dtype, rows + n, masked=0.2 if n > 2 else 0.0, empty=0.1)
    _check_distill(tp, z, ids, top, labels, 2.0, 0.6, (m, rows, n, k))
    _check_distill(tp, z, ids, top, None, 3.0, 1.0, (m, rows, n, k))


@pytest.mark.parametrize("m,rows,n", [(2, 12300, 12), (2, 2100, 200), (2, 2100, 400), (1, 1024, 1000)])
def test_distill_rows_nonfinite(tp, m, rows, n):  # noqa: F811
    """A row of NaN or of infinities stays a row, a row without classes adds nothing."""
    z, ids, top, labels = _distill_case(m, rows, n, 4, torch.float32, 6)
    _, ref = tp.distill(z, ids, top, labels, tau=2.0, alpha=0.6)
    bad = z.clone()
    bad[0, 1, 0], bad[0, 2, 1], bad[0, 3] = math.nan, math.inf, -math.inf
    _, dz = tp.distill(bad, ids, top, labels, tau=2.0, alpha=0.6)
    keep = torch.ones(m, rows, dtype=torch.bool, device="cuda")
    keep[0, 1:4] = False
    assert torch.equal(dz[keep], ref[keep])
    assert torch.isnan(dz[0, 1]).all() and torch.isnan(dz[0, 2]).any() and not dz[0, 3].any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d,f,o", [(16, 1500, 1000, 1500), (17, 1500, 1000, 1500), (24, 1024, 2048, 1024), (40, 1024, 2048, 1024),
                                        (64, 510, 2046, 510), (65, 128, 256, 128), (80, 2048, 4096, 2048), (160, 1024, 4096, 200)])
def test_gated_few_rows(tp, dtype, rows, d, f, o):  # noqa: F811
    x, wgu, wd, dy = _gated_case(dtype, rows, d, f, o, rows)
    y, saved = tp.gated_forward(x, wgu, wd, "silu", save=True)
    got = [y, *tp.gated_backward(dy, x, wgu, wd, saved)]
    again = [tp.gated_forward(x, wgu, wd, "silu"), *tp.gated_backward(dy, x, wgu, wd, saved)]
    for v, w, (ref, tol) in zip(got, again, _gated64(x, wgu, wd, "silu", dy, dtype)):
        assert torch.equal(v, w)
        _within(v, ref, tol, (rows, d, f))
    tp.ops_check()


@pytest.mark.parametrize("rows", [1, 8, 9, 32, 33, 64, 128])
@pytest.mark.parametrize("k,n", [(1024, 1000), (2048, 2048), (2050, 4096), (4096, 40)])
def test_product_few_rows(tp, rows, k, n):  # noqa: F811
    """fp32 outputs: the integers' sums are exact below 2^24, then three roundings."""
    g = _gen(rows + k)
    q = torch.randint(-30, 31, (rows, k), generator=g, device="cuda").to(torch.int8)
    w = torch.randint(-30, 31, (n, k), generator=g, device="cuda").to(torch.int8)
    a, b = torch.rand(rows, generator=g, device="cuda"), torch.rand(n, generator=g, device="cuda")
    bias = torch.randn(n, generator=g, device="cuda")
    y = tp.product_q8(q, a, w, b, bias, dtype=torch.float32)
    s = q.double() @ w.double().T
    ref = s * a.double()[:, None] * b.double() + bias.double()
    tol = 2.0 ** -24 * (3 * (s * a.double()[:, None] * b.double()).abs() + ref.abs()) + 1e-30
    _within(y, ref, 1.01 * tol, (rows, k, n))


@pytest.mark.parametrize("rows,d,f,o", [(2048, 64, 2048, 512), (2048, 256, 2048, 1024)])
def test_gated_backward_many_times(tp, rows, d, f, o):  # noqa: F811
    """The same bits in 15000 passes: what comes into shared memory for a chunk
    does not overtake the reading of the one before."""
    x, wgu, wd, dy = _gated_case(torch.bfloat16, rows, d, f, o, 5)
    _, saved = tp.gated_forward(x, wgu, wd, "gelu", save=True)
    ref = tp.gated_backward(dy, x, wgu, wd, saved)[1]
    bad = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(15000):
        bad += (tp.gated_backward(dy, x, wgu, wd, saved)[1] != ref).any()
    assert int(bad) == 0
    tp.ops_check()
