"""The student operators against their formulas in 64 bits: the gated block,
the RMS norm, the 8-bit product and the distillation loss, forward and
backward, over types, sizes, strides, masks and empty rows.

Bounds are derived, not fitted: ``u`` is the unit roundoff of the output type
(2^-8 bf16, 2^-24 fp32, one rounding), C = 2^-19 bounds an fp32 sum of a few
thousand terms on the tensor cores or in registers relative to the sum of its
terms' magnitudes (2^-24 a rounding; a tensor-core chain of 128 instructions
about 2^-20), and errors of intermediate values go through the next product
with the absolute values of its other operand.
"""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
C = 2.0 ** -19
TYPES = [torch.bfloat16, torch.float32]


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


# ------------------------------------------------------------- gated block
def _act64(name, g):
    if name == "relu":
        return g.clamp(min=0), (g > 0).double()
    if name == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    p = 0.5 * torch.special.erfc(-g / math.sqrt(2))
    return g * p, p + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)


def _gated64(x, wgu, wd, act, dy, dtype):
    """Values and error bounds of y, dx, dW_gu, dW_d."""
    u = U[dtype]
    f = wgu.shape[0] // 2
    x, wgu, wd = x.double(), wgu.double(), wd.double()
    wg, wu = wgu[:f], wgu[f:]
    g, up = x @ wg.T, x @ wu.T
    eg, eu = C * (x.abs() @ wg.abs().T), C * (x.abs() @ wu.abs().T)
    a, d = _act64(act, g)
    h, p = a * up, up * d
    # |act'| <= 1.13, |act''| <= 0.8; relu' jumps where g is within its error of 0
    ea = 1.13 * eg + 4 * C * a.abs()
    ed = 0.8 * eg + 4 * C * d.abs() + 4 * C
    if act == "relu":
        ed = (g.abs() <= eg).double()
    eh = ea * up.abs() + a.abs() * eu + u * h.abs()
    y = h @ wd.T
    ey = eh @ wd.abs().T + C * (h.abs() @ wd.abs().T) + u * y.abs()
    out = [(y, ey)]
    if dy is not None:
        dy = dy.double()
        ea, ep = ea + u * a.abs(), ed * up.abs() + d.abs() * eu + u * p.abs()
        dh = dy @ wd
        edh = C * (dy.abs() @ wd.abs())
        dg, du = dh * p, dh * a
        edg, edu = dh.abs() * ep + p.abs() * edh + u * dg.abs(), dh.abs() * ea + a.abs() * edh + u * du.abs()
        d2, e2 = torch.cat([dg, du], 1), torch.cat([edg, edu], 1)
        dx, dw, dd = d2 @ wgu, d2.T @ x, dy.T @ h
        out.append((dx, e2 @ wgu.abs() + C * (d2.abs() @ wgu.abs()) + u * dx.abs()))
        out.append((dw, e2.T @ x.abs() + C * (d2.abs().T @ x.abs()) + u * dw.abs()))
        out.append((dd, dy.abs().T @ eh + C * (dy.abs().T @ h.abs()) + u * dd.abs()))
    return [(v, 1.1 * e + 1e-30) for v, e in out]


def _gated_case(dtype, rows, d, f, o, seed, pad=0, off=0):
    g = _gen(seed)
    x = _rand(g, rows, d, dtype, pad=pad, off=off)
    wgu = _rand(g, 2 * f, d, dtype, 1 / math.sqrt(d))
    wd = _rand(g, o, f, dtype, 1 / math.sqrt(f))
    dy = _rand(g, rows, o, dtype, pad=pad, off=off)
    return x, wgu, wd, dy


GATED = [(1, 64, 64, 64), (1, 1, 1, 1), (2, 7, 5, 3), (5, 513, 130, 77), (8, 128, 256, 64), (9, 96, 40, 200), (16, 72, 1000, 8),
         (17, 256, 64, 256), (37, 512, 512, 512), (64, 33, 100, 65), (65, 320, 200, 129), (128, 128, 128, 128),
         (129, 129, 129, 129), (300, 389, 501, 389), (777, 64, 1024, 100), (1000, 520, 264, 520), (4100, 72, 80, 40)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", GATED)
def test_gated_forward_backward(tp, dtype, shape):
    rows, d, f, o = shape
    act = ("silu", "gelu", "relu")[(rows + d) % 3]
    x, wgu, wd, dy = _gated_case(dtype, rows, d, f, o, rows + d)
    y, saved = tp.gated_forward(x, wgu, wd, act, save=True)
    got = [y, *tp.gated_backward(dy, x, wgu, wd, saved)]
    assert torch.equal(y, tp.gated_forward(x, wgu, wd, act))   # what is kept changes nothing
    for name, v, (ref, tol) in zip(("y", "dx", "dw_gate_up", "dw_down"), got, _gated64(x, wgu, wd, act, dy, dtype)):
        assert v.dtype == dtype
        _within(v, ref, tol, (name, act))
    tp.ops_check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,off", [(8, 0), (3, 0), (0, 1), (5, 3)])
@pytest.mark.parametrize("rows", [3, 200])
def test_gated_strides(tp, dtype, pad, off, rows):
    """Spaced rows and odd addresses give the bits of packed ones."""
    x, wgu, wd, dy = _gated_case(dtype, rows, 104, 72, 56, 5, pad, off)
    y, saved = tp.gated_forward(x, wgu, wd, "silu", save=True)
    got = [y, *tp.gated_backward(dy, x, wgu, wd, saved)]
    xc, dyc = x.contiguous().clone(), dy.contiguous().clone()
    y2, saved2 = tp.gated_forward(xc, wgu, wd, "silu", save=True)
    for a, b in zip(got, [y2, *tp.gated_backward(dyc, xc, wgu, wd, saved2)]):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", TYPES)
def test_gated_large_tiles(tp, dtype):
    """Row and column counts over several of the largest tiles, a long reduction over the rows."""
    rows, d, f, o = (5000, 320, 520, 264) if dtype == torch.bfloat16 else (2100, 136, 200, 120)
    x, wgu, wd, dy = _gated_case(dtype, rows, d, f, o, 9)
    y, saved = tp.gated_forward(x, wgu, wd, "silu", save=True)
    got = [y, *tp.gated_backward(dy, x, wgu, wd, saved)]
    again = [tp.gated_forward(x, wgu, wd, "silu"), *tp.gated_backward(dy, x, wgu, wd, saved)]
    for v, w, (ref, tol) in zip(got, again, _gated64(x, wgu, wd, "silu", dy, dtype)):
        assert torch.equal(v, w)
        _within(v, ref, tol, dtype)


def test_gated_pairs_of_ctas(tp):
    x, wgu, wd, dy = _gated_case(torch.bfloat16, 6000, 1024, 1100, 1024, 4)
    y, saved = tp.gated_forward(x, wgu, wd, "gelu", save=True)
    got = [y, *tp.gated_backward(dy, x, wgu, wd, saved)]
    for v, (ref, tol) in zip(got, _gated64(x, wgu, wd, "gelu", dy, torch.bfloat16)):
        _within(v, ref, tol, "pairs")


@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
def test_gated_differences(tp, act):
    """The gradients against central differences of the kernels' own loss:
    h = 2^-6 leaves h^2 |third derivative| / 6 (below 10^-3 of the slope's
    scale here) and the fp32 rounding of the two losses."""
    rows, d, f, o = 40, 48, 64, 32
    x, wgu, wd, dy = _gated_case(torch.float32, rows, d, f, o, 21)
    if act == "relu":   # keep every gate away from the kink: g = +-(1 .. ), far more than h times a direction
        x = torch.sign(x)
        wgu = torch.cat([torch.where(torch.arange(f, device="cuda")[:, None] % 2 == 0, 1.0, -1.0).expand(f, d) * x[:1] / d * 4,
                         wgu[f:]]).contiguous()
        x = x[:1].expand(rows, d).contiguous()
    _, saved = tp.gated_forward(x, wgu, wd, act, save=True)
    grads = tp.gated_backward(dy, x, wgu, wd, saved)
    loss = lambda *p: float((tp.gated_forward(*p, act).double() * dy.double()).sum())  # noqa: E731
    h, g = 2.0 ** -6, _gen(3)
    for k, grad in enumerate(grads):
        base = [x, wgu, wd]
        v = torch.randn(base[k].shape, generator=g, device="cuda")
        v = v / v.norm() * math.sqrt(v.shape[0]) * 0.5
        up, down = list(base), list(base)
        up[k], down[k] = base[k] + h * v, base[k] - h * v
        moved = (up[k].double() - down[k].double())
        slope = loss(*up) - loss(*down)
        want = float((grad.double() * moved).sum())
        scale = float(grad.double().norm() * moved.norm())
        assert abs(slope - want) <= 2e-3 * scale, (act, k, slope, want, scale)


@pytest.mark.parametrize("dtype", TYPES)
def test_gated_no_rows(tp, dtype):
    x, wgu, wd, dy = _gated_case(dtype, 0, 24, 16, 8, 1)
    y, saved = tp.gated_forward(x, wgu, wd, save=True)
    assert y.shape == (0, 8)
    dx, dw, dd = tp.gated_backward(dy, x, wgu, wd, saved)
    assert dx.shape == (0, 24) and not dw.any() and not dd.any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [6, 140])
def test_gated_nonfinite_rows(tp, dtype, rows):
    """An infinite or NaN row stays in its own row of y and dx."""
    x, wgu, wd, dy = _gated_case(dtype, rows, 64, 96, 64, 2)
    x = x.clone()
    ref, saved = tp.gated_forward(x, wgu, wd, "silu", save=True)
    dref = tp.gated_backward(dy, x, wgu, wd, saved)[0]
    x[1, 3], x[4, 0] = float("nan"), float("inf")
    y, saved = tp.gated_forward(x, wgu, wd, "silu", save=True)
    dx = tp.gated_backward(dy, x, wgu, wd, saved)[0]
    keep = torch.ones(rows, dtype=torch.bool, device="cuda")
    keep[[1, 4]] = False
    assert torch.equal(y[keep], ref[keep]) and torch.equal(dx[keep], dref[keep])
    assert torch.isnan(y[1]).all() and not torch.isfinite(y[4]).all()


def test_gated_extremes(tp):
    """Gates far into both tails: no overflow inside the activations."""
    x = torch.tensor([[1.0], [-1.0], [30.0], [-30.0], [1e4], [-1e4]], device="cuda")
    wgu = torch.tensor([[1.0], [9.0], [1.0], [1.0]], device="cuda")
    wd = torch.eye(2, device="cuda")
    for act in ("silu", "gelu", "relu"):
        for dtype in TYPES:
            y = tp.gated_forward(x.to(dtype), wgu.to(dtype), wd.to(dtype), act)
            ref, tol = _gated64(x.to(dtype), wgu.to(dtype), wd.to(dtype), act, None, dtype)[0]
            _within(y, ref, tol, (act, dtype))


def test_other_stream(tp):
    """Operators on a stream of their own, with the host far ahead."""
    x, wgu, wd, _ = _gated_case(torch.bfloat16, 500, 256, 256, 256, 8)
    want = tp.gated_forward(x, wgu, wd)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        outs = [tp.gated_forward(x, wgu, wd) for _ in range(8)]
    outs += [tp.gated_forward(x, wgu, wd, stream=side) for _ in range(8)]
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(o, want) for o in outs)
    tp.ops_check(side)


# ------------------------------------------------------------------ RMS norm
EPS = 1e-6
NORM = [(1, 1), (3, 7), (2, 64), (9, 250), (70, 256), (5, 257), (33, 512), (4, 900), (300, 1000), (13, 1024), (6, 1030),
        (50, 2048), (3, 2050), (7, 4096), (2, 5000), (5, 8192), (3, 8200), (2, 16384), (3000, 96)]


def _norm64(x, res, w):
    s = x.double() + (res.double() if res is not None else 0)
    r = 1 / torch.sqrt((s * s).mean(1, keepdim=True) + EPS)
    return s, r, s * r * w.double()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", NORM)
@pytest.mark.parametrize("pad,off", [(0, 0), (3, 1)])
def test_rms_norm(tp, dtype, shape, pad, off):
    rows, d = shape
    g = _gen(rows * 7 + d)
    x, res = _rand(g, rows, d, dtype, pad=pad, off=off), _rand(g, rows, d, dtype, 3.0, pad=pad + 1, off=off)
    w = 1 + 0.3 * torch.randn(d, generator=g, device="cuda")
    u = U[dtype]
    for rr in (res, None):
        s, r, n = _norm64(x, rr, w)
        y, tot = tp.rms_norm(x, w, rr, eps=EPS)
        _within(y, n, (u + C) * n.abs(), "y")
        _within(tot, s, u * s.abs(), "sum") if rr is not None else None
        q, scale, tot2 = tp.rms_norm_q8(x, w, rr, eps=EPS)
        assert torch.equal(tot, tot2) and q.dtype == torch.int8
        want = n.abs().amax(1) / 127
        _within(scale, want, C * want, "scale")
        # n / scale to one rounding of each, then to the nearest integer
        off_by = (q.double() - n / want[:, None]).abs().max()
        assert float(off_by) <= 0.5 + 127 * 2 * C, float(off_by)
        assert int(q.abs().max()) == 127


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", NORM)
@pytest.mark.parametrize("pad,off", [(0, 0), (3, 1)])
def test_rms_norm_backward(tp, dtype, shape, pad, off):
    rows, d = shape
    g = _gen(rows * 7 + d + 1)
    s, dy = _rand(g, rows, d, dtype, 2.0, pad=pad, off=off), _rand(g, rows, d, dtype, pad=pad, off=off)
    dsum = _rand(g, rows, d, dtype, pad=pad + 2, off=off)
    w = 1 + 0.3 * torch.randn(d, generator=g, device="cuda")
    u = U[dtype]
    v, r, _ = _norm64(s, None, w)
    t = dy.double() * w.double()
    f = r * r * (t * v).mean(1, keepdim=True)
    ef = C * r * r * (t * v).abs().mean(1, keepdim=True) + C * f.abs()
    dw = (dy.double() * v * r).sum(0)
    edw = C * (dy.double() * v * r).abs().sum(0) + 1e-30
    for extra in (dsum, None):
        dx = r * (t - v * f) + (extra.double() if extra is not None else 0)
        tol = r * (C * t.abs() + C * (v * f).abs() + v.abs() * ef) + u * dx.abs() + 1e-30
        got, gw = tp.rms_norm_backward(dy, s, w, extra, eps=EPS)
        _within(got, dx, tol, "dx")
        _within(gw, dw, edw, "dw")
        again, gw2 = tp.rms_norm_backward(dy, s, w, extra, eps=EPS)
        assert torch.equal(got, again) and torch.equal(gw, gw2)


def test_rms_norm_differences(tp):
    """Central differences of sum(y dy): h = 2^-8 of values around 1 leaves a
    third-order term below 10^-4 of the scale."""
    g = _gen(4)
    rows, d = 20, 300
    x, dy = _rand(g, rows, d, torch.float32), _rand(g, rows, d, torch.float32)
    w = 1 + 0.3 * torch.randn(d, generator=g, device="cuda")
    dx, dw = tp.rms_norm_backward(dy, x, w, eps=EPS)
    loss = lambda a, b: float((tp.rms_norm(a, b, eps=EPS)[0].double() * dy.double()).sum())  # noqa: E731
    for k, grad in enumerate((dx, dw)):
        v = torch.randn(grad.shape, generator=g, device="cuda")
        h = 2.0 ** -8
        up = (x + h * v, w) if k == 0 else (x, w + h * v)
        down = (x - h * v, w) if k == 0 else (x, w - h * v)
        moved = (up[k].double() - down[k].double())
        want = float((grad.double() * moved).sum())
        assert abs(loss(*up) - loss(*down) - want) <= 1e-3 * float(grad.double().norm() * moved.norm())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [40, 3000])
def test_rms_norm_odd_rows(tp, dtype, d):
    """Rows of zeros, of one value, with infinities and NaN, of tiny and huge values."""
    g = _gen(11)
    x = _rand(g, 8, d, dtype).clone()
    x[0] = 0
    x[1] = 2
    x[2, 5] = float("nan")
    x[3, 7] = float("inf")
    x[4] *= 1e-18
    x[5] *= 1e15
    w = torch.ones(d, device="cuda")
    y, _ = tp.rms_norm(x, w, eps=EPS)
    _, _, n = _norm64(x, None, w)
    fine = [0, 1, 4, 5, 6, 7]
    _within(y[fine], n[fine], (U[dtype] + C) * n[fine].abs() + 1e-37, "odd rows")
    assert torch.isnan(y[2]).all() and not torch.isfinite(y[3]).all()
    q, scale, _ = tp.rms_norm_q8(x, w, eps=EPS)
    assert not q[0].any() and float(scale[0]) == 0 and (q[1] == 127).all()
    assert torch.isnan(scale[[2, 3]]).all() and not q[[2, 3]].any()
    got, gw = tp.rms_norm_backward(torch.ones_like(x[fine]), x[fine].contiguous(), w, eps=EPS)
    assert torch.isfinite(got).all() and torch.isfinite(gw).all()


def test_rms_norm_no_rows(tp):
    x = torch.zeros(0, 24, device="cuda")
    w = torch.ones(24, device="cuda")
    y, s = tp.rms_norm(x, w, x)
    q, scale, _ = tp.rms_norm_q8(x, w)
    dx, dw = tp.rms_norm_backward(x, x, w)
    assert y.shape == s.shape == q.shape == dx.shape == (0, 24) and scale.shape == (0,) and not dw.any()


# ------------------------------------------------------------- 8-bit product
PRODUCT = [(1, 1, 1), (1, 64, 10), (2, 100, 33), (3, 1024, 1000), (4, 17, 5), (5, 2048, 64), (8, 500, 300), (9, 512, 96),
           (16, 333, 77), (17, 128, 128), (31, 4096, 130), (37, 900, 1001), (64, 64, 64), (65, 250, 257), (100, 2048, 700),
           (129, 130, 131), (300, 1000, 515), (700, 384, 256), (2100, 520, 264)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", PRODUCT)
@pytest.mark.parametrize("pad,off", [(0, 0), (16, 0), (3, 1)])
def test_product_q8(tp, dtype, shape, pad, off):
    rows, k, n = shape
    g = _gen(rows + k + n)
    q = torch.randint(-128, 128, (rows * (k + pad) + off,), generator=g, device="cuda").to(torch.int8)
    q = q[off:].view(rows, k + pad)[:, :k]
    w = torch.randint(-128, 128, (n, k), generator=g, device="cuda").to(torch.int8)
    s, ws = torch.rand(rows, generator=g, device="cuda") + 0.5, torch.rand(n, generator=g, device="cuda") + 0.5
    b = 1000 * torch.randn(n, generator=g, device="cuda")
    acc = q.double() @ w.double().T
    # partial sums stay below 2^24 in magnitude: random signs, |sum| < 8 sqrt(k) 2^13
    for bias in (b, None):
        ref = acc * s.double()[:, None] * ws.double()
        tol = 2.0 ** -22 * ref.abs()
        if bias is not None:
            ref = ref + bias.double()
            tol = tol + 2.0 ** -24 * ref.abs()
        y = tp.product_q8(q, s, w, ws, bias, dtype=dtype)
        _within(y, ref, tol + U[dtype] * ref.abs(), "y")
    one_r, one_n = torch.ones(rows, device="cuda"), torch.ones(n, device="cuda")
    assert torch.equal(tp.product_q8(q, one_r, w, one_n, dtype=torch.float32).double(), acc)   # exact integers
    tp.ops_check()


def test_product_q8_extremes(tp):
    """Sums past 2^24 (all factors -128 or 127), scales of zero and NaN."""
    k = 5000
    for rows in (3, 40, 300):
        q = torch.full((rows, k), -128, dtype=torch.int8, device="cuda")
        w = torch.full((65, k), -128, dtype=torch.int8, device="cuda")
        w[1::2] = 127
        s, ws = torch.ones(rows, device="cuda"), torch.ones(65, device="cuda")
        s[1], s[2] = 0.0, float("nan")
        y = tp.product_q8(q, s, w, ws, dtype=torch.float32)
        acc = q.double() @ w.double().T
        _within(y[:1], acc[:1], C * acc[:1].abs(), "large sums")
        assert not y[1].any() and torch.isnan(y[2]).all()


def test_product_q8_no_rows(tp):
    q = torch.zeros(0, 24, dtype=torch.int8, device="cuda")
    y = tp.product_q8(q, torch.zeros(0, device="cuda"), torch.zeros(5, 24, dtype=torch.int8, device="cuda"),
                      torch.ones(5, device="cuda"))
    assert y.shape == (0, 5)


@pytest.mark.parametrize("rows", [2, 150])
def test_norm_then_product(tp, rows):
    """The served head: what the 8-bit pair gives is within the quantisation's
    half steps of the unquantised layer."""
    g = _gen(6)
    d, n = 512, 100
    x, w = _rand(g, rows, d, torch.bfloat16), torch.ones(d, device="cuda")
    W = torch.randn(n, d, generator=g, device="cuda") / math.sqrt(d)
    sw = W.abs().amax(1) / 127
    qw = torch.round(W / sw[:, None]).to(torch.int8)
    q, s, _ = tp.rms_norm_q8(x, w)
    y = tp.product_q8(q, s, qw, sw, dtype=torch.float32)
    _, _, nrm = _norm64(x, None, w)
    ref = nrm @ W.double().T
    tol = 0.51 * s.double()[:, None] * W.double().abs().sum(1) + 0.51 * sw.double() * (nrm.abs().sum(1, keepdim=True) +
                                                                                   0.51 * d * s.double()[:, None])
    _within(y, ref, tol, "head")


# -------------------------------------------------------------- distillation
def _distill64(z, ids, top, labels, tau, alpha):
    """Losses and gradients by the definition, and their error bounds."""
    m, rows, n = z.shape
    dt = z.dtype
    z = z.double()
    there = (ids >= 0) & (ids < n) & (top != -math.inf)
    t = torch.where(there, top.double() / tau, -math.inf)
    some = there.any(1)
    p = torch.where(some[:, None], torch.softmax(torch.where(some[:, None], t, 0.0), 1), 0.0) * there
    teach = torch.zeros(rows, n, device="cuda", dtype=torch.float64)
    teach.scatter_add_(1, torch.where(there, ids, 0).long(), p)
    alive = (z != -math.inf).any(2)
    zs = torch.where(alive[..., None], z, 0.0)
    zm = zs.amax(2, keepdim=True)
    lq = torch.log_softmax(zs / tau, 2)
    # an exponential: 2 ulp and its argument's rounding; a term of the loss: its magnitude's
    e = 2.0 ** -20 * (4 + ((zs - zm) / tau).clamp(min=-60).abs())
    idx = torch.where(there, ids, 0).long()[None].expand(m, -1, -1)
    zi, li = torch.gather(zs, 2, idx), torch.gather(lq, 2, idx)
    logp = torch.log(torch.where(p > 0, p, 1.0))
    on = (p > 0)[None]
    kd = tau ** 2 * torch.where(on, p * (logp[None] - li), 0.0).sum(2)
    size = tau ** 2 * torch.where(on, p * (2 + logp.abs()[None] + ((zi - zm) / tau).abs() + li.abs()), 0.0).sum(2)
    loss = alpha * kd * alive
    lsize = alpha * size
    dz = alpha * tau * (lq.exp() * some[None, :, None] - teach[None])
    edz = alpha * tau * (lq.exp() * e + 2.0 ** -19 * teach[None] * (1 + t.where(there, t.new_zeros(())).abs().amax(1)[None, :, None]))
    if labels is not None:
        ok = (labels >= 0) & (labels < n)
        at = torch.where(ok, labels, 0).long()
        l1 = torch.log_softmax(zs, 2)
        ly = torch.gather(l1, 2, at[None, :, None].expand(m, -1, 1))[..., 0]
        loss = loss + (1 - alpha) * torch.where(ok[None] & alive, -ly, 0.0)
        far = torch.gather(zs - zm, 2, at[None, :, None].expand(m, -1, 1))[..., 0].abs()
        lsize = lsize + (1 - alpha) * torch.where(ok[None], 2 + ly.abs() + far, 0.0)
        hot = torch.zeros(rows, n, device="cuda", dtype=torch.float64)
        hot[torch.arange(rows, device="cuda"), at] = 1.0
        dz = dz + (1 - alpha) * ok[None, :, None] * (l1.exp() - hot[None])
        edz = edz + (1 - alpha) * (l1.exp() * 4 * tau * e + 2.0 ** -19 * hot[None])
    dz = dz * alive[..., None] / rows
    edz = edz / rows + U[dt] * dz.abs() + 1e-30
    return (loss.mean(1), 2.0 ** -18 * lsize.where(alive, lsize.new_zeros(())).mean(1) + 1e-30), (dz, edz)


def _distill_case(m, rows, n, k, dtype, seed, masked=0.0, empty=0.0):
    g = _gen(seed)
    t = 2.5 * torch.randn(rows, n, generator=g, device="cuda")
    z = (torch.randn(m, rows, n, generator=g, device="cuda") + 0.5 * t).to(dtype)
    if masked:
        off = torch.rand(rows, n, generator=g, device="cuda") < masked
        t, z = t.masked_fill(off, -math.inf), z.masked_fill(off[None], -math.inf)
    top = torch.topk(t, min(k, n), 1)
    ids = torch.where(top.values > -math.inf, top.indices, -1).to(torch.int32)
    if empty:
        ids[torch.rand(rows, generator=g, device="cuda") < empty] = -1
    labels = torch.where(top.values[:, 0] > -math.inf, top.indices[:, 0], -1).to(torch.int32)
    labels[::7] = -1
    return z.contiguous(), ids.contiguous(), top.values.contiguous(), labels


def _check_distill(tp, z, ids, top, labels, tau, alpha, what):
    loss, dz = tp.distill(z, ids, top, labels, tau=tau, alpha=alpha)
    (rl, tl), (rz, tz) = _distill64(z, ids, top, labels, tau, alpha)
    _within(loss, rl, tl, ("loss", what))
    _within(dz, rz, tz, ("dz", what))
    only, none = tp.distill(z, ids, top, labels, tau=tau, alpha=alpha, grad=False)
    assert none is None and torch.equal(only, loss)
    again = tp.distill(z, ids, top, labels, tau=tau, alpha=alpha)
    assert torch.equal(again[0], loss) and torch.equal(again[1], dz)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [2, 3, 10, 16, 17, 32, 33, 64, 65, 128, 129, 256, 300, 513, 1024, 1025, 2000, 8192, 8195, 20001])
def test_distill(tp, dtype, n):
    k = {2: 1, 10: 4, 300: 128, 1025: 33, 20001: 100}.get(n, 8)
    m, rows = (3, 50) if n <= 300 else (2, 9)
    for tau, alpha, lab in ((1.0, 1.0, False), (2.0, 0.7, True), (4.0, 0.3, True), (3.0, 0.5, True), (0.7, 0.0, True)):
        z, ids, top, labels = _distill_case(m, rows, n, k, dtype, n + int(10 * tau))
        _check_distill(tp, z, ids, top, labels if lab else None, tau, alpha, (n, tau, alpha))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [2, 12, 200, 1500, 9001])
def test_distill_masks(tp, dtype, n):
    """Classes ruled out, rows without a teacher, rows without any class."""
    z, ids, top, labels = _distill_case(2, 40, n, 5, dtype, n, masked=0.5, empty=0.3)
    z[:, 3], ids[3], labels[3] = -math.inf, -1, -1      # nothing is left
    ids[4], labels[4] = -1, -1                          # neither teacher nor label
    z[0, 6] = -math.inf                                 # one student's row alone, where the teacher has entries
    for tau, alpha in ((2.0, 0.6), (3.0, 1.0)):
        _check_distill(tp, z, ids, top, labels, tau, alpha, "masks")
    _, dz = tp.distill(z, ids, top, labels, tau=2.0, alpha=0.6)
    assert not dz[:, 3].any() and not dz[:, 4].any() and not dz[0, 6].any()
    assert not dz[z == -math.inf].any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [9, 40, 600, 2500])
@pytest.mark.parametrize("low", [-1e4, -1e10, -3.3e38])
def test_distill_finite_masks(tp, dtype, n, low):
    """Classes ruled out by a large negative number instead of -inf, rows where
    that is all there is, and rows far from zero."""
    z, ids, top, labels = _distill_case(2, 12, n, 3, dtype, n)
    z[:, 2] = low
    z[:, 3, n // 2:] = low
    z[:, 4, : n // 2] = -math.inf
    z[:, 4, n // 2:] = low
    z[:, 5] += 1024.0
    z[:, 6] = (-low if low > -1e38 else 3e38)
    ids[2:5] = n - 1
    labels[2:5] = n - 1
    ids[3] = labels[3] = 0
    for tau in (1.0, 2.0, 3.0):
        _check_distill(tp, z, ids, top, labels, tau, 0.6, (n, low))


@pytest.mark.parametrize("n", [20, 3000])
def test_distill_entries(tp, n):
    """Entries of the same class add up, ids out of range and logits of -inf
    are no entries, the type's lowest value is an entry of weight zero."""
    z, _, _, labels = _distill_case(2, 6, n, 4, torch.float32, 5)
    ids = torch.tensor([[1, 1, 2, 1], [0, n, -7, 2 ** 31 - 1], [3, 4, 5, 6], [3, 4, 5, 6], [7, 7, 7, 7], [-1, -1, -1, 9]],
                       dtype=torch.int32, device="cuda")
    low = -3.4028234663852886e38
    top = torch.tensor([[1.0, 2.0, 0.5, -1.0], [1.0] * 4, [1.0, -math.inf, 2.0, low], [-math.inf] * 4, [low] * 4,
                        [0.0, 0.0, 0.0, -1e30]], device="cuda")
    labels[:2] = torch.tensor([1, n], dtype=torch.int32)
    _check_distill(tp, z, ids, top, labels, 2.0, 0.6, "entries")


@pytest.mark.parametrize("n", [50, 5000])
def test_distill_nonfinite(tp, n):
    """A NaN or +inf logit poisons its own row and its student's mean; a
    teacher's entry on a ruled-out class makes the loss infinite."""
    z, ids, top, labels = _distill_case(3, 10, n, 4, torch.float32, 6)
    ref, dref = tp.distill(z, ids, top, labels, tau=2.0, alpha=0.6)
    bad = z.clone()
    bad[0, 2, 5], bad[1, 4, 1] = float("nan"), float("inf")
    loss, dz = tp.distill(bad, ids, top, labels, tau=2.0, alpha=0.6)
    assert torch.isnan(loss[0]) and torch.isnan(loss[1]) and torch.equal(loss[2], ref[2])
    assert torch.isnan(dz[0, 2]).all() and torch.isnan(dz[1, 4]).any()
    keep = torch.ones(3, 10, dtype=torch.bool, device="cuda")
    keep[0, 2] = keep[1, 4] = False
    assert torch.equal(dz[keep], dref[keep])
    bad = z.clone()
    bad[0, 2, int(ids[2, 0])] = -math.inf
    loss, dz = tp.distill(bad, ids, top, None, tau=2.0, alpha=1.0)
    assert float(loss[0]) == math.inf and torch.isfinite(dz).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("off", [1, 3, 8])
def test_distill_addresses(tp, dtype, off):
    """Logits at odd addresses, odd row lengths."""
    for n in (77, 1501, 9003):
        z, ids, top, labels = _distill_case(2, 5, n, 6, dtype, off)
        mem = torch.empty(z.numel() + off, dtype=dtype, device="cuda")
        zo = mem[off:].view(z.shape)
        zo.copy_(z)
        a, b = tp.distill(z, ids, top, labels, tau=2.0, alpha=0.6), tp.distill(zo, ids, top, labels, tau=2.0, alpha=0.6)
        _check_distill(tp, zo, ids, top, labels, 2.0, 0.6, off)
        (_, tl), (_, tz) = _distill64(z, ids, top, labels, 2.0, 0.6)
        _within(a[0], b[0].double(), 2 * tl, "loss")
        _within(a[1], b[1].double(), 2 * tz, "dz")


def test_distill_differences(tp):
    """Central differences of the loss in 64 bits' worth of students: each
    student's loss changes by its own gradient."""
    z, ids, top, labels = _distill_case(4, 30, 40, 6, torch.float32, 12)
    _, dz = tp.distill(z, ids, top, labels, tau=2.0, alpha=0.6)
    v = torch.randn(z.shape, generator=_gen(1), device="cuda")
    h = 2.0 ** -5
    up, down = z + h * v, z - h * v
    lu, _ = tp.distill(up, ids, top, labels, tau=2.0, alpha=0.6, grad=False)
    ld, _ = tp.distill(down, ids, top, labels, tau=2.0, alpha=0.6, grad=False)
    moved = up.double() - down.double()
    want = (dz.double() * moved).sum((1, 2))
    scale = dz.double().flatten(1).norm(dim=1) * moved.flatten(1).norm(dim=1)
    assert ((lu.double() - ld.double() - want).abs() <= 1e-3 * scale).all()


def test_distill_no_rows(tp):
    z = torch.zeros(3, 0, 5, device="cuda")
    loss, dz = tp.distill(z, torch.zeros(0, 2, dtype=torch.int32, device="cuda"), torch.zeros(0, 2, device="cuda"))
    assert not loss.any() and dz.shape == z.shape


def test_distill_two_dims_and_pack_layout(tp):
    """[rows, n] is one student; students are independent of one another."""
    z, ids, top, labels = _distill_case(5, 64, 10, 3, torch.float32, 2)
    loss, dz = tp.distill(z, ids, top, labels, tau=2.0, alpha=0.6)
    for i in range(5):
        l1, d1 = tp.distill(z[i], ids, top, labels, tau=2.0, alpha=0.6)
        assert d1.shape == (64, 10) and torch.equal(l1[0], loss[i]) and torch.equal(d1, dz[i])


# ------------------------------------------------------- arguments on the GPU
def test_binding_refusals(tp):
    x = torch.zeros(4, 16, device="cuda")
    w = torch.ones(16, device="cuda")
    bad = [lambda: tp.gated_forward(x, torch.zeros(7, 16, device="cuda"), torch.zeros(3, 3, device="cuda")),
           lambda: tp.gated_forward(x.half(), torch.zeros(8, 16, device="cuda").half(), torch.zeros(3, 4, device="cuda").half()),
           lambda: tp.gated_forward(x, torch.zeros(8, 16, device="cuda"), torch.zeros(3, 4, device="cuda"), act="tanh"),
           lambda: tp.gated_forward(x.T, torch.zeros(8, 4, device="cuda"), torch.zeros(3, 4, device="cuda")),
           lambda: tp.gated_forward(x[:1].expand(4, 16), torch.zeros(8, 16, device="cuda"), torch.zeros(3, 4, device="cuda")),
           lambda: tp.rms_norm(x, w.double()), lambda: tp.rms_norm(x, w[:8]), lambda: tp.rms_norm(x, w, x[:2]),
           lambda: tp.rms_norm_backward(x, x.bfloat16(), w),
           lambda: tp.product_q8(x.to(torch.int8), w[:3], x.to(torch.int8), w[:4]),
           lambda: tp.product_q8(x, w[:4], x.to(torch.int8), w[:4]),
           lambda: tp.product_q8(x.to(torch.int8), w[:4], x.to(torch.int8), w[:4], dtype=torch.float16),
           lambda: tp.distill(x, torch.zeros(4, 2, device="cuda"), torch.zeros(4, 2, device="cuda")),
           lambda: tp.distill(x, torch.zeros(3, 2, dtype=torch.int32, device="cuda"), torch.zeros(3, 2, device="cuda")),
           lambda: tp.distill(x.T, torch.zeros(16, 2, dtype=torch.int32, device="cuda"), torch.zeros(16, 2, device="cuda"))]
    for k, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            print("accepted", k)
    ids, top = torch.zeros(4, 2, dtype=torch.int32, device="cuda"), torch.zeros(4, 2, device="cuda")
    for kw in (dict(tau=0.0), dict(alpha=2.0)):
        with pytest.raises(tp.TabpackError) as ei:
            tp.distill(x, ids, top, **kw)
        assert ei.value.status == tp.TP_EINVAL
    with pytest.raises(tp.TabpackError):
        tp.rms_norm(x, w, eps=-1.0)


def test_graph_capture(tp):
    """Every operator can be captured in a CUDA graph and replayed on new inputs."""
    g = _gen(1)
    x, wgu, wd, dy = _gated_case(torch.bfloat16, 60, 64, 96, 64, 3)
    x, w = x.contiguous(), torch.ones(64, device="cuda")
    qw, sw = torch.randint(-127, 128, (40, 64), generator=g, device="cuda").to(torch.int8), torch.full((40,), 0.01, device="cuda")
    ids = torch.randint(0, 40, (60, 3), generator=g, device="cuda").to(torch.int32)
    top = torch.randn(60, 3, generator=g, device="cuda")

    def work():
        y, saved = tp.gated_forward(x, wgu, wd, save=True)
        dx, dw, dd = tp.gated_backward(dy, x, wgu, wd, saved)
        q, s, tot = tp.rms_norm_q8(y, w, x)
        z = tp.product_q8(q, s, qw, sw, dtype=torch.float32)
        loss, dz = tp.distill(z, ids, top)
        return [y, dx, dw, dd, tot, z, loss, dz]

    work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = work()
    x.copy_(torch.randn(60, 64, generator=g, device="cuda"))
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(out, work()):
        assert torch.equal(a, b)
