"""The student operators at the edges of what they take."""
import math

import pytest

torch = pytest.importorskip("torch")

from test_gpu_ops import TYPES, U, _act64, _distill64, _gated64, _gated_case, _gen, _within, tp  # noqa: E402,F401

pytestmark = pytest.mark.gpu


# ------------------------------------------------- distillation: temperatures
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [700, 4096, 20001])
@pytest.mark.parametrize("tau,low", [(1e8, -1e8), (2.0 ** 20, -2.0 ** 21), (2.0 ** 18, -2.0 ** 27), (2.0 ** -18, -2.0 ** 9),
                                     (2.0 ** -26, -2.0)])
def test_distill_far_temperatures(tp, dtype, n, tau, low):  # noqa: F811
    """Classes far below the maximum count by the exponent of each softmax: a
    gap that leaves nothing of exp(z) may leave exp(z / tau) almost one (tau >
    1), and the other way round (tau < 1).  Bounds on the gradient: an exponential
    of a gap x is off by 2 ulp and its exponent's two roundings, 2^-20 (1 + |x|)
    in all, its softmax by twice that, the teacher's weights likewise."""
    rows, k, alpha = 6, 3, 0.5
    g = _gen(n)
    z = torch.zeros(2, rows, n, device="cuda")
    z[:, 0, : n // 2] = low                       # the first classes that a thread sees
    z[:, 1, n // 2:] = low
    z[:, 2, : n - 1] = low
    z[:, 3] = torch.where(torch.rand(n, generator=g, device="cuda") < 0.5, low, 0.0)
    z[:, 4] = low
    z[:, 5, : n // 2] = -math.inf
    z[1] *= 0.5
    z = z.to(dtype)
    ids = torch.tensor([[n - 1, 0, 5]], dtype=torch.int32, device="cuda").repeat(rows, 1)
    ids[5] = n - 1
    top = torch.tensor([[0.0, 0.5 * tau, -tau]], device="cuda").repeat(rows, 1)
    labels = torch.full((rows,), n - 1, dtype=torch.int32, device="cuda")
    for lab in (labels, None):
        loss, dz = tp.distill(z, ids, top, lab, tau=tau, alpha=alpha)
        (want, _), (ref, _) = _distill64(z, ids, top, lab, tau, alpha)
        zd = z.double()
        gap = zd.amax(2, keepdim=True) - zd
        err = lambda x: 2.0 ** -19 * (2 + x.clamp(max=200.0))  # noqa: E731
        e = alpha * tau * (torch.softmax(zd / tau, 2) * err(gap / tau))
        there = torch.zeros(rows, n, dtype=torch.float64, device="cuda").scatter_(1, ids.long(), 1.0)
        e = e + alpha * tau * there * 2.0 ** -18
        if lab is not None:
            e = e + (1 - alpha) * (torch.softmax(zd, 2) * err(gap) + 2.0 ** -22)
        _within(dz, ref, e / rows + U[dtype] * ref.abs() + 1e-30, (n, tau, low))
        # the loss is tau^2 times a difference of logarithms, each off by its size's rounding
        p = torch.softmax(top.double() / tau, 1)
        size = (p * (4 + torch.gather(gap / tau, 2, ids.long()[None].expand(2, -1, -1)))).sum(2) + math.log(n)
        tol = alpha * tau ** 2 * size
        if lab is not None:
            tol = tol + (1 - alpha) * (gap[:, :, n - 1] + math.log(n) + 4)
        _within(loss, want, 2.0 ** -18 * tol.mean(1), (n, tau, low))
        only, none = tp.distill(z, ids, top, lab, tau=tau, alpha=alpha, grad=False)
        assert none is None and torch.equal(only, loss)


# ------------------------------------------------------------------ streams
def test_inputs_of_calls_on_another_stream(tp):  # noqa: F811
    """Inputs that the caller lets go of at once stay whole until a call with
    stream= has read them: their memory is not given to the caller's own stream
    before that."""
    side = torch.cuda.Stream()
    g = _gen(5)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    rows, d, f, n, k = 300, 256, 512, 1000, 4
    x, w, wd, dy = (t.bfloat16() for t in (r(rows, d), r(2 * f, d) / 16, r(d, f) / 22, r(rows, d)))
    v, res = r(d), r(rows, d).bfloat16()
    q = torch.randint(-127, 128, (rows, d), generator=g, device="cuda").to(torch.int8)
    qw = torch.randint(-127, 128, (n, d), generator=g, device="cuda").to(torch.int8)
    s, sw, b, z, top = r(rows).abs(), r(n).abs(), r(n), r(2, rows, n), r(rows, k)
    ids = torch.randint(0, n, (rows, k), generator=g, device="cuda").int()
    y = torch.randint(0, n, (rows,), generator=g, device="cuda").int()
    saved = tp.gated_forward(x, w, wd, save=True)[1]
    calls = [(tp.gated_forward, (x, w, wd)), (tp.gated_backward, (dy, x, w, wd, saved)), (tp.rms_norm, (x, v, res)),
             (tp.rms_norm_q8, (x, v, res)), (tp.rms_norm_backward, (dy, x, v, res)), (tp.product_q8, (q, s, qw, sw, b)),
             (tp.distill, (z, ids, top, y))]
    flat = lambda o: list(o) if isinstance(o, tuple) else [o]  # noqa: E731
    want = [flat(fn(*a)) for fn, a in calls]
    for fn, a in calls:      # what is loaded or allocated for the first time may wait for the device
        fn(*a, stream=side)
        spare = [torch.zeros_like(t) for t in a + a]
        del spare
    torch.cuda.synchronize()
    for (fn, a), ref in zip(calls, want):
        copies = [t.clone() for t in a]
        where = [t.data_ptr() for t in copies]
        shapes = [(t.shape, t.dtype) for t in copies]
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            torch.cuda._sleep(100_000_000)            # about 50 ms
        got = flat(fn(*copies, stream=side))
        del copies
        again = [torch.zeros(sh, dtype=dt, device="cuda") for sh, dt in shapes]
        assert not set(where) & {t.data_ptr() for t in again}, fn.__name__
        torch.cuda.synchronize()
        for p, t in zip(got, ref):
            assert torch.equal(p, t), fn.__name__


@pytest.mark.parametrize("rows", [5, 40, 100, 300])
@pytest.mark.parametrize("where", ["x", "h"])
def test_gated_fp32_largest_values(tp, rows, where):  # noqa: F811
    """Finite fp32 values above bf16's largest (3.39e38), among the inputs or as
    weights and h: their parts are finite and sum up to them."""
    big = 3.4e38
    g = _gen(rows)
    d, f, o = 24, 40, 16
    x = torch.randn(rows, d, generator=g, device="cuda")
    x[:, 0] = 1.0
    wgu = torch.randn(2 * f, d, generator=g, device="cuda")
    wgu[:f] = 0
    wgu[:f, 0] = 1.0                                   # relu(g) = 1
    wd, dy = torch.randn(o, f, generator=g, device="cuda"), torch.randn(rows, o, generator=g, device="cuda")
    sign = 1.0 - 2.0 * (torch.arange(rows, device="cuda") % 2)
    if where == "x":                                   # u about 10^8
        x[:, 1] = torch.where(torch.arange(rows, device="cuda") % 3 == 0, x[:, 1], big * sign)
        wgu[f:, 1] = 1e-30
        dy = 1e-12 * dy
    else:                                              # u and h of +-3.4e38 in every other column
        x[:, 1] = sign
        wgu[f::2, 1] = big
        wd, dy = 1e-30 * wd, 1e-3 * dy
    y, saved = tp.gated_forward(x, wgu, wd, "relu", save=True)
    got = [y, *tp.gated_backward(dy, x, wgu, wd, saved)]
    for name, v, (ref, tol) in zip(("y", "dx", "dw_gate_up", "dw_down"), got, _gated64(x, wgu, wd, "relu", dy, torch.float32)):
        _within(v, ref, tol, (name, rows))


# ------------------------------------------------------------ norm into 8 bits
@pytest.mark.parametrize("d", [200, 203, 1024, 5000])
@pytest.mark.parametrize("size", [1.0, 1e-37, 3e-42, 1e30])
def test_rms_norm_q8_rounds_the_quotient(tp, d, size):  # noqa: F811
    """q is n / scale of the n and the scale that the same call gives, to the
    nearest integer, ties to even, at most 127 (a scale below the normal
    numbers is off by up to half of itself).  The quotient of two fp32 numbers is
    no closer to a tie than 2^-26 of itself unless it is one, so 64 bits decide."""
    rows = 4_000_000 // d
    g = _gen(d)
    x = torch.randn(rows, d, generator=g, device="cuda")
    x[:2] = torch.randint(-253, 254, (2, d), generator=g, device="cuda") / 4     # n / scale at and beside k / 2
    x[:2, 0] = 63.5
    w = (torch.ones(d, device="cuda") if size == 1.0 else 1 + 0.3 * torch.randn(d, generator=g, device="cuda")) * size
    y, q = torch.empty_like(x), torch.empty(rows, d, dtype=torch.int8, device="cuda")
    scale = torch.empty(rows, device="cuda")
    st = tp.load_library().pack_rms_norm(x.data_ptr(), d, None, 0, w.data_ptr(), rows, d, 1e-6, tp.FP32, None, y.data_ptr(),
                                         q.data_ptr(), scale.data_ptr(), torch.cuda.current_stream().cuda_stream)
    assert st == tp.TP_OK
    assert torch.equal(scale, (y.abs().amax(1).double() / 127).float())
    ratio = torch.where(scale[:, None] > 0, y.double() / scale.double()[:, None], 0.0)
    want = ratio.round().clamp(-127, 127)
    assert int((q.double() != want).sum()) == 0, float((q.double() - ratio).abs().max())


# ------------------------------------------------------------ gated block
@pytest.mark.parametrize("rows", [60, 2000])
def test_gelu_tail(tp, rows):  # noqa: F811
    """y = GELU(v) exactly once rounded (one pair, u = 1, Wd = 1), out to where
    it leaves the normal numbers: half a step of bf16, and 2^-15 of the value for
    an exponential of up to -84 in fp32.  Then its gradient at u, dh act(v)."""
    v = torch.linspace(-12.9, 12.9, rows, device="cuda").to(torch.bfloat16)
    x = torch.stack([v, torch.ones_like(v)], 1).contiguous()
    wgu = torch.eye(2, device="cuda", dtype=torch.bfloat16)
    wd = torch.ones(1, 1, device="cuda", dtype=torch.bfloat16)
    y, saved = tp.gated_forward(x, wgu, wd, "gelu", save=True)
    z = v.double()
    ref = z * 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
    step = lambda r: torch.exp2(torch.floor(torch.log2(r.abs().clamp(min=1e-300))) - 8)  # noqa: E731
    _within(y[:, 0], ref, step(ref) + 2.0 ** -15 * ref.abs(), "gelu")
    dy = torch.full((rows, 1), 1.5, device="cuda", dtype=torch.bfloat16)
    dx = tp.gated_backward(dy, x, wgu, wd, saved)[0]
    _within(dx[:, 1], 1.5 * ref, step(1.5 * ref) + 2.0 ** -15 * 1.5 * ref.abs(), "du")


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("rows,at", [(1, 0), (24, 23), (1100, 0), (1100, 37), (1100, 1099)])
def test_kept_values_have_24_bits(tp, act, rows, at):  # noqa: F811
    """act(g) and u act'(g) are kept to 16 significant bits: one row has a
    gradient, so that dW_gu = [dg du]^T x has one term and is rounded only where
    dg and du are, half a step of bf16; 2^-15 more for what was kept and
    for the activation.  Kept as bf16 they would be off by up to a step (that
    more than one value in ten shows it is checked with the oracle).  By both kernels that
    keep them: up to 1024 rows of odd widths and above."""
    f = 999
    g = _gen(rows + at)
    x = torch.exp2(torch.randint(-1, 2, (rows, 1), generator=g, device="cuda").float()).to(torch.bfloat16)
    wgu = (1.5 * torch.randn(2 * f, 1, generator=g, device="cuda")).to(torch.bfloat16)
    wd = torch.randn(1, f, generator=g, device="cuda").to(torch.bfloat16)
    dy = torch.zeros(rows, 1, device="cuda", dtype=torch.bfloat16)
    dy[at] = 1.5
    _, saved = tp.gated_forward(x, wgu, wd, act, save=True)
    _, dw, _ = tp.gated_backward(dy, x, wgu, wd, saved)
    xr = float(x[at, 0])
    gate, up = wgu[:f, 0].double() * xr, wgu[f:, 0].double() * xr
    a, d = _act64(act, gate)
    dh = 1.5 * wd[0].double()
    ref = torch.cat([dh * up * d, dh * a]) * xr
    step = torch.exp2(torch.floor(torch.log2(ref.abs().clamp(min=1e-30))) - 8)
    # act' is 1 + ...: a difference near its zero, good to 2^-20 of its terms
    slack = 2.0 ** -15 * ref.abs() + torch.cat([(dh * up).abs() * 2.0 ** -18, torch.zeros_like(dh)]) * xr
    _within(dw[:, 0], ref, step + slack, (act, rows))
    coarse = torch.cat([dh.float() * (up * d).to(torch.bfloat16).float(), dh.float() * a.to(torch.bfloat16).float()])
    coarse = coarse.to(torch.bfloat16).double() * xr
    for half in (slice(0, f), slice(f, 2 * f)):
        over = ((coarse - ref).abs() > step + slack)[half]
        assert float(over.double().mean()) > 0.1, (act, half)


# ----------------------------------------------------------------- give-up path
def test_wait_gives_up(tp):  # noqa: F811
    """A cluster's sums that are never announced: the clusters that wait for
    them give up after the limit, the launch ends, every stream's check says
    so once, and the next calls are right."""
    L = tp.load_library()
    # dW's few tiles of a long reduction, whose K blocks are shared out
    x, wgu, wd, dy = _gated_case(torch.bfloat16, 20011, 256, 256, 256, 3)
    y, saved = tp.gated_forward(x, wgu, wd, save=True)
    ref = tp.gated_backward(dy, x, wgu, wd, saved)
    other = torch.cuda.Stream()
    tp.ops_check()
    tp.ops_check(other)
    assert L.pack_debug_ops_withhold() == tp.TP_OK
    tp.gated_backward(dy, x, wgu, wd, saved)
    torch.cuda.synchronize()
    for stream in (other, None):               # neither takes the other's report
        with pytest.raises(tp.TabpackError) as ei:
            tp.ops_check(stream)
        assert ei.value.status == tp.TP_ETIMEOUT and "site 47" in str(ei.value)
        tp.ops_check(stream)
    for a, b in zip(tp.gated_backward(dy, x, wgu, wd, saved), ref):
        assert torch.equal(a, b)
    tp.ops_check()
    tp.ops_check(other)


@pytest.mark.parametrize("rows,d,f,o", [(4043, 5, 2354, 477), (2048, 64, 2048, 512), (4000, 40, 1000, 300)])
def test_gated_backward_between_forwards(tp, rows, d, f, o):  # noqa: F811
    """The same bits in 1500 backward passes, each right after two forward ones
    (one pass in seven of the first shape, otherwise, had pieces of what comes
    into shared memory for the next chunk)."""
    x, wgu, wd, dy = _gated_case(torch.bfloat16, rows, d, f, o, 5)
    _, saved = tp.gated_forward(x, wgu, wd, "gelu", save=True)
    ref = tp.gated_backward(dy, x, wgu, wd, saved)
    bad = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(1500):
        hold = tp.gated_forward(x, wgu, wd, "gelu", save=True)
        tp.gated_forward(x, wgu, wd, "gelu")
        got = tp.gated_backward(dy, x, wgu, wd, saved)
        for a, b in zip(got, ref):
            bad += (a != b).any()
    del hold
    assert int(bad) == 0
    tp.ops_check()
