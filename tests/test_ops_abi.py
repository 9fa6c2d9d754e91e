"""Argument checks and workspace sizes of the student operators
(include/tabpack_ops.h), without a GPU: every refusal comes before the first
CUDA call."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

SOME = ctypes.c_void_p(4096)   # never read: the calls end before any launch
ODD = ctypes.c_void_p(4097)


@pytest.fixture(scope="module")
def tp():
    from paper_2607_05380_gb300 import build
    build.build()
    import paper_2607_05380_gb300 as tpm
    return tpm


def _bytes(fn, *a):
    v = ctypes.c_int64(-1)
    return fn(*a, ctypes.byref(v)), v.value


def test_workspace_sizes(tp):
    L = tp.load_library()
    s, f, b = (ctypes.c_int64() for _ in range(3))
    assert L.pack_gated_bytes(100, 64, 72, 64, tp.BF16, ctypes.byref(s), ctypes.byref(f), ctypes.byref(b)) == tp.TP_OK
    assert s.value >= 3 * 100 * 72 * 2 and f.value >= 100 * 72 * 2 and b.value >= 2 * 100 * 72 * 2
    s32 = ctypes.c_int64()
    assert L.pack_gated_bytes(100, 64, 72, 64, tp.FP32, ctypes.byref(s32), None, None) == tp.TP_OK
    assert s32.value >= 100 * 72 * (6 + 4 + 4)
    assert L.pack_gated_bytes(0, 64, 72, 64, tp.BF16, ctypes.byref(s), ctypes.byref(f), ctypes.byref(b)) == tp.TP_OK
    assert (s.value, f.value, b.value) == (0, 0, 0)
    # beyond 2^31 bytes and elements
    assert L.pack_gated_bytes(1 << 20, 4096, 8192, 4096, tp.BF16, ctypes.byref(s), ctypes.byref(f), ctypes.byref(b)) == tp.TP_OK
    assert s.value >= 3 * (1 << 20) * 8192 * 2
    assert _bytes(L.pack_rms_norm_bytes, 5, 100) == (tp.TP_OK, 400)
    st, n = _bytes(L.pack_product_q8_bytes, 1000, 100, 30, tp.BF16)
    assert st == tp.TP_OK and n >= 0
    assert _bytes(L.pack_product_q8_bytes, 0, 100, 30, tp.BF16) == (tp.TP_OK, 0)
    assert _bytes(L.pack_distill_bytes, 3, 70) == (tp.TP_OK, 840)


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(rows=1 << 31), dict(d=0), dict(f=0), dict(d_out=0), dict(d=1 << 18),
                                 dict(act=3), dict(act=-1), dict(prec=2), dict(ldx=63), dict(x=None), dict(wgu=None),
                                 dict(wd=None), dict(y=None), dict(ws=None), dict(ws=ODD), dict(n=0), dict(saved=ODD)])
def test_gated_forward_refusals(tp, bad):
    a = dict(x=SOME, ldx=64, wgu=SOME, wd=SOME, rows=5, d=64, f=72, d_out=64, act=1, prec=0, y=SOME, saved=None, ws=SOME,
             n=1 << 40)
    a.update(bad)
    L = tp.load_library()
    st = L.pack_gated_forward(a["x"], a["ldx"], a["wgu"], a["wd"], a["rows"], a["d"], a["f"], a["d_out"], a["act"],
                              a["prec"], a["y"], a["saved"], a["ws"], a["n"], None)
    assert st == tp.TP_EINVAL and L.pack_last_error(None)


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(d=0), dict(prec=-1), dict(ldx=63), dict(lddy=63), dict(x=None),
                                 dict(dy=None), dict(wgu=None), dict(wd=None), dict(saved=None), dict(saved=ODD), dict(dx=None),
                                 dict(dwgu=None), dict(dwd=None), dict(ws=None), dict(ws=ODD), dict(n=1)])
def test_gated_backward_refusals(tp, bad):
    a = dict(dy=SOME, lddy=64, x=SOME, ldx=64, wgu=SOME, wd=SOME, saved=SOME, rows=5, d=64, f=72, d_out=64, prec=0, dx=SOME,
             dwgu=SOME, dwd=SOME, ws=SOME, n=1 << 40)
    a.update(bad)
    st = tp.load_library().pack_gated_backward(a["dy"], a["lddy"], a["x"], a["ldx"], a["wgu"], a["wd"], a["saved"],
                                               a["rows"], a["d"], a["f"], a["d_out"], a["prec"], a["dx"], a["dwgu"],
                                               a["dwd"], a["ws"], a["n"], None)
    assert st == tp.TP_EINVAL


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(d=0), dict(d=16385), dict(eps=-1.0), dict(eps=float("nan")), dict(prec=7),
                                 dict(ldx=63), dict(ldr=63), dict(x=None), dict(w=None), dict(q=SOME), dict(scale=SOME),
                                 dict(y=None)])
def test_rms_norm_refusals(tp, bad):
    a = dict(x=SOME, ldx=64, r=SOME, ldr=64, w=SOME, rows=5, d=64, eps=1e-6, prec=0, sum=None, y=SOME, q=None, scale=None)
    a.update(bad)
    st = tp.load_library().pack_rms_norm(a["x"], a["ldx"], a["r"], a["ldr"], a["w"], a["rows"], a["d"], a["eps"], a["prec"],
                                         a["sum"], a["y"], a["q"], a["scale"], None)
    assert st == tp.TP_EINVAL


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(d=0), dict(eps=-1.0), dict(prec=7), dict(lds=63), dict(lddy=63),
                                 dict(ldds=63), dict(dy=None), dict(s=None), dict(w=None), dict(dx=None), dict(ws=None),
                                 dict(ws=ODD), dict(n=0)])
def test_rms_norm_backward_refusals(tp, bad):
    a = dict(dy=SOME, lddy=64, s=SOME, lds=64, w=SOME, ds=SOME, ldds=64, rows=5, d=64, eps=1e-6, prec=0, dx=SOME, dw=SOME,
             ws=SOME, n=1 << 30)
    a.update(bad)
    st = tp.load_library().pack_rms_norm_backward(a["dy"], a["lddy"], a["s"], a["lds"], a["w"], a["ds"], a["ldds"], a["rows"],
                                                  a["d"], a["eps"], a["prec"], a["dx"], a["dw"], a["ws"], a["n"], None)
    assert st == tp.TP_EINVAL


def test_sizes_past_the_limits(tp):
    """2^40 elements a matrix, whatever the workspace."""
    L = tp.load_library()
    v = ctypes.c_int64()
    assert L.pack_gated_bytes(1 << 30, 2048, 64, 64, tp.BF16, ctypes.byref(v), None, None) == tp.TP_EINVAL
    assert L.pack_product_q8_bytes(1 << 30, 64, 2048, tp.BF16, ctypes.byref(v)) == tp.TP_EINVAL
    assert L.pack_distill_bytes(2, (1 << 30), ctypes.byref(v)) == tp.TP_EINVAL


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(k=0), dict(n=0), dict(k=1 << 18), dict(prec=3), dict(ldq=63),
                                 dict(q=None), dict(s=None), dict(w=None), dict(ws=None), dict(y=None)])
def test_product_refusals(tp, bad):
    a = dict(q=SOME, ldq=64, s=SOME, w=SOME, ws=SOME, b=None, rows=700, k=64, n=72, prec=0, y=SOME, work=SOME, nb=1 << 40)
    a.update(bad)
    st = tp.load_library().pack_product_q8(a["q"], a["ldq"], a["s"], a["w"], a["ws"], a["b"], a["rows"], a["k"], a["n"],
                                           a["prec"], a["y"], a["work"], a["nb"], None)
    assert st == tp.TP_EINVAL


@pytest.mark.parametrize("bad", [dict(m=0), dict(m=65536), dict(rows=-1), dict(rows=1 << 31), dict(n=1), dict(k=0),
                                 dict(k=129), dict(tau=0.0), dict(tau=-1.0), dict(tau=float("inf")), dict(tau=float("nan")),
                                 dict(alpha=-0.1), dict(alpha=1.1), dict(alpha=float("nan")), dict(prec=2), dict(loss=None),
                                 dict(z=None), dict(ids=None), dict(top=None), dict(ws=None), dict(ws=ODD), dict(nb=4)])
def test_distill_refusals(tp, bad):
    a = dict(z=SOME, m=2, rows=5, n=10, ids=SOME, top=SOME, k=4, y=None, tau=2.0, alpha=0.5, prec=1, loss=SOME, dz=SOME,
             ws=SOME, nb=1 << 30)
    a.update(bad)
    st = tp.load_library().pack_distill(a["z"], a["m"], a["rows"], a["n"], a["ids"], a["top"], a["k"], a["y"], a["tau"],
                                        a["alpha"], a["prec"], a["loss"], a["dz"], a["ws"], a["nb"], None)
    assert st == tp.TP_EINVAL


def test_binding_refuses_cpu_tensors(tp):
    x, w = torch.zeros(2, 8), torch.zeros(16, 8)
    with pytest.raises(ValueError):
        tp.gated_forward(x, w, torch.zeros(8, 8))
    with pytest.raises(ValueError):
        tp.rms_norm(x, torch.ones(8))
    with pytest.raises(ValueError):
        tp.product_q8(x.to(torch.int8), torch.ones(2), w.to(torch.int8), torch.ones(16))
    with pytest.raises(ValueError):
        tp.distill(x, torch.zeros(2, 1, dtype=torch.int32), torch.zeros(2, 1))


def test_no_gpu_is_an_error_status(tp):
    if torch.cuda.is_available():
        pytest.skip("host has a GPU")
    L = tp.load_library()
    st = L.pack_rms_norm(SOME, 8, None, 0, SOME, 2, 8, 1e-6, 0, None, SOME, None, None, None)
    assert st == tp.TP_ECUDA and b"no CUDA device" in L.pack_last_error(None)
