"""What embedding, dropout, layer norm and the 8-bit floating point products
refuse, and their workspace sizes; without a GPU: every refusal comes before the
first CUDA call."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

SOME = ctypes.c_void_p(4096)   # never read: the calls end before any launch
ODD = ctypes.c_void_p(4097)
MANY = 1 << 40


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
    for n, vocab, d in ((257, 1, 1), (5000, 300, 33), (50000, 1 << 20, 64), (2000000, 7, 128), (1 << 22, 1 << 30, 256)):
        st, b = _bytes(L.pack_embed_bytes, n, vocab, d)
        # two lists of ids and places, a byte per row of the table
        assert st == tp.TP_OK and b >= 16 * n + vocab
        assert b <= 24 * n + vocab + 2 * (n // 64 + 2) * (d * 4 + 4) + 65536
    assert _bytes(L.pack_embed_bytes, 0, 10, 10) == (tp.TP_OK, 0)
    assert _bytes(L.pack_embed_bytes, 256, 10, 10) == (tp.TP_OK, 0)   # a few tokens are not sorted
    assert _bytes(L.pack_layer_norm_bytes, 5, 100) == (tp.TP_OK, 5 * 2 * 100 * 4)
    assert _bytes(L.pack_layer_norm_bytes, 0, 100) == (tp.TP_OK, 0)
    assert _bytes(L.pack_product_f8_bytes, 1000, 100, 300, 1) == (tp.TP_OK, 0)
    assert _bytes(L.pack_product_f8_bytes, 0, 100, 300, 0) == (tp.TP_OK, 0)
    st, b = _bytes(L.pack_product_f8_bytes, 100000, 101, 300, 0)
    assert st == tp.TP_OK and b >= 100300 * 112


@pytest.mark.parametrize("bad", [dict(size=2), dict(size=0), dict(n=-1), dict(n=1 << 31), dict(vocab=0), dict(vocab=-5),
                                 dict(vocab=(1 << 31) - 1), dict(d=0), dict(d=1 << 18), dict(tprec=2), dict(prec=-1), dict(ld=15),
                                 dict(ids=None), dict(table=None), dict(out=None), dict(ids=ODD), dict(n=1 << 30, d=2048, ld=2048)])
def test_embed_refusals(tp, bad):
    a = dict(ids=SOME, size=4, n=5, table=SOME, ld=16, vocab=9, d=16, tprec=1, prec=0, out=SOME)
    a.update(bad)
    L = tp.load_library()
    assert L.pack_embed(a["ids"], a["size"], a["n"], a["table"], a["ld"], a["vocab"], a["d"], 1.0, a["tprec"], a["prec"], a["out"],
                        None) == tp.TP_EINVAL and L.pack_last_error(None)
    assert L.pack_embed_backward(a["table"], a["ld"], a["ids"], a["size"], a["n"], a["vocab"], a["d"], 1.0, a["prec"], a["tprec"],
                                 a["out"], SOME, MANY, None) == tp.TP_EINVAL


@pytest.mark.parametrize("ws,n", [(None, MANY), (ODD, MANY), (SOME, 100)])
def test_workspaces_refused(tp, ws, n):
    L = tp.load_library()
    assert L.pack_embed_backward(SOME, 16, SOME, 4, 500, 9, 16, 1.0, 0, 1, SOME, ws, n, None) == tp.TP_EINVAL
    assert L.pack_layer_norm_backward(SOME, 64, SOME, 64, SOME, SOME, None, 0, 5, 64, 0, SOME, SOME, SOME, ws, n, None) == tp.TP_EINVAL
    assert L.pack_product_f8(SOME, 101, SOME, SOME, 101, SOME, None, 1000, 101, 300, 0, SOME, ws, n, None) == tp.TP_EINVAL


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(rows=1 << 31), dict(d=0), dict(d=1 << 18), dict(p=1.0), dict(p=-0.1),
                                 dict(p=float("nan")), dict(prec=2), dict(ldx=15), dict(ldr=15), dict(x=None), dict(y=None),
                                 dict(rows=1 << 30, d=4096, ldx=4096, ldr=4096)])
def test_dropout_refusals(tp, bad):
    a = dict(x=SOME, ldx=16, res=SOME, ldr=16, rows=5, d=16, p=0.5, prec=0, y=SOME)
    a.update(bad)
    L = tp.load_library()
    assert L.pack_dropout(a["x"], a["ldx"], a["res"], a["ldr"], a["rows"], a["d"], a["p"], 1, 2, 3, a["prec"], a["y"],
                          None) == tp.TP_EINVAL and L.pack_last_error(None)


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(rows=1 << 31), dict(d=0), dict(d=16385), dict(eps=-1.0), dict(eps=float("nan")),
                                 dict(prec=3), dict(ldx=63), dict(ldr=63), dict(x=None), dict(w=None),
                                 dict(sum=None, y=None, stats=None), dict(stats=ctypes.c_void_p(4100))])
def test_layer_norm_refusals(tp, bad):
    a = dict(x=SOME, ldx=64, res=SOME, ldr=64, w=SOME, rows=5, d=64, eps=1e-5, prec=0, sum=SOME, y=SOME, stats=SOME)
    a.update(bad)
    L = tp.load_library()
    assert L.pack_layer_norm(a["x"], a["ldx"], a["res"], a["ldr"], a["w"], None, a["rows"], a["d"], a["eps"], a["prec"], a["sum"],
                             a["y"], a["stats"], None) == tp.TP_EINVAL and L.pack_last_error(None)


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(d=0), dict(prec=3), dict(lddy=63), dict(lds=63), dict(ldd=63), dict(dy=None),
                                 dict(s=None), dict(w=None), dict(stats=None), dict(stats=ctypes.c_void_p(4100)), dict(dx=None)])
def test_layer_norm_backward_refusals(tp, bad):
    a = dict(dy=SOME, lddy=64, s=SOME, lds=64, w=SOME, stats=SOME, dsum=SOME, ldd=64, rows=5, d=64, prec=0, dx=SOME)
    a.update(bad)
    L = tp.load_library()
    assert L.pack_layer_norm_backward(a["dy"], a["lddy"], a["s"], a["lds"], a["w"], a["stats"], a["dsum"], a["ldd"], a["rows"],
                                      a["d"], a["prec"], a["dx"], SOME, SOME, SOME, MANY, None) == tp.TP_EINVAL


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(rows=1 << 31), dict(k=0), dict(k=1 << 18), dict(block=64), dict(block=0),
                                 dict(prec=2), dict(ldx=63), dict(ldq=63), dict(x=None), dict(q=None), dict(scale=None),
                                 dict(rows=128 * 65536, block=128)])
def test_quantise_f8_refusals(tp, bad):
    a = dict(x=SOME, ldx=64, rows=5, k=64, block=1, prec=0, q=SOME, ldq=64, scale=SOME)
    a.update(bad)
    L = tp.load_library()
    assert L.pack_quantise_f8(a["x"], a["ldx"], a["rows"], a["k"], a["block"], a["prec"], a["q"], a["ldq"], a["scale"],
                              None) == tp.TP_EINVAL and L.pack_last_error(None)


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(rows=1 << 31), dict(k=0), dict(n=0), dict(k=1 << 18), dict(n=1 << 18),
                                 dict(prec=2), dict(ldq=63), dict(ldw=63), dict(q=None), dict(scale=None), dict(w=None),
                                 dict(ws=None), dict(y=None), dict(rows=1 << 30, n=4096)])
@pytest.mark.parametrize("rows", [5, 5000])
def test_product_f8_refusals(tp, bad, rows):
    a = dict(q=SOME, ldq=64, scale=SOME, w=SOME, ldw=64, ws=SOME, rows=rows, k=64, n=72, prec=0, y=SOME)
    a.update(bad)
    L = tp.load_library()
    assert L.pack_product_f8(a["q"], a["ldq"], a["scale"], a["w"], a["ldw"], a["ws"], None, a["rows"], a["k"], a["n"], a["prec"],
                             a["y"], SOME, MANY, None) == tp.TP_EINVAL and L.pack_last_error(None)


class Fake:
    """Stands in for a CUDA tensor where only its description is looked at."""

    def __init__(self, *shape, dtype=torch.float32, device=0):
        self.shape, self.dtype, self._device, self.is_cuda = torch.Size(shape), dtype, device, True

    def stride(self):
        return tuple(torch.Size(self.shape[i + 1:]).numel() for i in range(len(self.shape)))

    def dim(self):
        return len(self.shape)

    def is_contiguous(self):
        return True

    def get_device(self):
        return self._device

    def data_ptr(self):
        return 4096


I64, F8 = torch.int64, torch.float8_e4m3fn
CALLS = {"embed": [((7,), I64), ((9, 16), None)], "embed_backward": [((7, 16), None), ((7,), I64)],
         "layer_norm": [((5, 16), None), ((16,), None), ((16,), None), ((5, 16), None)],
         "layer_norm_backward": [((5, 16), None), ((5, 16), None), ((16,), None), ((5, 2), None), ((5, 16), None)],
         "product_f8": [((5, 200), F8), ((5, 2), None), ((150, 200), F8), ((2, 2), None), ((150,), None)],
         "quantise_f8": [((5, 200), None)], "dropout": [((5, 16), None)]}
MORE = {"embed_backward": (9,), "dropout": (0.5, 1)}


def _call(tp, name, tensors, **kw):
    return getattr(tp, name)(*tensors, *MORE.get(name, ()), **kw)


def _fakes(name, bad=None, **kw):
    return [Fake(*s, dtype=t or torch.float32, **(kw if i == bad else {})) for i, (s, t) in enumerate(CALLS[name])]


@pytest.mark.parametrize("name", sorted(CALLS))
def test_tensors_of_another_device(tp, name):
    for other in range(len(CALLS[name])):
        for there in (1, -1)[len(CALLS[name]) == 1:]:   # (one tensor alone: the current device decides)
            with pytest.raises(ValueError, match="device|CUDA"):
                _call(tp, name, _fakes(name, other, device=there))
    with pytest.raises(ValueError, match="device|CUDA"):
        tp.dropout(Fake(5, 16), 0.5, 1, residual=Fake(5, 16, device=1))


@pytest.mark.parametrize("name", sorted(CALLS))
def test_types_and_shapes(tp, name):
    """A tensor of another type, or with a dimension of another size, is refused."""
    for i, (shape, t) in enumerate(CALLS[name]):
        fakes = _fakes(name)
        fakes[i] = Fake(*shape, dtype=torch.int16)
        with pytest.raises(ValueError):
            _call(tp, name, fakes)
        if name in ("quantise_f8", "dropout") or (name, i) in (("embed", 0), ("embed", 1), ("layer_norm", 0)):
            continue   # (the tensor that the sizes are taken from)
        for dim in range(len(shape)):
            fakes = _fakes(name)
            fakes[i] = Fake(*(n + 1 + 128 * (dim == d) if dim == d else n for d, n in enumerate(shape)), dtype=t or torch.float32)
            if name == "embed_backward" and (i, dim) == (0, 1):
                continue   # (any d)
            with pytest.raises(ValueError):
                _call(tp, name, fakes)


BIG = 1 << 32


@pytest.mark.parametrize("name,shapes", [
    ("embed", [(5,), (9, BIG + 16)]), ("embed", [(5,), (BIG + 9, 16)]), ("embed_backward", [(5, BIG + 16), (5,)]),
    ("dropout", [(5, BIG + 16)]), ("layer_norm", [(5, BIG + 16), (BIG + 16,)]),
    ("layer_norm_backward", [(5, BIG + 16), (5, BIG + 16), (BIG + 16,), (5, 2)]), ("quantise_f8", [(5, BIG + 16)]),
    ("product_f8", [(5, BIG + 16), (5, 1), (9, BIG + 16), (1, 1)]), ("product_f8", [(5, 16), (5, 1), (BIG + 9, 16), (1, 1)])])
def test_sizes_past_32_bits(tp, name, shapes):
    """A width of 2^32 + 10 is no width of 10."""
    types = {i: t for i, (_, t) in enumerate(CALLS[name])}
    with pytest.raises(ValueError, match="2\\^31"):
        _call(tp, name, [Fake(*s, dtype=types[i] or torch.float32) for i, s in enumerate(shapes)])


def test_numbers(tp):
    with pytest.raises(ValueError, match="2\\^31"):
        tp.embed_backward(Fake(7, 16), Fake(7, dtype=I64), BIG + 9)
    for kw in (dict(seed=1 << 64), dict(seed=-1), dict(seed=1, step=1 << 32), dict(seed=1, site=-1)):
        with pytest.raises(ValueError, match="bits"):
            tp.dropout(Fake(5, 16), 0.5, **kw)
    with pytest.raises(ValueError, match="block_rows"):
        tp.quantise_f8(Fake(5, 16), 64)
    for fn, a in ((tp.embed, [Fake(7, dtype=I64), Fake(9, 16)]), (tp.embed_backward, [Fake(7, 16), Fake(7, dtype=I64), 9]),
                  (tp.product_f8, _fakes("product_f8"))):
        with pytest.raises(ValueError, match="dtype"):
            fn(*a, dtype=torch.float16)


def test_names(tp):
    """The operators are names of the package."""
    for name in [*CALLS, "dropout_backward"]:
        assert name in dir(tp) and getattr(tp, name) is getattr(tp.ops, name)
