"""What the student operators refuse, beyond single bad arguments; without a GPU."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

SOME = ctypes.c_void_p(4096)   # never read: the calls end before any launch


@pytest.fixture(scope="module")
def tp():
    from paper_2607_05380_gb300 import build
    build.build()
    import paper_2607_05380_gb300 as tpm
    return tpm


@pytest.mark.parametrize("tau", [2.0 ** -61, 1e-40, 2.0 ** 61, 1e20, 3e38])
def test_distill_temperature_range(tp, tau):
    """Beyond 2^-60..2^60, tau^2 or 1 / tau leaves fp32's range and the loss would be no number."""
    st = tp.load_library().pack_distill(SOME, 2, 5, 10, SOME, SOME, 4, None, tau, 0.5, 1, SOME, SOME, SOME, 1 << 30, None)
    assert st == tp.TP_EINVAL and b"tau" in tp.load_library().pack_last_error(None)


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


I8, I32, U8 = torch.int8, torch.int32, torch.uint8


def _calls(tp):
    """Each entry point with the descriptions of right arguments."""
    n_saved = ctypes.c_int64()
    assert tp.load_library().pack_gated_bytes(5, 16, 24, 8, 1, ctypes.byref(n_saved), None, None) == tp.TP_OK
    x, w = lambda **k: Fake(5, 16, **k), lambda **k: Fake(16, **k)  # noqa: E731
    gu, down = lambda **k: Fake(48, 16, **k), lambda **k: Fake(8, 24, **k)  # noqa: E731
    return {"gated_forward": (tp.gated_forward, [x, gu, down]),
            "gated_backward": (tp.gated_backward, [lambda **k: Fake(5, 8, **k), x, gu, down,
                                                   lambda **k: Fake(n_saved.value, dtype=U8, **k)]),
            "rms_norm": (tp.rms_norm, [x, w, x]), "rms_norm_q8": (tp.rms_norm_q8, [x, w, x]),
            "rms_norm_backward": (tp.rms_norm_backward, [x, x, w, x]),
            "product_q8": (tp.product_q8, [lambda **k: Fake(5, 16, dtype=I8, **k), lambda **k: Fake(5, **k),
                                           lambda **k: Fake(9, 16, dtype=I8, **k), lambda **k: Fake(9, **k),
                                           lambda **k: Fake(9, **k)]),
            "distill": (tp.distill, [lambda **k: Fake(2, 5, 10, **k), lambda **k: Fake(5, 3, dtype=I32, **k),
                                     lambda **k: Fake(5, 3, **k), lambda **k: Fake(5, dtype=I32, **k)])}


@pytest.mark.parametrize("name", ["gated_forward", "gated_backward", "rms_norm", "rms_norm_q8", "rms_norm_backward",
                                  "product_q8", "distill"])
def test_tensors_of_another_device(tp, name):
    """A kernel reads every tensor on the device it runs on: one of another
    device, whichever it is, is refused before anything is allocated or launched."""
    fn, args = _calls(tp)[name]
    for other in range(len(args)):
        for there in (1, -1):
            with pytest.raises(ValueError, match="device|CUDA"):
                fn(*(a(device=there if i == other else 0) for i, a in enumerate(args)))


BIG = 1 << 32


@pytest.mark.parametrize("name,shapes", [
    ("gated_forward", [(5, BIG + 16), (48, BIG + 16), (8, 24)]), ("gated_forward", [(5, 16), (2 * BIG + 48, 16), (8, BIG + 24)]),
    ("gated_forward", [(5, 16), (48, 16), (BIG + 8, 24)]),
    ("gated_backward", [(5, BIG + 8), (5, 16), (48, 16), (BIG + 8, 24), (1 << 20,)]),
    ("rms_norm", [(5, BIG + 16), (BIG + 16,)]), ("rms_norm_q8", [(5, BIG + 16), (BIG + 16,)]),
    ("rms_norm_backward", [(5, BIG + 16), (5, BIG + 16), (BIG + 16,)]),
    ("product_q8", [(5, BIG + 16), (5,), (9, BIG + 16), (9,)]), ("product_q8", [(5, 16), (5,), (BIG + 9, 16), (BIG + 9,)]),
    ("distill", [(5, BIG + 10), (5, 3), (5, 3)]), ("distill", [(5, 10), (5, BIG + 3), (5, BIG + 3)])])
def test_sizes_past_32_bits(tp, name, shapes):
    """A width of 2^32 + 10 is no width of 10."""
    types = {"product_q8": {0: I8, 2: I8}, "distill": {1: I32}, "gated_backward": {4: U8}}.get(name, {})
    with pytest.raises(ValueError, match="2\\^31"):
        getattr(tp, name)(*(Fake(*s, dtype=types.get(i, torch.float32)) for i, s in enumerate(shapes)))


@pytest.mark.parametrize("n", [2 ** 31 - 1, 2 ** 31 - 512, 2 ** 31 - 1023])
def test_distill_classes_past_the_limit(tp, n):
    """A thread's class number, up to 512 past a row's last, has 32 bits."""
    L = tp.load_library()
    assert L.pack_distill(SOME, 1, 0, n, None, None, 4, None, 2.0, 0.5, 0, SOME, None, None, 0, None) == tp.TP_EINVAL
    assert b"n " in L.pack_last_error(None)
