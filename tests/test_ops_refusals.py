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
