"""Workspaces that the binding keeps for calls on the default stream: calls of
all sizes, one after another and from several threads, give the bits that the
same calls give alone on streams of their own."""
import threading

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tp():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_05380_gb300 import build
    build.build()
    import paper_2607_05380_gb300 as tpm
    tpm.load_library()
    return tpm


def _calls(tp, seed):
    """Calls with small and large workspaces, in an order that mixes them."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")
    calls = []
    for rows, d, f in ((1, 64, 128), (700, 130, 260), (3, 512, 512), (2500, 256, 512), (40, 96, 1000)):
        x, dy = r(rows, d).bfloat16(), r(rows, d).bfloat16()
        w, down = (r(2 * f, d) / d ** 0.5).bfloat16(), (r(d, f) / f ** 0.5).bfloat16()

        def gated(x=x, dy=dy, w=w, down=down):
            y, saved = tp.gated_forward(x, w, down, act="gelu", save=True)
            return (y, *tp.gated_backward(dy, x, w, down, saved))
        calls.append(gated)
        calls.append(lambda x=x, dy=dy, v=r(d): tp.rms_norm_backward(dy, x, v))
        q = torch.randint(-127, 128, (rows, d), generator=g, device="cuda").to(torch.int8)
        k = torch.randint(-127, 128, (f, d), generator=g, device="cuda").to(torch.int8)
        calls.append(lambda q=q, k=k, a=r(rows).abs(), b=r(f).abs(): (tp.product_q8(q, a, k, b),))
        z, top = r(2, rows, f), torch.rand(rows, 4, generator=g, device="cuda")
        ids = torch.stack([torch.randperm(f, generator=g, device="cuda")[:4] for _ in range(rows)]).int()
        calls.append(lambda z=z, ids=ids, top=top: tp.distill(z, ids, top))
    return calls


def _equal(got, ref):
    return all(torch.equal(a, b) for a, b in zip(got, ref))


def test_sizes_in_turn(tp):
    calls = _calls(tp, 1)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        ref = [c() for c in calls]
    torch.cuda.synchronize()
    for order in (range(len(calls)), reversed(range(len(calls)))):
        got = {i: calls[i]() for i in order}
        torch.cuda.synchronize()
        assert all(_equal(got[i], ref[i]) for i in got)
    tp.ops_check()


def test_threads(tp):
    sets = [_calls(tp, 2 + i) for i in range(4)]
    torch.cuda.synchronize()
    ref = [[c() for c in calls] for calls in sets]
    torch.cuda.synchronize()
    bad = []

    def work(i):
        for _ in range(5):
            if not all(_equal(c(), r) for c, r in zip(sets[i], ref[i])):
                bad.append(i)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(sets))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad
    tp.ops_check()
