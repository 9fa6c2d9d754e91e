"""Embedding, dropout, layer norm and 8-bit floating point products used
together: the example that trains a network on a table with category columns
and serves it in 8 bits."""
import os
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_05380_gb300 import build
    build.build()
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import category_student
    return category_student


def test_run(example):
    """It runs, and its 8-bit form stays near it: e4m3 rounds each factor by at
    most 2^-4, of random sign over the sums of two layers: well below 2^-2 of the logits."""
    got = example.run(rows=4096, n_val=1024, epochs=1, width=128, blocks=2, quiet=True)
    assert got["loss"] == got["loss"]
    assert got["f8_off"] < 0.25


def _step_inputs(example, rows=300):
    cat, num, y = example.make_table(rows, [4, 60, 900], 9, 5, seed=4)
    net = example.CategoryStudent([4, 60, 900], 9, 5, d_emb=16, width=64, hidden=96, blocks=2, p=0.2, seed=3)
    net.opt.step = lambda: None
    return net, cat, num, y


def test_gradients(example):
    """Every parameter's gradient of one step against autograd in fp32 on the same
    bf16 weights and the same masks, norm-wise.  The chain rounds to bf16 about
    sixteen times between the loss and the table (dropout's and the norms' outputs
    besides the blocks'), each an error of at most 2^-8 of its operand: below
    16 * 2^-8 = 0.0625 in all."""
    import paper_2607_05380_gb300 as tp
    net, cat, num, y = _step_inputs(example)
    ids, rows = net.ids(cat), len(cat)
    p = {k: v.float().clone().requires_grad_(True) for k, v in net.w.items()}
    # the masks as factors, from the operator on ones
    mask = lambda d, site: tp.dropout(torch.ones(rows, d, device="cuda"), net.p, net.seed, 0, site)  # noqa: E731
    e = torch.where((ids >= 0)[..., None], p["table"][ids.clamp(min=0)] * net.scale, 0.0).view(rows, -1)
    out, s = torch.cat([e * mask(net.d_cat, 0), num], 1) @ p["in"].T, None
    for k in range(2):
        s = out if s is None else out + s
        n = torch.nn.functional.layer_norm(s, (64,), p["norm", k], p["bias", k], 1e-5)
        gate, up = (n @ p["gate_up", k].T).chunk(2, 1)
        out = (torch.nn.functional.silu(gate) * up) @ p["down", k].T * mask(64, 1 + k)
    z = torch.nn.functional.layer_norm(out + s, (64,), p["norm", "last"], p["bias", "last"], 1e-5) @ p["head"].T
    loss = torch.nn.functional.cross_entropy(z, y.long())
    loss.backward()
    got = net.step(cat, num, y)
    want = float(loss.detach())
    assert abs(float(got[0]) - want) <= 0.01 * want
    for k, v in net.w32.items():
        off = float((v.grad - p[k].grad).norm() / p[k].grad.norm())
        assert off < 0.0625, (k, off)


def test_steps_repeat(example):
    """The same steps give the same bits, here and on another stream."""
    runs = []
    for stream in (None, None, torch.cuda.Stream()):
        net, cat, num, y = _step_inputs(example, 2000)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            net.step(cat, num, y)
        torch.cuda.synchronize()
        runs.append({k: v.grad.clone() for k, v in net.w32.items()})
    for other in runs[1:]:
        assert torch.equal(runs[0]["table"], other["table"])
        assert all(torch.equal(runs[0][k], other[k]) for k in (("norm", 0), ("bias", "last")))


def test_captured_steps(example):
    """A pass captured into a graph and replayed on new inputs gives the eager
    pass's bits; two graphs replayed in turn do not disturb each other."""
    import paper_2607_05380_gb300 as tp
    net, cat, num, y = _step_inputs(example, 700)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    ids = net.ids(cat).clone()
    dy = torch.randn(700 * 3, 16, generator=g, device="cuda").bfloat16()
    w, ws = tp.quantise_f8(net.w32["in"], 128)

    def work():
        e = tp.embed(ids, net.w["table"], 2.0, dtype=torch.bfloat16).view(700, -1)
        x = torch.cat([tp.dropout(e, 0.3, 7, 1, 2), num.to(torch.bfloat16)], 1)
        h = tp.product_f8(*tp.quantise_f8(x), w, ws)
        n, s, stats = tp.layer_norm(h, net.w["norm", 0], net.w["bias", 0], save=True)
        return [x, h, n, *tp.layer_norm_backward(n, s, net.w["norm", 0], stats), tp.embed_backward(dy, ids.view(-1), 964)]
    stream = torch.cuda.Stream()
    graphs, outs = [], []
    with torch.cuda.stream(stream):
        work()
        for _ in range(2):
            graph = torch.cuda.CUDAGraph()
            torch.cuda.synchronize()
            with torch.cuda.graph(graph, stream=stream):
                outs.append(work())
            graphs.append(graph)
    for turn in range(4):
        ids.copy_(ids.roll(turn + 1, 0))
        dy.copy_(dy.roll(1, 0))
        torch.cuda.synchronize()
        graphs[turn % 2].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs[turn % 2], work()))
    tp.ops_check()
