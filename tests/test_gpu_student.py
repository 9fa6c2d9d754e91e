"""The student operators used together: the example that distils a pack's
ensemble into a network of gated blocks and serves it with an 8-bit head."""
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
    import student
    return student


def test_distilled_student(example):
    """A student that only had the teacher's top classes and the labels follows
    the ensemble far above chance (one class in ten), and its 8-bit head gives
    the logits within the quantisation: half a step of 1/127 in each of the two
    factors, over 128 terms of random sign, and the bf16 logits' rounding."""
    got = example.run(rows=8192, n_val=2048, members=4, pack_epochs=2, epochs=4, width=128, blocks=2, quiet=True)
    assert got["loss"] == got["loss"]
    assert got["student"] > 0.3 and got["agree"] > 0.3
    assert got["q8_off"] < 0.05
    assert abs(got["student_q8"] - got["student"]) < 0.05


def test_student_gradients(example):
    """Every parameter's gradient of one step against autograd in fp32 on the
    same bf16 weights, norm-wise.  The chain rounds to bf16 about ten times
    between the loss and the first layer (activations, gradients at the block's
    inner products, outputs), each an error of at most 2^-8 of its operand:
    below 10 * 2^-8 = 0.04 in all."""
    st = example.Student(40, 10, width=64, hidden=96, blocks=2, seed=3)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.randn(300, 40, generator=g, device="cuda")
    ids = torch.stack([torch.randperm(10, generator=g, device="cuda")[:3] for _ in range(300)]).to(torch.int32)
    top = torch.randn(300, 3, generator=g, device="cuda")
    y = torch.randint(0, 10, (300,), generator=g, device="cuda").to(torch.int32)
    p = {k: v.float().clone().requires_grad_(True) for k, v in st.w.items()}
    norm = lambda v, w: v * torch.rsqrt((v * v).mean(1, keepdim=True) + 1e-6) * w  # noqa: E731
    out, s = x.to(torch.bfloat16).float() @ p["in"].T, None
    for k in range(2):
        s = out if s is None else out + s
        gate, up = (norm(s, p["norm", k]) @ p["gate_up", k].T).chunk(2, 1)
        out = (torch.nn.functional.silu(gate) * up) @ p["down", k].T
    z = norm(out + s, p["norm"]) @ p["head"].T
    t = torch.softmax(top / 2.0, 1)
    lq = torch.log_softmax(z / 2.0, 1)
    kd = 4.0 * (t * (t.log() - torch.gather(lq, 1, ids.long()))).sum(1)
    loss = (0.7 * kd + 0.3 * torch.nn.functional.cross_entropy(z, y.long(), reduction="none")).mean()
    loss.backward()
    st.opt.step = lambda: None
    got = st.step(x, ids, top, y)
    want = float(loss.detach())
    assert abs(float(got[0]) - want) <= 0.01 * want
    for k, v in st.p.items():
        off = float((v.grad - p[k].grad).norm() / p[k].grad.norm())
        assert off < 0.04, (k, off)
