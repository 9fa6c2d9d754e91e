"""Distil a selected ensemble into one network, and serve that in 8 bits.

A pack of MLPs is trained on a synthetic ten-class table and its online
ensemble selected; the ensemble's mean probabilities on the training rows
become the teacher's top logits.  The student is a residual network of gated
blocks (RMS norm, gated feed-forward, residual sum), trained on them with the
student operators; then its head answers in 8 bits.

    python examples/student.py [--rows 32768] [--epochs 6] [--width 256] [--blocks 2]

Prints the validation accuracy of the ensemble, of the student, and of the
student with the 8-bit head.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2607_05380_gb300 as tp  # noqa: E402
from workloads import WORKLOADS, batch_indices, make_data, sample_hparams  # noqa: E402


class Student:
    """Residual network of gated blocks: fp32 parameters, bf16 copies for the products."""

    def __init__(self, d_in, n_out, width=256, hidden=512, blocks=2, act="silu", lr=2e-3, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        linear = lambda o, i: (2 * torch.rand(o, i, generator=g, device="cuda") - 1) / math.sqrt(i)  # noqa: E731
        self.act, self.blocks = act, blocks
        p = {"in": linear(width, d_in), "head": linear(n_out, width), "norm": torch.ones(width, device="cuda")}
        for k in range(blocks):
            p["norm", k] = torch.ones(width, device="cuda")
            p["gate_up", k] = linear(2 * hidden, width)
            p["down", k] = linear(width, hidden)
        self.p = p
        self.opt = torch.optim.AdamW(p.values(), lr=lr, weight_decay=1e-3)
        self.refresh()

    def refresh(self):
        """bf16 copies of the matrices."""
        self.w = {k: v if v.dim() == 1 else v.to(torch.bfloat16) for k, v in self.p.items()}

    def trunk(self, x, keep=None):
        """The residual stream and the last block's output, before the last norm."""
        w = self.w
        y, s = x.to(torch.bfloat16) @ w["in"].T, None
        for k in range(self.blocks):
            n, s = tp.rms_norm(y, w["norm", k], s)
            if keep is None:
                y = tp.gated_forward(n, w["gate_up", k], w["down", k], self.act)
            else:
                y, saved = tp.gated_forward(n, w["gate_up", k], w["down", k], self.act, save=True)
                keep.append((n, s, saved))
        return y, s

    def logits(self, x):
        y, s = self.trunk(x)
        return tp.rms_norm(y, self.w["norm"], s)[0] @ self.w["head"].T

    def step(self, x, ids, top, labels, tau=2.0, alpha=0.7):
        """One training step on a batch; returns the loss (a device tensor)."""
        w, keep = self.w, []
        y, s = self.trunk(x, keep)
        n, s = tp.rms_norm(y, w["norm"], s)
        loss, dz = tp.distill(n @ w["head"].T, ids, top, labels, tau=tau, alpha=alpha)
        grad = {"head": dz.T @ n}
        ds, grad["norm"] = tp.rms_norm_backward(dz @ w["head"], s, w["norm"])
        for k in reversed(range(self.blocks)):
            n, s, saved = keep[k]
            dn, grad["gate_up", k], grad["down", k] = tp.gated_backward(ds, n, w["gate_up", k], w["down", k], saved)
            ds, grad["norm", k] = tp.rms_norm_backward(dn, s, w["norm", k], ds)
        grad["in"] = ds.T @ x.to(torch.bfloat16)
        for k, v in self.p.items():
            v.grad = grad[k].float()
        self.opt.step()
        self.refresh()
        return loss

    def quantise_head(self):
        """int8 head weights with a scale per class."""
        scale = self.p["head"].abs().amax(1) / 127
        return torch.round(self.p["head"] / scale[:, None]).to(torch.int8), scale

    def logits_q8(self, x, head):
        y, s = self.trunk(x)
        q, scale, _ = tp.rms_norm_q8(y, self.w["norm"], s)
        return tp.product_q8(q, scale, *head, dtype=torch.float32)


def teach(online, x, k=4, chunk=8192):
    """The ensemble's k largest mean probabilities of every row, as classes and logits."""
    prob = torch.cat([online.predict(part.contiguous()) for part in x.split(chunk)])
    top = torch.topk(prob, k, 1)
    return top.indices.to(torch.int32).contiguous(), top.values.clamp(min=1e-8).log().contiguous()


def run(rows=32768, n_val=4096, members=8, pack_epochs=3, epochs=6, batch=512, width=256, blocks=2, quiet=False):
    wl = WORKLOADS["large"]
    d = make_data(wl, "cuda", n_train=rows, n_val=n_val)
    hp = sample_hparams(wl, m=members)
    x, y, xv, yv = d["X_train"], d["y_train"], d["X_val"], d["y_val"]
    pack = tp.Pack(wl.d_in, wl.d_out, wl.task, hp["depth"], hp["width"], hp["dropout"], hp["lr"], hp["wd"], max_batch=batch)
    online = tp.OnlineEnsemble(pack, n_val, m_ens=4)
    step = 0
    for epoch in range(pack_epochs):
        for idx in batch_indices(rows, batch, epoch):
            pack.train_step(x, torch.from_numpy(idx).cuda(), y, step)
            step += 1
        if online.epoch(xv, yv):
            break
    accuracy = lambda z: float((z.argmax(1) == yv).float().mean())  # noqa: E731
    ensemble = online.predict(xv)
    ids, top = teach(online, x)
    student = Student(wl.d_in, wl.d_out, width, 2 * width, blocks)
    for epoch in range(epochs):
        for idx in batch_indices(rows, batch, epoch, seed=5):
            i = torch.from_numpy(idx).cuda().long()
            loss = student.step(x[i], ids[i], top[i], y[i])
    z = student.logits(xv)
    z8 = student.logits_q8(xv, student.quantise_head())
    tp.ops_check()
    got = dict(ensemble=accuracy(ensemble), student=accuracy(z), student_q8=accuracy(z8), loss=float(loss[0]),
               agree=float((z.argmax(1) == ensemble.argmax(1)).float().mean()),
               q8_off=float((z8 - z.float()).abs().max() / z.float().abs().max()))
    online.close()
    pack.close()
    if not quiet:
        print(f"validation accuracy: ensemble {got['ensemble']:.4f}, student {got['student']:.4f}, "
              f"with the 8-bit head {got['student_q8']:.4f}; last loss {got['loss']:.4f}")
    return got


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--rows", type=int, default=32768)
    ap.add_argument("--epochs", type=int, default=6)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--blocks", type=int, default=2)
    a = ap.parse_args()
    run(rows=a.rows, epochs=a.epochs, width=a.width, blocks=a.blocks)
