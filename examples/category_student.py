"""Train one network on a table with category columns, and serve it in 8 bits.

A row's category columns are looked up in one embedding table (a column's values
are a range of its rows; -1 is a missing value), dropped out and joined by the
numeric columns; a residual network of gated blocks with layer norms and dropout
follows.  Served, the input layer and the head are 8-bit floating point products.

    python examples/category_student.py [--rows 32768] [--epochs 4] [--width 256] [--blocks 2]

Prints the validation accuracy of the network and of its 8-bit form.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2607_05380_gb300 as tp  # noqa: E402


class CategoryStudent:
    """fp32 parameters, bf16 copies for the products; sizes: the columns' numbers of values."""

    def __init__(self, sizes, d_num, n_out, d_emb=16, width=256, hidden=512, blocks=2, p=0.1, lr=2e-3, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        linear = lambda o, i: (2 * torch.rand(o, i, generator=g, device="cuda") - 1) / math.sqrt(i)  # noqa: E731
        self.blocks, self.p, self.seed, self.steps = blocks, p, seed, 0
        self.first = torch.tensor([0, *sizes[:-1]], device="cuda").cumsum(0)   # each column's first row of the table
        self.d_cat, self.scale = len(sizes) * d_emb, math.sqrt(d_emb)
        w = {"table": torch.randn(sum(sizes), d_emb, generator=g, device="cuda") / d_emb,
             "in": linear(width, self.d_cat + d_num), "head": linear(n_out, width)}
        for k in range(blocks):
            w["gate_up", k], w["down", k] = linear(2 * hidden, width), linear(width, hidden)
        for k in (*range(blocks), "last"):
            w["norm", k], w["bias", k] = torch.ones(width, device="cuda"), torch.zeros(width, device="cuda")
        self.w32 = w
        self.opt = torch.optim.AdamW(w.values(), lr=lr, weight_decay=1e-3)
        self.refresh()

    def refresh(self):
        """bf16 copies of the matrices that products read; the table is looked up as it is."""
        self.w = {k: v if v.dim() == 1 or k == "table" else v.to(torch.bfloat16) for k, v in self.w32.items()}

    def ids(self, cat):
        """Rows of the table: of column c its value plus the column's first row."""
        return torch.where(cat >= 0, cat + self.first, -1)

    def inputs(self, ids, num):
        e = tp.embed(ids, self.w["table"], self.scale, dtype=torch.bfloat16).view(len(ids), self.d_cat)
        return e, num.to(torch.bfloat16)

    def trunk(self, y, keep=None):
        """From the input layer's output to the last norm's; keep: for a training step, with dropout."""
        w, s = self.w, None
        for k in range(self.blocks):
            n, s, stats = tp.layer_norm(y, w["norm", k], w["bias", k], s, save=True)
            if keep is None:
                y = tp.gated_forward(n, w["gate_up", k], w["down", k])
                continue
            y, saved = tp.gated_forward(n, w["gate_up", k], w["down", k], save=True)
            y = tp.dropout(y, self.p, self.seed, self.steps, 1 + k)
            keep.append((n, s, stats, saved))
        n, s, stats = tp.layer_norm(y, w["norm", "last"], w["bias", "last"], s, save=True)
        return n, s, stats

    def logits(self, cat, num):
        x = torch.cat(self.inputs(self.ids(cat), num), 1)
        return self.trunk(x @ self.w["in"].T)[0] @ self.w["head"].T

    def step(self, cat, num, labels):
        """One training step on a batch; returns the loss (a device tensor)."""
        w, keep, ids = self.w, [], self.ids(cat)
        e, num = self.inputs(ids, num)
        x = torch.cat([tp.dropout(e, self.p, self.seed, self.steps, 0), num], 1)
        n, s, stats = self.trunk(x @ w["in"].T, keep)
        none = torch.full((len(x), 1), -1, dtype=torch.int32, device="cuda")   # no teacher: labels alone
        loss, dz = tp.distill(n @ w["head"].T, none, none.float(), labels, alpha=0.0)
        grad = {"head": dz.T @ n}
        ds, grad["norm", "last"], grad["bias", "last"] = tp.layer_norm_backward(dz @ w["head"], s, w["norm", "last"], stats)
        for k in reversed(range(self.blocks)):
            n, s, stats, saved = keep[k]
            dy = tp.dropout_backward(ds, self.p, self.seed, self.steps, 1 + k)
            dn, grad["gate_up", k], grad["down", k] = tp.gated_backward(dy, n, w["gate_up", k], w["down", k], saved)
            ds, grad["norm", k], grad["bias", k] = tp.layer_norm_backward(dn, s, w["norm", k], stats, ds)
        grad["in"] = ds.T @ x
        de = tp.dropout_backward((ds @ w["in"])[:, :self.d_cat], self.p, self.seed, self.steps, 0)
        grad["table"] = tp.embed_backward(de.view(*ids.shape, -1), ids, len(w["table"]), self.scale)
        for k, v in self.w32.items():
            v.grad = grad[k].float()
        self.opt.step()
        self.refresh()
        self.steps += 1
        return loss

    def quantise(self):
        """The input layer and the head in 8 bits."""
        return tp.quantise_f8(self.w32["in"], 128), tp.quantise_f8(self.w32["head"], 128)

    def logits_f8(self, cat, num, layers):
        x = torch.cat(self.inputs(self.ids(cat), num), 1)
        n, _, _ = self.trunk(tp.product_f8(*tp.quantise_f8(x), *layers[0]))
        return tp.product_f8(*tp.quantise_f8(n), *layers[1], dtype=torch.float32)


def make_table(rows, sizes, d_num, n_out, seed=0):
    """Category values (frequent ones first, some missing), numbers, and labels that depend on both."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    r = lambda *s: torch.rand(*s, generator=g, device="cuda")  # noqa: E731
    size = torch.tensor(sizes, device="cuda")
    cat = (r(rows, len(sizes)) ** 2 * size).long().clamp(max=size - 1)
    num = torch.randn(rows, d_num, generator=g, device="cuda")
    score = num @ torch.randn(d_num, n_out, generator=g, device="cuda")
    for c, k in enumerate(sizes):
        score += torch.randn(k, n_out, generator=g, device="cuda")[cat[:, c]]
    cat = torch.where(r(rows, len(sizes)) < 0.03, -1, cat)
    return cat, num, score.argmax(1).to(torch.int32)


def run(rows=32768, n_val=4096, epochs=4, batch=512, width=256, blocks=2, quiet=False):
    sizes, d_num, n_out = [4, 12, 60, 300, 5000], 11, 7
    cat, num, y = make_table(rows + n_val, sizes, d_num, n_out)
    net = CategoryStudent(sizes, d_num, n_out, width=width, hidden=2 * width, blocks=blocks)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    for _ in range(epochs):
        for i in torch.randperm(rows, generator=g, device="cuda").split(batch):
            loss = net.step(cat[i], num[i], y[i])
    cv, nv, yv = cat[rows:], num[rows:], y[rows:]
    z, z8 = net.logits(cv, nv), net.logits_f8(cv, nv, net.quantise())
    tp.ops_check()
    accuracy = lambda z: float((z.argmax(1) == yv).float().mean())  # noqa: E731
    got = dict(net=accuracy(z), net_f8=accuracy(z8), loss=float(loss[0]),
               f8_off=float((z8 - z.float()).norm() / z.float().norm()))
    if not quiet:
        print(f"validation accuracy: {got['net']:.4f}, in 8 bits {got['net_f8']:.4f}; last loss {got['loss']:.4f}")
    return got


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--rows", type=int, default=32768)
    ap.add_argument("--epochs", type=int, default=4)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--blocks", type=int, default=2)
    a = ap.parse_args()
    run(rows=a.rows, epochs=a.epochs, width=a.width, blocks=a.blocks)
