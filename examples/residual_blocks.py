"""A classifier of residual gated feed-forward blocks, trained and then asked one row at a time, on libdn's calls alone:

    x_0 = GELU(D(X) We^T + be),  n_0 = rms(x_0)                            dn_dropout, dn_linear_forward, dn_norm_forward
    b_l = D(ffn_l(n_l)),  x_{l+1} = x_l + gate_l rms(b_l),  n_{l+1} = rms(x_{l+1})        dn_ffn_forward, dn_norm_forward
    softmax(W n_L + b)                                                     the dense net (dn.Net)

The backward pass starts at the net's dn_input_gradient and goes back through the same calls' counterparts; the fp32 parameters take
dn_sgd_step, and blocks of 16 bits work on rounded copies of them.  PyTorch supplies memory, casts and the random start.

    python examples/residual_blocks.py --type bf16 --width 256 --hidden 512 --blocks 2 --steps 200
"""
import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2001_04206_amd import dn, synth

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
DEV = "cuda:0"


class Blocks:
    def __init__(self, features, width, hidden, classes, blocks, max_rows, dtype=torch.float32, drop=0.0, seed=1):
        self.width, self.hidden, self.blocks, self.dtype, self.drop, self.seed = width, hidden, blocks, dtype, drop, seed
        g = torch.Generator().manual_seed(seed)

        def normal(*shape, std):
            return (torch.randn(shape, generator=g) * std).to(DEV)

        p = {"We": normal(width, features, std=features ** -0.5), "be": torch.zeros(width, device=DEV), "pre0": torch.ones(width, device=DEV)}
        for i in range(blocks):
            p.update({"Wg%d" % i: normal(hidden, width, std=width ** -0.5), "Wu%d" % i: normal(hidden, width, std=width ** -0.5),
                      "Wd%d" % i: normal(width, hidden, std=hidden ** -0.5), "gate%d" % i: torch.full((1, width), 0.5, device=DEV),
                      "post%d" % i: torch.ones(width, device=DEV), "pre%d" % (i + 1): torch.ones(width, device=DEV)})
        self.params = p                                                        # fp32, what the update rule changes
        self.grads = {k: torch.zeros_like(v) for k, v in p.items()}            # sums over the rows of a step
        self.velocity = {k: torch.zeros_like(v) for k, v in p.items()}
        self.w = p if dtype == torch.float32 else {k: v.to(dtype) for k, v in p.items()}   # what the calls read
        self.head = dn.Net([width, classes], [dn.DN_ACT_SOFTMAX], dn.DN_LOSS_CROSS_ENTROPY, max_rows)
        self.head.set_all([(torch.randn(classes, width, generator=g) * width ** -0.5).numpy()], [np.zeros(classes, np.float32)])

    def offset(self, step, which):
        """Another one for every mask of every step."""
        return step * (self.blocks + 1) + which

    def forward(self, X, step=None):
        """n_L.  With a step's number, dropout is on and what the backward pass reads is kept."""
        w, rows, train = self.w, X.shape[0], step is not None
        new = lambda *shape: torch.empty(shape, dtype=self.dtype, device=DEV)
        drop = self.drop if train else 0.0
        X = X.to(self.dtype)
        if drop:
            X, kept = new(*X.shape), X
            dn.dn_dropout(kept, X, drop, self.seed, self.offset(step, self.blocks))
        z, x, n = new(rows, self.width) if train else None, new(rows, self.width), new(rows, self.width)
        dn.dn_linear_forward(X, w["We"], w["be"], None, x, z, act=dn.DN_ACT_GELU)
        dn.dn_norm_forward(x, None, None, None, None, w["pre0"], None, None, n)
        self.kept = [(X, z, x)]
        for i in range(self.blocks):
            b, gu = new(rows, self.width), new(rows, 2 * self.hidden) if train else None
            dn.dn_ffn_forward(n, w["Wg%d" % i], None, w["Wu%d" % i], None, w["Wd%d" % i], None, None, b, gu, drop=drop, seed=self.seed,
                              offset=0 if step is None else self.offset(step, i))
            x, x_in, n, n_in = new(rows, self.width), x, new(rows, self.width), n
            dn.dn_norm_forward(x_in, b, w["gate%d" % i], w["post%d" % i], None, w["pre%d" % (i + 1)], None, x, n)
            if train:
                self.kept.append((n_in, gu, b, x))
        return n

    def backward(self, dn_top, step):
        """The gradients of every parameter, from the derivative with respect to n_L."""
        w, g, rows = self.w, self.grads, dn_top.shape[0]
        new = lambda: torch.empty(rows, self.width, dtype=self.dtype, device=DEV)
        dx, d_n = None, dn_top
        for i in reversed(range(self.blocks)):
            n_in, gu, b, x = self.kept[i + 1]
            dx_in, db, dn_in = new(), new(), new()
            dn.dn_norm_backward(x, b, w["gate%d" % i], w["post%d" % i], None, w["pre%d" % (i + 1)], dx, d_n, dx_in, db, g["gate%d" % i],
                                g["post%d" % i], None, g["pre%d" % (i + 1)], None)
            dn.dn_ffn_backward(n_in, w["Wg%d" % i], w["Wu%d" % i], w["Wd%d" % i], gu, db, dn_in, g["Wg%d" % i], None, g["Wu%d" % i], None,
                               g["Wd%d" % i], None, drop=self.drop, seed=self.seed, offset=self.offset(step, i))
            dx, d_n = dx_in, dn_in
        X, z, x = self.kept[0]
        dx_in = new()
        dn.dn_norm_backward(x, None, None, None, None, w["pre0"], dx, d_n, dx_in, None, None, None, None, g["pre0"], None)
        dn.dn_linear_backward(X, w["We"], z, dx_in, None, g["We"], g["be"], act=dn.DN_ACT_GELU)

    def step(self, X, labels, step, lr, momentum, loss=None):
        """One step of training; `loss` (one fp32 number on the device) receives the mean loss before it."""
        n, rows = self.forward(X, step).float(), X.shape[0]
        self.head.dn_forward(n)
        self.head.dn_backward(labels, loss)
        top = torch.empty(rows, self.width, device=DEV)
        self.head.dn_input_gradient(top)
        self.backward(top.to(self.dtype), step)
        self.head.dn_update(lr, momentum)
        for k, v in self.params.items():
            dn.dn_sgd_step(v, self.grads[k], self.velocity[k], lr / rows, momentum)
            if self.w is not self.params:
                self.w[k].copy_(v)

    def answer(self, X):
        """The classes' probabilities of some rows, one or many."""
        out = torch.empty(X.shape[0], self.head.widths[-1], device=DEV)
        self.head.dn_forward(self.forward(X).float(), out)
        return out


def main(argv=None):
    a = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    a.add_argument("--type", choices=TYPES, default="bf16")
    for name, value in (("width", 256), ("hidden", 512), ("blocks", 2), ("features", 64), ("classes", 10), ("rows", 256), ("steps", 200)):
        a.add_argument("--" + name, type=int, default=value)
    a.add_argument("--drop", type=float, default=0.1)
    a.add_argument("--lr", type=float, default=0.05)
    a = a.parse_args(argv)
    batches = 16
    task = synth.learnable((a.features, 8, a.classes), n_samples=(batches + 1) * a.rows, batch=a.rows)
    X, labels = torch.from_numpy(task.X).to(DEV), torch.from_numpy(task.labels).to(DEV)
    net = Blocks(a.features, a.width, a.hidden, a.classes, a.blocks, a.rows, TYPES[a.type], a.drop)
    loss = torch.zeros(1, device=DEV)
    for step in range(a.steps):
        at = step % batches * a.rows
        net.step(X[at:at + a.rows], labels[at:at + a.rows], step, a.lr, 0.9, loss)
        if step % 50 == 0 or step == a.steps - 1:
            print("step %4d  loss %.4f" % (step, loss.item()), flush=True)
    test, want = X[-a.rows:], labels[-a.rows:].long()
    together = net.answer(test)
    print("held out: %.1f %% right" % (100 * (together.argmax(1) == want).float().mean().item()))
    torch.cuda.synchronize()
    start = time.perf_counter()
    alone = torch.cat([net.answer(test[i:i + 1]) for i in range(a.rows)])
    torch.cuda.synchronize()
    print("one row at a time: %.1f us a row, probabilities within %.2g of those of %d rows together"
          % ((time.perf_counter() - start) / a.rows * 1e6, (alone - together).abs().max().item(), a.rows))
    net.head.close()


if __name__ == "__main__":
    main()
