"""The example of residual blocks, which runs the block's operators together: every gradient of a whole step against 64 bits, a
training run whose loss falls, and single rows against many."""
import os
import sys

import pytest
import torch

from ffn_util import TYPES, UNIT
from paper_2001_04206_amd import synth
from parity_util import announce

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def rms(v, w):
    return v / (v.square().mean(1, keepdim=True) + 1e-5).sqrt() * w


def forward64(net, p, X):
    x = torch.nn.functional.gelu(X @ p["We"].t() + p["be"])
    n = rms(x, p["pre0"])
    for i in range(net.blocks):
        b = (torch.nn.functional.silu(n @ p["Wg%d" % i].t()) * (n @ p["Wu%d" % i].t())) @ p["Wd%d" % i].t()
        x = x + p["gate%d" % i] * rms(b, p["post%d" % i])
        n = rms(x, p["pre%d" % (i + 1)])
    return n


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,width,hidden", [(1, 40, 72), (37, 65, 131), (300, 128, 264)])
def test_gradients_of_a_step(kind, rows, width, hidden):
    """Every value on the way is rounded to the type some 20 times through two blocks and back, each adding its unit roundoff (less:
    2^-9 of a number in the mean for bf16) to what the values before it left, so sqrt(20) unit roundoffs in 2-norm; a factor of 4 for
    what the norms and the gates amplify.  fp32: 2^-24 sqrt(terms) of sums of up to 300 terms at each of them."""
    from residual_blocks import Blocks
    announce("residual blocks' gradients %s %s" % (kind, (rows, width, hidden)))
    dtype = TYPES[kind]
    net = Blocks(50, width, hidden, 5, 2, rows, dtype)
    g = torch.Generator().manual_seed(3)
    X = torch.randn(rows, 50, generator=g).to(dtype).float().cuda()
    top = torch.randn(rows, width, generator=g).to(dtype).cuda()
    n = net.forward(X, 0)
    net.backward(top, 0)
    p = {k: v.double().cpu().requires_grad_() for k, v in net.w.items()}
    want = forward64(net, p, X.double().cpu())
    want.backward(top.double().cpu())
    tol = 4 * 20 ** 0.5 * (UNIT[dtype] if dtype != torch.float32 else 2.0 ** -24 * 300 ** 0.5)
    pairs = [("n", n, want)] + [(k, net.grads[k], v.grad) for k, v in p.items()]
    for k, got, ref in pairs:
        off = (got.double().cpu() - ref.detach()).norm().item() / ref.detach().norm().item()
        assert off <= tol, "%s: %.3g of %.3g" % (k, off, tol)
    net.head.close()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_training_and_single_rows(kind):
    from residual_blocks import Blocks
    announce("residual blocks' training %s" % kind)
    rows, batches = 128, 4
    task = synth.learnable((32, 8, 6), n_samples=batches * rows, batch=rows)
    X, labels = torch.from_numpy(task.X).cuda(), torch.from_numpy(task.labels).cuda()
    net = Blocks(32, 96, 160, 6, 2, rows, TYPES[kind], drop=0.1)
    loss, seen = torch.zeros(1, device="cuda"), []
    for step in range(80):
        at = step % batches * rows
        net.step(X[at:at + rows], labels[at:at + rows], step, 0.05, 0.9, loss)
        seen.append(loss.item())
    assert all(v == v for v in seen)
    assert sum(seen[-batches:]) < 0.5 * sum(seen[:batches]), (seen[:batches], seen[-batches:])
    together = net.answer(X[:8])
    alone = torch.cat([net.answer(X[i:i + 1]) for i in range(8)])
    # the same roundings but for the order of sums, which moves a rounding here and there: one unit of a logit of a few, four times
    assert (alone - together).abs().max().item() <= 16 * UNIT[TYPES[kind]] * (1 if kind == "bf16" else 300 ** 0.5)
    net.head.close()
