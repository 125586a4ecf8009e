"""Gradients of the dense layer and of the norms against central differences of their own forward calls, in fp32 (the gated block's are
in test_gpu_ffn.py): along a random direction of every input, a quarter of its size, with a step of 2^-7.  The differences' own error is
the step's square over the curvature (6e-5) and the sums' rounding over the step (2^-24 sqrt(rows d) 2^7, 4e-4 of a derivative of
about its size), so 2e-3."""
import pytest
import torch

from ffn_util import ACTS, Make
from paper_2001_04206_amd import dn
from parity_util import announce

pytestmark = pytest.mark.gpu
STEP, TOL = 2.0 ** -7, 2e-3


def against_differences(make, p, loss, grad):
    for k, v in p.items():
        way = make(*v.shape)
        way = way / way.norm() * v.norm() / 4
        up, down = (loss({**p, k: v + s * way}) for s in (STEP, -STEP))
        by = (grad[k].double() * way.double()).sum().item()
        size = grad[k].double().norm().item() * way.double().norm().item() / way.numel() ** 0.5
        assert abs((up - down) / (2 * STEP) - by) <= TOL * max(abs(by), size), (k, (up - down) / (2 * STEP), by)


@pytest.mark.parametrize("rows", [3, 24, 90])
@pytest.mark.parametrize("act", ["linear", "tanh", "gelu", "silu", "sigmoid"])
def test_linear(act, rows):
    announce("linear gradients against differences %s %d" % (act, rows))
    make = Make(torch.float32, 6)
    n, m = 40, 56
    p = {"X": make(rows, n), "W": make(m, n, std=n ** -0.5), "b": make(m)}
    dY = make(rows, m)

    def loss(q, z=None):
        y = make.out(rows, m)
        dn.dn_linear_forward(q["X"], q["W"], q["b"], None, y, z, act=ACTS[act], drop=0.3, seed=4)
        return (y.double() * dY.double()).sum().item()

    z = make.out(rows, m)
    loss(p, z)
    grad = {k: make.out(*v.shape) for k, v in p.items()}
    dn.dn_linear_backward(p["X"], p["W"], z, dY, grad["X"], grad["W"], grad["b"], act=ACTS[act], drop=0.3, seed=4)
    against_differences(make, p, loss, grad)


@pytest.mark.parametrize("group", [1, 7, 24])
@pytest.mark.parametrize("pre", [dn.DN_NORM_RMS, dn.DN_NORM_LAYER])
@pytest.mark.parametrize("post", [dn.DN_NORM_NONE, dn.DN_NORM_RMS, dn.DN_NORM_LAYER])
def test_norm(post, pre, group):
    announce("norm gradients against differences %d %d %d" % (post, pre, group))
    make = Make(torch.float32, 7)
    rows, d = 24, 72
    p = {"x": make(rows, d), "b": make(rows, d), "gate": make(-(-rows // group), d, mean=1.0), "pre_w": make(d, mean=1.0)}
    if post != dn.DN_NORM_NONE:
        p["post_w"] = make(d, mean=1.0)
    if post == dn.DN_NORM_LAYER:
        p["post_b"] = make(d)
    if pre == dn.DN_NORM_LAYER:
        p["pre_b"] = make(d)
    dx_out, dnorm = make(rows, d), make(rows, d)
    how = dict(post=post, pre=pre, scale=0.5, rows_per_gate=group)

    def loss(q, x_out=None):
        x_out, n_out = make.out(rows, d) if x_out is None else x_out, make.out(rows, d)
        dn.dn_norm_forward(q["x"], q["b"], q["gate"], q.get("post_w"), q.get("post_b"), q["pre_w"], q.get("pre_b"), x_out, n_out, **how)
        return (x_out.double() * dx_out.double() + n_out.double() * dnorm.double()).sum().item()

    x_out = make.out(rows, d)
    loss(p, x_out)
    grad = {k: make.out(*v.shape) for k, v in p.items()}
    dn.dn_norm_backward(x_out, p["b"], p["gate"], p.get("post_w"), p.get("post_b"), p["pre_w"], dx_out, dnorm, grad["x"], grad["b"],
                        grad["gate"], grad.get("post_w"), grad.get("post_b"), grad["pre_w"], grad.get("pre_b"), **how)
    against_differences(make, p, loss, grad)
