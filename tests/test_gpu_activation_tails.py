"""Activations and their derivatives far from zero, element by element against 64 bits.  One input of 1 and weights z make net inputs of
exactly z; a derivative is the weight gradient of one row of X = 1 and dY = 1, fp32 whatever the type."""
import math

import pytest
import torch

from ffn_util import ACTS, DEV, TYPES, UNIT
from paper_2001_04206_amd import dn
from parity_util import announce

pytestmark = pytest.mark.gpu


def net_inputs(dtype, most):
    return torch.linspace(-most, most, 8 * 97, dtype=torch.float64).to(dtype).to(DEV)


def derivative(dtype, z, act):
    one = torch.ones(1, 1, dtype=dtype, device=DEV)
    dW = torch.full((len(z), 1), float("nan"), device=DEV)
    dn.dn_linear_backward(one, z[:, None].contiguous(), z[None, :].contiguous(), torch.ones_like(z)[None, :], None, dW, None, act=act)
    return dW[:, 0].double().cpu()


def normal64(z):
    return 0.5 * torch.erfc(-z / math.sqrt(2)), torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)


def gelu_unit(z):
    """An argument z / sqrt 2 with two roundings moves its erfc by z^2 times as much relatively, the exponential's by z^2 / 2 times;
    16 units in the last place for either function, a few for the products: 2^-24 (2 z^2 + 40)."""
    return 2.0 ** -24 * (2 * z * z + 40)


def test_gelu_of_fp32():
    """Down to -12, where it is 10^-32 (below -13 the distribution function has no normal fp32 number)."""
    announce("gelu's tail")
    z = net_inputs(torch.float32, 12.0)
    Y = torch.full((1, len(z)), float("nan"), device=DEV)
    dn.dn_linear_forward(torch.ones(1, 1, device=DEV), z[:, None].contiguous(), None, None, Y, act=ACTS["gelu"])
    z64 = z.double().cpu()
    c, p = normal64(z64)
    want, got = z64 * c, Y[0].double().cpu()
    off = (got - want).abs() / (gelu_unit(z64) * want.abs()).clamp(min=1e-300)
    assert off.max() <= 1, (z64[off.argmax()], off.max())
    got, want = derivative(torch.float32, z, ACTS["gelu"]), c + z64 * p
    off = (got - want).abs() / (gelu_unit(z64) * (c + (z64 * p).abs()))
    assert off.max() <= 1, (z64[off.argmax()], off.max())


@pytest.mark.parametrize("act", ["sigmoid", "tanh"])
@pytest.mark.parametrize("kind", TYPES)
def test_derivatives_of_saturated_units(kind, act):
    """A sigmoid's derivative e / (1 + e)^2 with e = exp(-|z|), a tanh's 4 e / (1 + e)^2 with e = exp(-2 |z|), where 1 - f would
    have lost them: 16 units of fp32, in 16 bits 2^-24 |z| times 6 for the exponential's argument, then one rounding to the type, whose
    smallest step (f16) is 2^-24."""
    announce("saturated %s %s" % (act, kind))
    dtype = TYPES[kind]
    z = net_inputs(dtype, 16.0 if act == "sigmoid" else 8.0)
    z64 = z.double().cpu()
    e = torch.exp(-z64.abs() * (1 if act == "sigmoid" else 2))
    want = (1 if act == "sigmoid" else 4) * e / (1 + e) ** 2
    unit = 2.0 ** -24 * 16 if kind == "f32" else 2.0 ** -24 * (16 + 6 * z64.abs()) + UNIT[dtype]
    off = (derivative(dtype, z, ACTS[act]) - want).abs() / (unit * want + (2.0 ** -25 if kind == "f16" else 0))
    assert off.max() <= 1, (z64[off.argmax()], off.max())
