"""A row's sum over its choices where these cancel: pairs' results in fewer bits than the sum can bear would show."""
import pytest
import torch

from ffn_util import ACTS, DEV, TYPES, Make, close, df64, f64, tolerance
from paper_2001_04206_amd import dn

pytestmark = pytest.mark.gpu

SHAPES = [(3, 64, 40), (37, 129, 96), (120, 256, 192), (700, 320, 192), (1000, 101, 55), (2048, 512, 264), (4096, 1024, 512)]


def twins(rows, dtype):
    """Two experts that every row takes, with weights 1 and -1; the lists."""
    expert = torch.tensor([0, 1], dtype=torch.int32, device=DEV).expand(rows, 2).contiguous()
    weight = torch.tensor([1.0, -1.0], device=DEV).expand(rows, 2).contiguous()
    lists = [torch.empty(n, dtype=torch.int32, device=DEV) for n in (3, 2 * rows, 2 * rows)]
    dn.dn_route_lists(expert, *lists)
    return weight, lists


def nearly(w, make):
    """w [1][..] and the same with 2^-6 of noise, both of the type."""
    noise = make(*w.shape, std=float(w.double().std()) * 2.0 ** -6)
    return torch.cat((w, (w.double() + noise.double()).to(w.dtype)))


def held(got, one, other, dtype, terms, what):
    """What both pairs round alike (H, or dG and dU) and the result's own rounding count relative to the difference; what each rounds by itself, its fp32
    sum and 2^-17 for 24 bits, relative to a pair's result, which is `times` as large.  With pairs' results rounded to 16 bits it would not pass."""
    want = one - other
    times = (one.norm() / want.norm()).item()
    sums = 2.0 ** -24 * (terms ** 0.5 + 16)
    tol = tolerance(dtype, terms, 2) + 2 * times * (sums + (0 if dtype == torch.float32 else 2.0 ** -17))
    assert times > 20
    if dtype != torch.float32:
        assert ((one.to(dtype).double() - other.to(dtype).double()) - want).norm() > 2 * tol * want.norm()
    close(got, want, tol, what)


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("rows,d,f", SHAPES)
def test_outputs_that_cancel(name, rows, d, f):
    dtype, act = TYPES[name], "silu"
    make = Make(dtype, rows)
    weight, lists = twins(rows, dtype)
    X, Wg, Wu = make(rows, d), make(1, f, d, std=d ** -0.5), make(1, f, d, std=d ** -0.5)
    Wd = nearly(make(1, d, f, std=f ** -0.5), make)
    Y = make.out(rows, d)
    dn.dn_experts_forward(X, torch.cat((Wg, Wg)), torch.cat((Wu, Wu)), Wd, weight, *lists, None, Y, act=ACTS[act])
    x, wg, wu, wd = (t.double() for t in (X, Wg[0], Wu[0], Wd))
    h = f64(x @ wg.T, act) * (x @ wu.T)
    held(Y, h @ wd[0].T, h @ wd[1].T, dtype, d + f, "Y")


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("rows,d,f", SHAPES)
def test_gradients_that_cancel(name, rows, d, f):
    dtype, act = TYPES[name], "silu"
    make = Make(dtype, rows + 1)
    weight, lists = twins(rows, dtype)
    X, dY, Wd, gu = make(rows, d), make(rows, d), make(1, d, f, std=f ** -0.5), make(rows, 2 * f)
    Wg, Wu = (nearly(make(1, f, d, std=d ** -0.5), make) for _ in range(2))
    dX, dW, dweight = make.out(rows, d), [make.out(2, f, d), make.out(2, f, d), make.out(2, d, f)], make.out(rows, 2, dtype=torch.float32)
    dn.dn_experts_backward(X, Wg, Wu, torch.cat((Wd, Wd)), weight, *lists, torch.cat((gu, gu)), dY, dX, *dW, dweight, act=ACTS[act])
    g, u = gu.double().split(f, 1)
    dh = dY.double() @ Wd[0].double()
    dg, du = dh * u * df64(g, act), dh * f64(g, act)
    one, other = (dg @ Wg[e].double() + du @ Wu[e].double() for e in range(2))
    held(dX, one, other, dtype, d + 2 * f, "dX")
