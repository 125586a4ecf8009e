"""Tensors of more than 2^32 bytes: the last rows of each against their formula, the same rows computed by themselves, or ones."""
import pytest
import torch

from ffn_util import DEV, close, tolerance
from paper_2001_04206_amd import dn
from parity_util import announce

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def filled(rows, cols, seed):
    """Normal numbers, the same 1021 rows over and over: made quickly, and a row read from the wrong place is another one."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    few = torch.randn(1021, cols, generator=g, device=DEV).to(BF16)
    out = torch.empty(rows, cols, dtype=BF16, device=DEV)
    for at in range(0, rows, 1021):
        out[at:at + 1021] = few[:min(1021, rows - at)]
    return out


def test_linear():
    rows, n, m = 70001, 32768, 24       # X: 4.6 GB
    announce("long linear")
    X, W = filled(rows, n, 1), (torch.randn(m, n, device=DEV) * n ** -0.5).to(BF16)
    Y = torch.full((rows, m), float("nan"), dtype=BF16, device=DEV)
    dn.dn_linear_forward(X, W, None, None, Y)
    at = torch.tensor([0, 1, 65535, 65536, 65537, 69999, 70000], device=DEV)
    close(Y[at], X[at].double() @ W.double().t(), tolerance(BF16, n), "Y")
    dY = filled(rows, m, 2)
    dX, dW = torch.full_like(X, float("nan")), torch.full((m, n), float("nan"), device=DEV)
    dn.dn_linear_backward(X, W, None, dY, dX, dW, None, grad_scale=1.0)
    close(dX[at], dY[at].double() @ W.double(), tolerance(BF16, m), "dX")
    cols = torch.tensor([0, 5, 255, 256, 32767], device=DEV)
    close(dW[:, cols], dY.double().t() @ X[:, cols].double(), tolerance(torch.float32, rows), "dW")


def test_wide_weights():
    rows, n, m = 3, 65536, 33000        # W: 4.3 GB
    for rows in (3, 20):
        announce("long weights, %d rows" % rows)
        X, W = filled(rows, n, 3), filled(m, n, 4)
        Y = torch.full((rows, m), float("nan"), dtype=BF16, device=DEV)
        dn.dn_linear_forward(X, W, None, None, Y)
        at = torch.tensor([0, 1, 32766, 32767, 32768, 32999], device=DEV)
        close(Y[:, at], X.double() @ W[at].double().t(), tolerance(BF16, n), "Y")
        del X, W


def test_block():
    rows, d, f = 300007, 24, 4096       # GU: 4.9 GB
    announce("long block")
    X = filled(rows, d, 5)
    Wg, Wu, Wd = ((torch.randn(a, b, device=DEV) * b ** -0.5).to(BF16) for a, b in ((f, d), (f, d), (d, f)))
    Y, GU = torch.full_like(X, float("nan")), torch.full((rows, 2 * f), float("nan"), dtype=BF16, device=DEV)
    dn.dn_ffn_forward(X, Wg, None, Wu, None, Wd, None, None, Y, GU)
    at = torch.tensor([0, 262143, 262144, 300006], device=DEV)
    g, u = X[at].double() @ Wg.double().t(), X[at].double() @ Wu.double().t()
    close(GU[at], torch.cat((g, u), 1), tolerance(BF16, d), "GU")
    close(Y[at], (g * torch.sigmoid(g) * u) @ Wd.double().t(), tolerance(BF16, f + d, 2), "Y")
    dY, dX = filled(rows, d, 6), torch.full_like(X, float("nan"))
    dW = [torch.empty_like(w) for w in (Wg, Wu, Wd)]
    dn.dn_ffn_backward(X, Wg, Wu, Wd, GU, dY, dX, dW[0], None, dW[1], None, dW[2], None)
    g, u = GU[at, :f].double(), GU[at, f:].double()
    s, dh = torch.sigmoid(g), dY[at].double() @ Wd.double()
    want = (dh * u * s * (1 + g * (1 - s))) @ Wg.double() + (dh * g * s) @ Wu.double()
    close(dX[at], want, tolerance(BF16, 2 * f + d, 2), "dX")


def test_norm_and_dropout():
    rows, d = 300007, 8192              # 4.9 GB
    announce("long norm")
    x, b = filled(rows, d, 7), filled(rows, d, 8)
    x_out, n_out = torch.full_like(x, float("nan")), torch.full_like(x, float("nan"))
    dn.dn_norm_forward(x, b, None, None, None, None, None, x_out, n_out)
    few = torch.arange(rows - 700, rows, device=DEV)
    a, c = torch.empty(700, d, dtype=BF16, device=DEV), torch.empty(700, d, dtype=BF16, device=DEV)
    dn.dn_norm_forward(x[few], b[few], None, None, None, None, None, a, c)
    assert torch.equal(a, x_out[few]) and torch.equal(c, n_out[few])
    dx, db = torch.full_like(x, float("nan")), torch.full_like(x, float("nan"))
    dn.dn_norm_backward(x_out, b, None, None, None, None, None, x, dx, db, None, None, None, None, None)
    dn.dn_norm_backward(x_out[few], b[few], None, None, None, None, None, x[few], a, c, None, None, None, None, None)
    assert torch.equal(a, dx[few]) and torch.equal(c, db[few])
    announce("long dropout")
    x.fill_(1)
    dn.dn_dropout(x, dx, 0.5, 3, 4)
    low = torch.ones(rows - 700, 1, dtype=BF16, device=DEV)     # the same rows' first columns by themselves
    assert torch.equal(dx[:rows - 700, :1], torch.where(dx[:rows - 700, :1] == 0, 0.0, 2.0).to(BF16))
    dn.dn_dropout(low, low, 0.5, 3, 4)
    assert torch.equal(low, dx[:rows - 700, :1])
    assert torch.isfinite(dx[-1].float()).all() and abs((dx[-1] == 0).float().mean().item() - 0.5) < 5 * (0.25 / d) ** 0.5
