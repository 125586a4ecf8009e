"""Dense layers and gated blocks of shapes that between them take every kernel that the library's rule chooses for them: each tile with each
epilogue, whole and in parts of k, and each kernel for few rows (test_block_kernels.py holds the list against the rule).  Against the
formulas in 64 bits on the device; every tensor that a call writes starts as NaN."""
import pytest
import torch

from ffn_util import ACTS, DEV, TYPES, Make, df64, f64, tolerance
from paper_2001_04206_amd import dn
from parity_util import announce

pytestmark = pytest.mark.gpu

# rows, n_in, n_out and rows, d, f: of 16-bit types and of fp32
LINEAR = {
    16: [(8, 17, 4328), (27, 216, 4352), (47, 224, 4360), (55, 416, 4105), (457, 456, 33), (976, 1291, 1896), (1087, 7505, 67), (1480, 6279, 2889),
         (1605, 2717, 723), (1832, 2435, 7265)],
    32: [(1, 9, 8), (8, 8, 4261), (487, 1328, 1035), (3293, 936, 9)]}
BLOCK = {
    16: [(1, 8, 8), (1, 16, 32), (1, 621, 195), (3, 16, 17), (3, 19, 16), (5, 16, 31), (5, 17, 16), (7, 4201, 24), (8, 16, 4583), (9, 17, 4939),
         (21, 33, 17), (21, 152, 224), (21, 240, 4633), (24, 4232, 19), (27, 19, 4205), (33, 35, 4309), (39, 21, 19), (40, 4265, 27), (47, 136, 352),
         (48, 368, 5973), (49, 376, 4805), (51, 19, 19), (51, 39, 4139), (53, 4472, 17), (64, 280, 208), (69, 463, 8), (403, 73, 8767), (707, 3144, 1317),
         (923, 8328, 72), (2017, 7184, 2051), (2377, 1815, 3487), (2671, 1289, 695), (6576, 2767, 744)],
    32: [(1, 8, 8), (1, 9, 8448), (3, 8, 8), (3, 9, 9), (5, 8, 9), (5, 8, 4849), (5, 11, 4136), (5, 13, 8), (5, 4656, 9), (17, 16, 4541), (19, 9, 8),
         (19, 9, 4161), (19, 4419, 8), (19, 5624, 9), (23, 8, 9), (33, 17, 5848), (33, 4519, 16), (37, 8, 6821), (39, 15, 8), (41, 8, 9), (43, 4112, 15),
         (49, 17, 4625), (51, 8, 5071), (51, 9, 11), (53, 4619, 8), (59, 16, 8), (59, 4129, 15), (71, 9, 225), (231, 259, 9), (2480, 1357, 8),
         (8889, 8, 165)]}


def of(shapes):
    return [pytest.param(kind, s, id="%s-%s" % (kind, "x".join(map(str, s)))) for kind in TYPES for s in shapes[32 if kind == "f32" else 16]]


def near(got, want, tol, what):
    """ffn_util.close() on the device."""
    got = got.double()
    assert got.shape == want.shape and torch.isfinite(got).all(), what
    off = (got - want).abs()
    norm = want.norm().item()
    if want.numel() < 64:
        norm = max(norm, 4 * want.numel() ** 0.5)
    assert off.norm().item() <= tol * norm + 1e-30, "%s: %.3g of %.3g" % (what, off.norm().item() / max(norm, 1e-30), tol)
    worst = (off / want.abs().clamp(min=max(norm / want.numel() ** 0.5, 1e-30))).max().item()
    assert worst <= 8 * tol + 1e-30, "%s: an element is %.3g off, %.3g allowed" % (what, worst, 8 * tol)


def mask(rows, cols, drop, seed, offset):
    if drop == 0:
        return 1.0
    x = torch.ones(rows, cols, device=DEV)
    dn.dn_dropout(x, x, drop, seed, offset)
    return (x != 0).double() * (65536 / (65536 - int(drop * 65536 + 0.5)))


# with everything; with nothing that may be left out
@pytest.mark.parametrize("full", [True, False], ids=["full", "bare"])
@pytest.mark.parametrize("kind,shape", of(LINEAR))
def test_linear(kind, shape, full):
    announce("kernels: linear %s %s %s" % (kind, shape, full))
    dtype, (rows, n, m) = TYPES[kind], shape
    act, drop = ("gelu", 0.25) if full else ("linear", 0.0)
    make = Make(dtype, 21)
    X, W, R, dY = make(rows, n), make(m, n, std=n ** -0.5), make(rows, m), make(rows, m)
    b = make(m, std=0.3) if full else None
    Y, Z = make.out(rows, m), make.out(rows, m) if full else None
    dn.dn_linear_forward(X, W, b, R if full else None, Y, Z, act=ACTS[act], drop=drop, seed=5, offset=6)
    keep = mask(rows, m, drop, 5, 6)
    z = X.double() @ W.double().t() + (b.double() if full else 0)
    near(Y, f64(z, act) * keep + (R.double() if full else 0), tolerance(dtype, n), "Y")
    if full:
        near(Z, z, tolerance(dtype, n), "Z")
    z = make(rows, m) if full else None       # (of size 1, as tolerance() has it; the forward pass's own would do)
    grads = dtype if full else torch.float32
    dX, dW, db = make.out(rows, n), make.out(m, n, dtype=grads), make.out(m, dtype=grads) if full else None
    dn.dn_linear_backward(X, W, z, dY, dX, dW, db, act=ACTS[act], drop=drop, seed=5, offset=6, grad_scale=0.5)
    delta = dY.double() * keep * (df64(z, act) if full else 1)
    near(dX, delta @ W.double(), tolerance(dtype, m, 1 + full), "dX")
    tol = tolerance(dtype, rows, 2) if full else tolerance(torch.float32, rows)      # delta's rounding and the gradient's own
    near(dW, 0.5 * (delta.t() @ X.double()), tol, "dW")
    if full:
        near(db, 0.5 * delta.sum(0), tol, "dbias")


@pytest.mark.parametrize("full", [True, False], ids=["full", "bare"])
@pytest.mark.parametrize("kind,shape", of(BLOCK))
def test_block(kind, shape, full):
    announce("kernels: block %s %s %s" % (kind, shape, full))
    dtype, (rows, d, f) = TYPES[kind], shape
    act, drop = ("silu", 0.2) if full else ("gelu", 0.0)
    make = Make(dtype, 22)
    X, R, dY, GU = make(rows, d), make(rows, d), make(rows, d), make(rows, 2 * f)
    Wg, Wu, Wd = make(f, d, std=d ** -0.5), make(f, d, std=d ** -0.5), make(d, f, std=f ** -0.5)
    bg, bu, bd = (make(k, std=0.3) if full else None for k in (f, f, d))
    Y, kept = make.out(rows, d), make.out(rows, 2 * f) if full else None
    dn.dn_ffn_forward(X, Wg, bg, Wu, bu, Wd, bd, R if full else None, Y, kept, act=ACTS[act], drop=drop, seed=5, offset=6)
    keep, x, wg, wu, wd = mask(rows, d, drop, 5, 6), X.double(), Wg.double(), Wu.double(), Wd.double()
    g, u = x @ wg.t() + (bg.double() if full else 0), x @ wu.t() + (bu.double() if full else 0)
    y = (f64(g, act) * u) @ wd.t() + (bd.double() if full else 0)
    near(Y, y * keep + (R.double() if full else 0), tolerance(dtype, f + d, 2), "Y")      # H is rounded to the tensors' type
    if full:
        near(kept, torch.cat((g, u), 1), tolerance(dtype, d), "GU")
    grads = torch.float32 if full else dtype
    dX, dW = make.out(rows, d), [make.out(*s, dtype=grads) for s in ((f, d), (f, d), (d, f))]
    db = [make.out(k, dtype=grads) if full else None for k in (f, f, d)]
    dn.dn_ffn_backward(X, Wg, Wu, Wd, GU, dY, dX, dW[0], db[0], dW[1], db[1], dW[2], db[2], act=ACTS[act], drop=drop, seed=5, offset=6, grad_scale=0.25)
    g, u = GU.double().split(f, 1)
    dz = dY.double() * keep
    dh = dz @ wd
    dg, du = dh * u * df64(g, act), dh * f64(g, act)
    near(dX, dg @ wg + du @ wu, tolerance(dtype, 2 * f + d, 2), "dX")
    tol = tolerance(dtype, rows + d, 2)       # dG, dU and H are rounded to the tensors' type
    for name, got, want in zip(("dWg", "dWu", "dWd"), dW, (dg.t() @ x, du.t() @ x, dz.t() @ (f64(g, act) * u))):
        near(got, 0.25 * want, tol, name)
    if full:
        for name, got, want in zip(("dbg", "dbu", "dbd"), db, (dg, du, dz)):
            near(got, 0.25 * want.sum(0), tol, name)


def test_gradients_of_a_long_block():
    """dWg, dWu and dWd of 300007 rows, whose GU is 4.9 GB, in blocks of rows."""
    rows, d, f, dtype = 300007, 24, 4096, torch.bfloat16
    announce("kernels: long block")
    g = torch.Generator(device=DEV).manual_seed(3)
    X, dY, GU = (torch.randn(rows, k, generator=g, device=DEV).to(dtype) for k in (d, d, 2 * f))
    Wg, Wu, Wd = ((torch.randn(a, b, generator=g, device=DEV) * b ** -0.5).to(dtype) for a, b in ((f, d), (f, d), (d, f)))
    dX, dW = torch.full_like(X, float("nan")), [torch.full_like(w, float("nan")) for w in (Wg, Wu, Wd)]
    dn.dn_ffn_backward(X, Wg, Wu, Wd, GU, dY, dX, dW[0], None, dW[1], None, dW[2], None)
    want = [torch.zeros(w.shape, dtype=torch.float64, device=DEV) for w in (Wg, Wu, Wd)]
    for at in range(0, rows, 30011):
        x, dy, gu = (t[at:at + 30011].double() for t in (X, dY, GU))
        a, u = gu.split(f, 1)
        s, dh = torch.sigmoid(a), dy @ Wd.double()
        want[0] += (dh * u * s * (1 + a * (1 - s))).t() @ x
        want[1] += (dh * a * s).t() @ x
        want[2] += dy.t() @ (a * s * u)
    for name, got, w in zip(("dWg", "dWu", "dWd"), dW, want):
        near(got, w, tolerance(dtype, rows + d, 2), name)
