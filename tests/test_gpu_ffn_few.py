"""Few rows (dn_linear_forward and dn_ffn_forward with up to 64 of them): both kernels that may take them, rows that end at odd
places, workspaces of exactly the bytes that were asked for, and the smallest numbers of a type."""
import ctypes as C

import pytest
import torch

from ffn_util import ACTS, DEV, TYPES, Make, close, f64, tolerance
from paper_2001_04206_amd import dn
from parity_util import announce
from test_gpu_ffn import block, linear_case

pytestmark = pytest.mark.gpu


# rows and how a row ends: below 16 bytes, just past them, one short of a block of k, in the middle of one
@pytest.mark.parametrize("rows", [2, 3, 4, 5, 16, 17, 32, 48, 49, 64])
@pytest.mark.parametrize("kind", TYPES)
def test_rows_and_widths(kind, rows):
    for n, m in ((1, 9), (3, 17), (7, 40), (9, 5), (127, 24), (1031, 33), (520, 4099)):
        announce("few rows %s %d x %d x %d" % (kind, rows, n, m))
        linear_case(kind, (rows, n, m), "tanh", bias=True, res=True, drop=0.2, keep=True, pad=0)
        linear_case(kind, (rows, n, m), "linear", bias=False, res=False, drop=0.0, keep=False, pad=1)


# d and f so that the first product, the second, both or neither may be taken by tiles
@pytest.mark.parametrize("shape", [(20, 24, 4104), (20, 4104, 24), (24, 2000, 2000), (40, 7, 3001), (40, 3001, 7), (64, 1, 5000),
                                   (64, 5000, 3), (64, 3000, 2048), (33, 2049, 3001)], ids=str)
@pytest.mark.parametrize("kind", TYPES)
def test_workspace_is_not_left(kind, shape):
    rows, d, f = shape
    announce("few rows, workspace %s %s" % (kind, shape))
    dtype, make, t = block(kind, shape, "silu", True, 0.0, 0)
    code = {"f32": dn.DN_F32, "f16": dn.DN_F16, "bf16": dn.DN_BF16}[kind]
    desc = dn.FfnDesc(code, code, dn.DN_ACT_SILU, rows, d, f, 0, 0, 0, 0.0, 1.0, 0, 0)
    need = dn.lib().dn_ffn_forward_workspace_bytes(C.addressof(desc))
    room = torch.full((need + 2 ** 21,), 0xA5, dtype=torch.uint8, device=DEV)   # whatever is written past its end lands here
    Y = make.out(rows, d)
    dn.dn_ffn_forward(t["X"], t["Wg"], t["bg"], t["Wu"], t["bu"], t["Wd"], t["bd"], t["R"], Y, workspace=room[2 ** 20:2 ** 20 + need])
    assert (room[:2 ** 20] == 0xA5).all() and (room[2 ** 20 + need:] == 0xA5).all()
    w = {k: v.double() for k, v in t.items() if v is not None}
    h = f64(w["X"] @ w["Wg"].t() + w["bg"], "silu") * (w["X"] @ w["Wu"].t() + w["bu"])
    close(Y, h @ w["Wd"].t() + w["bd"] + w["R"], tolerance(dtype, f + d, 2), "%s %s" % (kind, shape))


@pytest.mark.parametrize("rows", [1, 2, 4, 8, 40, 70])
def test_smallest_numbers_of_f16(rows):
    """Operands below 2^-14 keep their value: times 2^10 they add up to numbers that 16 bits hold like any other."""
    announce("smallest numbers, %d rows" % rows)
    make = Make(torch.float16, 2)
    X, W = make(rows, 200, std=2.0 ** -17), make(48, 200, std=2.0 ** 10)
    assert (X.abs() < 2.0 ** -14).all()
    Y, Z = make.out(rows, 48), make.out(48, rows)
    dn.dn_linear_forward(X, W, None, None, Y, act=ACTS["linear"])
    dn.dn_linear_forward(W, X, None, None, Z, act=ACTS["linear"])
    want, tol = X.double() @ W.double().t(), tolerance(torch.float16, 200)
    # elements are about 0.1; close() holds few of them against sizes of 1 to 4
    close(Y.double() * 16, want * 16, tol, "small X")
    close(Z.double() * 16, want.t() * 16, tol, "small W")


def test_not_finite_past_the_end_of_a_row():
    """What lies between rows, and in the row after, takes no part."""
    for kind, dtype in TYPES.items():
        for rows in (1, 3, 20, 64):
            announce("between rows %s %d" % (kind, rows))
            wide, weights = (torch.full((n, 48), float("nan"), dtype=dtype, device=DEV) for n in (rows, 24))
            wide[:, :37] = 1
            weights[:, :37] = 0.5
            Y = torch.full((rows, 24), float("nan"), dtype=dtype, device=DEV)
            dn.dn_linear_forward(wide[:, :37], weights[:, :37], None, None, Y, act=ACTS["linear"])
            assert (Y == 18.5).all()


@pytest.mark.parametrize("rows", [1, 20, 64, 200])
@pytest.mark.parametrize("kind", TYPES)
def test_tensors_that_begin_anywhere(kind, rows):
    """Every tensor one element past a multiple of 16 bytes, with rows whose lengths are such multiples."""
    announce("tensors that begin anywhere %s %d" % (kind, rows))
    dtype, make, t = block(kind, (rows, 128, 256), "silu", True, 0.0, 0)

    def shift(v):
        flat = torch.full((v.numel() + 2,), float("nan"), dtype=v.dtype, device=DEV)
        flat[1:-1] = v.flatten()
        return flat, flat[1:-1].view(v.shape)

    s = {k: shift(v)[1] for k, v in t.items() if v is not None}
    (whole, Y), (_, GU) = shift(make.out(rows, 128)), shift(make.out(rows, 512))
    dn.dn_ffn_forward(s["X"], s["Wg"], s["bg"], s["Wu"], s["bu"], s["Wd"], s["bd"], s["R"], Y, GU)
    w = {k: v.double() for k, v in t.items() if v is not None}
    g, u = w["X"] @ w["Wg"].t() + w["bg"], w["X"] @ w["Wu"].t() + w["bu"]
    close(Y, (f64(g, "silu").to(DEV) * u) @ w["Wd"].t() + w["bd"] + w["R"], tolerance(dtype, 384, 2), "Y")
    close(GU, torch.cat((g, u), 1), tolerance(dtype, 128), "GU")
    assert whole[0].isnan() and whole[-1].isnan()
    dX, dW = shift(make.out(rows, 128))[1], [shift(make.out(*t[k].shape))[1] for k in ("Wg", "Wu", "Wd")]
    dn.dn_ffn_backward(s["X"], s["Wg"], s["Wu"], s["Wd"], s["GU"], s["dY"], dX, dW[0], None, dW[1], None, dW[2], None)
    same, sameW = make.out(rows, 128), [make.out(*t[k].shape) for k in ("Wg", "Wu", "Wd")]
    dn.dn_ffn_backward(t["X"], t["Wg"], t["Wu"], t["Wd"], t["GU"], t["dY"], same, sameW[0], None, sameW[1], None, sameW[2], None)
    assert torch.equal(dX, same) and all(torch.equal(a, b) for a, b in zip(dW, sameW))   # copied to where the other lies: the same sums
