"""Dense layers with an epilogue, the gated feed-forward block and dropout (dn_linear_*, dn_ffn_*, dn_dropout) against their
formulas in 64 bits.  Every tensor that a call writes starts as NaN."""
import ctypes as C

import numpy as np
import pytest
import torch

from ffn_util import ACTS, DEV, TYPES, Make, close, df64, f64, mask64, numbers, tolerance
from paper_2001_04206_amd import dn
from parity_util import announce

pytestmark = pytest.mark.gpu

# rows, n_in, n_out: one of everything; few rows (at most 64), tiles of 128 with and without 16-byte pieces, k in parts, tiles
# of 256 (from 192 of them on) with rows, columns and k that end inside one
SHAPES = [(1, 1, 1), (1, 64, 16), (1, 4096, 40), (3, 40, 24), (16, 72, 33), (17, 100, 136), (33, 1000, 7), (64, 256, 48), (65, 128, 130),
          (130, 200, 264), (257, 65, 129), (300, 2048, 136), (127, 1021, 777), (3900, 72, 3336), (3900, 3336, 72),
          (70, 3336, 3900)]


def linear_case(kind, shape, act, bias, res, drop, keep, pad, seed=1):
    dtype, (rows, n, m) = TYPES[kind], shape
    make = Make(dtype, seed)
    X, W = make(rows, n, pad=pad), make(m, n, std=n ** -0.5, pad=pad)
    b = make(m, std=0.3) if bias else None
    R = make(rows, m, pad=pad) if res else None
    Y = make.out(rows, m + pad)[:, :m]
    Z = make.out(rows, m) if keep else None
    dn.dn_linear_forward(X, W, b, R, Y, Z, act=ACTS[act], drop=drop, seed=2 ** 63 + 5, offset=2 ** 32 + 7)
    z = X.double() @ W.double().t()
    z = z.cpu() + (b.double().cpu() if bias else 0)
    want = f64(z, act) * mask64(rows, m, drop, 2 ** 63 + 5, 2 ** 32 + 7) + (R.double().cpu() if res else 0)
    what = "%s %s %s" % (kind, shape, act)
    close(Y, want, tolerance(dtype, n), what + " Y")
    if keep:
        close(Z, z, tolerance(dtype, n), what + " Z")


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("kind", TYPES)
def test_linear_forward(kind, shape):
    announce("linear forward %s %s" % (kind, shape))
    linear_case(kind, shape, "gelu", bias=True, res=True, drop=0.25, keep=True, pad=0)
    linear_case(kind, shape, "linear", bias=False, res=False, drop=0.0, keep=False, pad=8)
    linear_case(kind, shape, "silu", bias=False, res=True, drop=0.0, keep=False, pad=3)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("kind", TYPES)
def test_linear_activations(kind, act):
    for shape in ((5, 48, 40), (140, 64, 72)):
        announce("linear activation %s %s %s" % (kind, act, shape))
        linear_case(kind, shape, act, bias=True, res=False, drop=0.0, keep=True, pad=0)


def linear_back_case(kind, shape, act, bias, drop, pad, f32_grads, seed=2, scale=0.5):
    dtype, (rows, n, m) = TYPES[kind], shape
    gtype = torch.float32 if f32_grads else dtype
    make = Make(dtype, seed)
    X, W = make(rows, n, pad=pad), make(m, n, std=n ** -0.5, pad=pad)
    Z, dY = make(rows, m).contiguous(), make(rows, m, pad=pad)
    dX, dW, db = make.out(rows, n), make.out(m, n, dtype=gtype), make.out(m, dtype=gtype) if bias else None
    dn.dn_linear_backward(X, W, None if act == "linear" else Z, dY, dX, dW, db, act=ACTS[act], drop=drop, seed=11, offset=3,
                          grad_scale=scale)
    delta = dY.double().cpu() * mask64(rows, m, drop, 11, 3)
    if act != "linear":
        delta = delta * df64(Z.cpu(), act)
    what = "%s %s %s" % (kind, shape, act)
    # delta is rounded to the tensors' type where an activation makes it new numbers
    mid = 0 if act == "linear" else 1
    close(dX, delta.to(DEV) @ W.double(), tolerance(dtype, m, 1 + mid), what + " dX")
    tol = tolerance(dtype, rows, mid + (not f32_grads)) if mid or not f32_grads else tolerance(torch.float32, rows)
    close(dW, scale * (delta.to(DEV).t() @ X.double()), tol, what + " dW")
    if bias:
        close(db, scale * delta.sum(0), tol, what + " dbias")


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("kind", TYPES)
def test_linear_backward(kind, shape):
    announce("linear backward %s %s" % (kind, shape))
    linear_back_case(kind, shape, "gelu", bias=True, drop=0.25, pad=0, f32_grads=False)
    linear_back_case(kind, shape, "linear", bias=False, drop=0.0, pad=8, f32_grads=True)
    linear_back_case(kind, shape, "linear", bias=True, drop=0.1, pad=3, f32_grads=True)


@pytest.mark.parametrize("act", ACTS)
def test_linear_backward_activations(act):
    for kind in TYPES:
        announce("linear backward activation %s %s" % (kind, act))
        linear_back_case(kind, (40, 48, 72), act, bias=True, drop=0.0, pad=0, f32_grads=False)


# rows, d, f
BLOCKS = [(1, 1, 1), (1, 64, 128), (5, 40, 72), (37, 101, 211), (64, 128, 256), (100, 96, 200), (129, 65, 131), (333, 256, 520),
          (2100, 72, 2968), (70, 2056, 3336), (3000, 40, 4104), (4000, 3336, 24)]


def block(kind, shape, act, bias, drop, pad, seed=3):
    dtype, (rows, d, f) = TYPES[kind], shape
    make = Make(dtype, seed)
    t = {"X": make(rows, d, pad=pad), "Wg": make(f, d, std=d ** -0.5), "Wu": make(f, d, std=d ** -0.5),
         "Wd": make(d, f, std=f ** -0.5), "R": make(rows, d, pad=pad), "dY": make(rows, d, pad=pad), "GU": make(rows, 2 * f)}
    for k, n in (("bg", f), ("bu", f), ("bd", d)):
        t[k] = make(n, std=0.3) if bias else None
    return dtype, make, t


@pytest.mark.parametrize("shape", BLOCKS, ids=str)
@pytest.mark.parametrize("kind", TYPES)
def test_ffn_forward(kind, shape):
    rows, d, f = shape
    for act, bias, drop, pad, keep in (("silu", True, 0.2, 0, True), ("gelu", False, 0.0, 8, False), ("relu", True, 0.0, 3, True)):
        announce("ffn forward %s %s %s" % (kind, shape, act))
        dtype, make, t = block(kind, shape, act, bias, drop, pad)
        Y, GU = make.out(rows, d), make.out(rows, 2 * f) if keep else None
        dn.dn_ffn_forward(t["X"], t["Wg"], t["bg"], t["Wu"], t["bu"], t["Wd"], t["bd"], t["R"], Y, GU, act=ACTS[act], drop=drop,
                          seed=9, offset=1)
        w = {k: v.double() for k, v in t.items() if v is not None}
        g, u = w["X"] @ w["Wg"].t() + w.get("bg", 0), w["X"] @ w["Wu"].t() + w.get("bu", 0)
        y = (f64(g, act) * u) @ w["Wd"].t() + w.get("bd", 0)
        y = y.cpu() * mask64(rows, d, drop, 9, 1) + w["R"].cpu()
        what = "%s %s %s" % (kind, shape, act)
        close(Y, y, tolerance(dtype, f + d, 2), what + " Y")   # H is rounded to the tensors' type
        if keep:
            close(GU, torch.cat((g, u), 1), tolerance(dtype, d), what + " GU")


@pytest.mark.parametrize("f32_grads", [False, True], ids=["own", "f32"])
@pytest.mark.parametrize("shape", BLOCKS, ids=str)
@pytest.mark.parametrize("kind", TYPES)
def test_ffn_backward(kind, shape, f32_grads):
    rows, d, f = shape
    for act, bias, drop, pad in (("silu", True, 0.2, 0), ("gelu", False, 0.0, 3)):
        announce("ffn backward %s %s %s" % (kind, shape, act))
        dtype, make, t = block(kind, shape, act, bias, drop, pad)
        gtype = torch.float32 if f32_grads else dtype
        dX = make.out(rows, d)
        out = {k: make.out(*t[k].shape, dtype=gtype) for k in ("Wg", "Wu", "Wd")}
        out.update({k: make.out(n, dtype=gtype) if bias else None for k, n in (("bg", f), ("bu", f), ("bd", d))})
        dn.dn_ffn_backward(t["X"], t["Wg"], t["Wu"], t["Wd"], t["GU"], t["dY"], dX, out["Wg"], out["bg"], out["Wu"], out["bu"],
                           out["Wd"], out["bd"], act=ACTS[act], drop=drop, seed=9, offset=1, grad_scale=0.25)
        w = {k: v.double() for k, v in t.items() if v is not None}
        g, u = w["GU"][:, :f], w["GU"][:, f:]
        dz = w["dY"] * mask64(rows, d, drop, 9, 1).to(DEV)
        dh = dz @ w["Wd"]
        dg, du = dh * u * df64(g, act), dh * f64(g, act)
        want = {"Wg": dg.t() @ w["X"], "Wu": du.t() @ w["X"], "Wd": dz.t() @ (f64(g, act) * u), "bg": dg.sum(0), "bu": du.sum(0),
                "bd": dz.sum(0)}
        what = "%s %s %s " % (kind, shape, act)
        close(dX, dg @ w["Wg"] + du @ w["Wu"], tolerance(dtype, 2 * f + d, 2), what + "dX")
        for k, v in out.items():
            if v is not None:   # dG, dU and H are rounded to the tensors' type
                close(v, 0.25 * want[k], tolerance(dtype, rows + d, 2), what + "d" + k)


def test_gradients_against_differences():
    """The block's and the layer's gradients against central differences of their own forward passes, in fp32: along a random
    direction of every input, with a step of 2^-7.  The differences' own error is the step's square over the curvature (6e-5)
    and the sums' rounding over the step (2^-24 sqrt(rows d) 2^7, 4e-4 of a derivative of about its size), so 2e-3."""
    announce("gradients against differences")
    make = Make(torch.float32, 5)
    rows, d, f, h = 24, 40, 56, 2.0 ** -7
    p = {"X": make(rows, d), "Wg": make(f, d, std=d ** -0.5), "bg": make(f), "Wu": make(f, d, std=d ** -0.5), "bu": make(f),
         "Wd": make(d, f, std=f ** -0.5), "bd": make(d)}
    dY = make(rows, d)

    def loss(q, gu=None):
        y = make.out(rows, d)
        dn.dn_ffn_forward(q["X"], q["Wg"], q["bg"], q["Wu"], q["bu"], q["Wd"], q["bd"], None, y, gu, drop=0.3, seed=4)
        return (y.double() * dY.double()).sum().item()

    gu = make.out(rows, 2 * f)
    loss(p, gu)
    grad = {k: make.out(*v.shape) for k, v in p.items()}
    dn.dn_ffn_backward(p["X"], p["Wg"], p["Wu"], p["Wd"], gu, dY, grad["X"], grad["Wg"], grad["bg"], grad["Wu"], grad["bu"],
                       grad["Wd"], grad["bd"], drop=0.3, seed=4)
    for k, v in p.items():
        way = make(*v.shape)
        way = way / way.norm() * v.norm() / 4
        up, down = (loss({**p, k: v + s * way}) for s in (h, -h))
        by = (grad[k].double() * way.double()).sum().item()
        size = grad[k].double().norm().item() * way.double().norm().item() / way.numel() ** 0.5
        assert abs((up - down) / (2 * h) - by) <= 2e-3 * max(abs(by), size), (k, (up - down) / (2 * h), by)


# ---- dropout ---------------------------------------------------------------------------------------------------------

def test_dropout_numbers():
    """Kept elements are those whose number is at least t; the generator's first word for a zero counter and key is 6627e8d5."""
    assert [int(v) for v in numbers(1, 8, 0, 0)[0][:2]] == [0xE8D5, 0x6627]
    for kind, dtype in TYPES.items():
        for rows, cols, drop, seed, offset in ((1, 1, 0.5, 0, 0), (3, 37, 0.1, 2 ** 64 - 1, 2 ** 64 - 1), (300, 9, 0.9, 77, 2 ** 32)):
            announce("dropout %s %s" % (kind, (rows, cols, drop)))
            x = Make(dtype, 1)(rows, cols)
            y = torch.full_like(x, float("nan"))
            dn.dn_dropout(x, y, drop, seed, offset)
            t = int(drop * 65536 + 0.5)
            kept = torch.from_numpy(numbers(rows, cols, seed, offset) >= t)
            want = torch.where(kept, x.cpu().float() * np.float32(65536 / (65536 - t)), torch.zeros(())).to(dtype)
            assert torch.equal(y.cpu(), want)


def test_dropout_edges():
    announce("dropout edges")
    x = torch.randn(50, 1000, device=DEV)
    y = torch.full_like(x, float("nan"))
    dn.dn_dropout(x, y, 0.0, 1, 2)
    assert torch.equal(x, y)
    dn.dn_dropout(x, y, 1 - 2 ** -20, 1, 2)             # all but one number in 65536
    assert (y != 0).float().mean().item() < 1e-3
    dn.dn_dropout(x, y, 0.3, 1, 2)
    assert abs((y == 0).float().mean().item() - 0.3) < 5 * (0.21 / x.numel()) ** 0.5
    other = torch.empty_like(x)
    dn.dn_dropout(x, other, 0.3, 1, 3)
    assert abs(((y == 0) & (other == 0)).float().mean().item() - 0.09) < 5 * (0.0819 / x.numel()) ** 0.5
    dn.dn_dropout(x, x, 0.3, 1, 2)                      # in place
    assert torch.equal(x, y)
    bad = torch.full((8, 64), float("inf"), device=DEV)  # what is dropped is zero whatever it was
    bad[::2] = float("nan")
    out = torch.empty_like(bad)
    dn.dn_dropout(bad, out, 0.5, 3, 0)
    kept = torch.from_numpy(numbers(8, 64, 3, 0) >= 32768).to(DEV)
    assert torch.equal(out == 0, ~kept)
    wide = torch.zeros(20, 70, device=DEV)              # rows apart: nothing between them is written
    dn.dn_dropout(torch.ones(20, 37, device=DEV), wide[:, 5:42], 0.5, 3, 0)
    assert wide[:, :5].abs().sum() == 0 and wide[:, 42:].abs().sum() == 0 and wide.abs().sum() > 0


# ---- numbers that are not finite, types' ends -----------------------------------------------------------------------------

@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("shape", [(20, 48, 40), (200, 72, 136), (200, 71, 135)], ids=str)
def test_what_is_not_finite_stays_in_its_row(kind, shape):
    announce("linear not finite %s %s" % (kind, shape))
    rows, n, m = shape
    make = Make(TYPES[kind], 8)
    X, W = make(rows, n), make(m, n)
    X[3, n - 1] = float("nan")
    X[7, 0] = float("inf")
    W[5, 2] = float("inf")
    Y = make.out(rows, m)
    dn.dn_linear_forward(X, W, None, None, Y)
    bad = ~torch.isfinite(Y)
    want = torch.zeros_like(bad)
    want[3] = want[7] = True
    want[:, 5] = True
    assert torch.equal(bad, want)
    dX, dW, db = make.out(rows, n), make.out(m, n), make.out(m)
    dY = make(rows, m)
    dY[2, m - 1] = float("nan")
    X, W = make(rows, n), make(m, n)
    dn.dn_linear_backward(X, W, None, dY, dX, dW, db)
    assert torch.isnan(dX[2]).all() and torch.isfinite(dX[:2]).all() and torch.isfinite(dX[3:]).all()
    assert torch.isnan(dW[m - 1]).all() and torch.isfinite(dW[:m - 1]).all()
    assert torch.isnan(db[m - 1]) and torch.isfinite(db[:m - 1]).all()


@pytest.mark.parametrize("act", ["sigmoid", "tanh", "relu", "silu", "gelu"])
def test_activations_far_out(act):
    """Infinite and very large net inputs: the limits, not NaN."""
    announce("activations far out %s" % act)
    for dtype in TYPES.values():
        z = torch.tensor([[-float("inf"), -3e4, -200.0, -40.0, 40.0, 200.0, 3e4, float("inf")]], device=DEV).to(dtype)
        one, none = torch.ones(1, 1, dtype=dtype, device=DEV), None
        Y = torch.empty(1, 8, dtype=dtype, device=DEV)
        dn.dn_linear_forward(one, z.t().contiguous(), none, none, Y, act=ACTS[act])
        assert not torch.isnan(Y).any(), (act, Y)
        low, high = {"sigmoid": (0, 1), "tanh": (-1, 1), "relu": (0, None), "silu": (0, None), "gelu": (0, None)}[act]
        assert (Y[0, :4].float() - low).abs().max() < 1e-6
        assert torch.equal(Y[0, 4:], torch.full_like(Y[0, 4:], high) if high is not None else z[0, 4:])
        dX, dW = torch.empty(1, 1, dtype=dtype, device=DEV), torch.empty(8, 1, dtype=dtype, device=DEV)
        dn.dn_linear_backward(one, z.t().contiguous(), z, torch.ones_like(z), None, dW, None, act=ACTS[act])
        want = {"sigmoid": (0, 0), "tanh": (0, 0)}.get(act, (0, 1))
        assert (dW[:4].float() - want[0]).abs().max() < 1e-6 and (dW[4:].float() - want[1]).abs().max() < 1e-6


# ---- as calls of a program ---------------------------------------------------------------------------------------------

def test_in_place_residual_and_determinism():
    announce("residual in place")
    for rows in (8, 300):
        make = Make(torch.bfloat16, 4)
        X, W, R = make(rows, 256), make(64, 256, std=1 / 16), make(rows, 64)
        Y = make.out(rows, 64)
        dn.dn_linear_forward(X, W, None, R, Y, drop=0.1, seed=1)
        dn.dn_linear_forward(X, W, None, R, R, drop=0.1, seed=1)
        assert torch.equal(Y, R)
        again = make.out(rows, 64)
        dn.dn_linear_forward(X, W, None, None, Y)
        dn.dn_linear_forward(X, W, None, None, again)
        assert torch.equal(Y, again)


def test_another_stream_and_graph():
    """A training pass on a side stream, then captured in a graph and replayed beside the program's own work."""
    announce("ffn on a stream and in a graph")
    rows, d, f = 150, 64, 136
    dtype, make, t = block("bf16", (rows, d, f), "silu", True, 0.1, 0)
    Y, GU, dX = make.out(rows, d), make.out(rows, 2 * f), make.out(rows, d)
    grads = [make.out(f, d), make.out(f), make.out(f, d), make.out(f), make.out(d, f), make.out(d)]
    spaces = [torch.empty(64 << 20, dtype=torch.uint8, device=DEV) for _ in range(2)]

    def step():
        dn.dn_ffn_forward(t["X"], t["Wg"], t["bg"], t["Wu"], t["bu"], t["Wd"], t["bd"], t["R"], Y, GU, drop=0.1, seed=2,
                          workspace=spaces[0])
        dn.dn_ffn_backward(t["X"], t["Wg"], t["Wu"], t["Wd"], GU, t["dY"], dX, *grads, drop=0.1, seed=2, workspace=spaces[1])

    step()
    torch.cuda.synchronize()
    want = [v.clone() for v in [Y, GU, dX] + grads]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for v in [Y, GU, dX] + grads:
        v.fill_(float("nan"))
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    for v, w in zip([Y, GU, dX] + grads, want):
        assert torch.equal(v, w)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        t["X"].mul_(-1)
        step()
        torch.cuda.synchronize()
        want = [v.clone() for v in [Y, GU, dX] + grads]
        for v in [Y, GU, dX] + grads:
            v.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for v, w in zip([Y, GU, dX] + grads, want):
            assert torch.equal(v, w), k


def test_nothing_outside_is_written():
    """Outputs inside larger buffers, and a workspace of exactly the bytes asked for: what lies around them stays."""
    announce("guards")
    for kind, rows, d, f in (("bf16", 70, 65, 131), ("f32", 129, 40, 72), ("f16", 5, 33, 17)):
        dtype, make, t = block(kind, (rows, d, f), "silu", True, 0.1, 0)
        e = torch.empty((), dtype=dtype).element_size()

        def guarded(*shape):
            n = int(np.prod(shape))
            flat = torch.full((n + 256,), 7.0, dtype=dtype, device=DEV)
            return flat, flat[128:128 + n].view(*shape)

        bufs = {k: guarded(*s) for k, s in (("Y", (rows, d)), ("GU", (rows, 2 * f)), ("dX", (rows, d)), ("Wg", (f, d)), ("bg", (f,)),
                                            ("Wu", (f, d)), ("bu", (f,)), ("Wd", (d, f)), ("bd", (d,)))}
        v = {k: b[1] for k, b in bufs.items()}
        lib = dn.lib()
        desc = dn.FfnDesc(dn._type_of(t["X"], "X"), dn._type_of(t["X"], "X"), dn.DN_ACT_SILU, rows, d, f, 0, 0, 0, 0.1, 1.0, 1, 1)
        need = [lib.dn_ffn_forward_workspace_bytes(C.addressof(desc)), lib.dn_ffn_backward_workspace_bytes(C.addressof(desc))]
        spaces = [torch.full((n + 512,), 99, dtype=torch.uint8, device=DEV) for n in need]
        dn.dn_ffn_forward(t["X"], t["Wg"], t["bg"], t["Wu"], t["bu"], t["Wd"], t["bd"], t["R"], v["Y"], v["GU"], drop=0.1, seed=1,
                          offset=1, workspace=spaces[0][:need[0]])
        dn.dn_ffn_backward(t["X"], t["Wg"], t["Wu"], t["Wd"], t["GU"], t["dY"], v["dX"], v["Wg"], v["bg"], v["Wu"], v["bu"], v["Wd"],
                           v["bd"], drop=0.1, seed=1, offset=1, workspace=spaces[1][:need[1]])
        torch.cuda.synchronize()
        for k, (flat, _) in bufs.items():
            assert (flat[:128] == 7).all() and (flat[-128:] == 7).all(), (kind, k)
        for s, n in zip(spaces, need):
            assert (s[n:] == 99).all(), kind
        assert e in (2, 4)


def test_refusals_of_the_binding():
    x = torch.zeros(4, 8, device=DEV)
    w = torch.zeros(3, 8, device=DEV)
    y = torch.zeros(4, 3, device=DEV)
    bad = [lambda: dn.dn_linear_forward(x.cpu(), w, None, None, y), lambda: dn.dn_linear_forward(x, w.half(), None, None, y),
           lambda: dn.dn_linear_forward(x, w[:, :7], None, None, y), lambda: dn.dn_linear_forward(x, w, None, None, y.t()),
           lambda: dn.dn_linear_forward(x.double(), w, None, None, y), lambda: dn.dn_linear_forward(x.t()[:4], w, None, None, y),
           lambda: dn.dn_linear_forward(x, w, None, None, y, workspace=x), lambda: dn.dn_dropout(x, y, 0.1, 0)]
    for call in bad[:6] + bad[7:]:
        with pytest.raises(TypeError):
            call()
    with pytest.raises(dn.DnError):
        dn.dn_linear_forward(x[:0], w, None, None, y[:0])
    for kw in ({"act": 9}, {"act": dn.DN_ACT_SOFTMAX}, {"drop": 1.0}, {"drop": float("nan")}):
        with pytest.raises(dn.DnError):
            dn.dn_linear_forward(x, w, None, None, y, **kw)
