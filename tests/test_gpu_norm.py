"""The norms around a block with its gate, scale and residual (dn_norm_*) against their formulas in 64 bits."""
import pytest
import torch

from ffn_util import DEV, TYPES, Make, close, tolerance
from paper_2001_04206_amd import dn
from parity_util import announce

pytestmark = pytest.mark.gpu

NONE, RMS, LAYER = dn.DN_NORM_NONE, dn.DN_NORM_RMS, dn.DN_NORM_LAYER
# rows, d, rows of a gate: one of everything; every number of threads a row and pieces a thread; groups that end inside a part, parts that
# end inside a group, one row a gate
SHAPES = [(1, 1, 1), (1, 4096, 1), (3, 7, 2), (5, 512, 5), (37, 513, 10), (64, 1021, 64), (9, 2049, 4), (5, 4097, 3), (3, 16384, 3),
          (5000, 40, 1700), (5000, 24, 1), (9000, 16, 7)]


def norm64(v, how, w, b):
    if how == NONE:
        return v
    if how == LAYER:
        v = v - v.mean(1, keepdim=True)
    v = v / (v.square().mean(1, keepdim=True) + 1e-5).sqrt()
    return v * (1 if w is None else w) + (0 if b is None else b)


def tensors(kind, shape, post, pre, gated, weights, seed=1):
    rows, d, per = shape
    make = Make(TYPES[kind], seed)
    t = {"x": make(rows, d, std=2.0, mean=0.5), "b": make(rows, d, mean=0.3),
         "gate": make(-(-rows // per), d, std=0.2, mean=1.0) if gated else None,
         "post_w": make(d, std=0.1, mean=1.0) if post and weights else None, "post_b": make(d, std=0.1) if post == LAYER and weights else None,
         "pre_w": make(d, std=0.1, mean=1.0) if pre and weights else None, "pre_b": make(d, std=0.1) if pre == LAYER and weights else None}
    return make, t


def step64(w, post, per, scale):
    rows = w["b"].shape[0]
    gate = 1 if w.get("gate") is None else w["gate"].repeat_interleave(per, 0)[:rows]
    return scale * gate * norm64(w["b"], post, w.get("post_w"), w.get("post_b"))


KINDS = [(RMS, RMS, True, True), (LAYER, LAYER, True, True), (NONE, LAYER, False, True), (RMS, NONE, True, False), (NONE, RMS, True, False)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("kind", TYPES)
def test_forward(kind, shape):
    rows, d, per = shape
    for post, pre, gated, weights in KINDS:
        announce("norm forward %s %s post %d pre %d" % (kind, shape, post, pre))
        make, t = tensors(kind, shape, post, pre, gated, weights)
        x_out, n_out = make.out(rows, d), make.out(rows, d) if pre else None
        dn.dn_norm_forward(t["x"], t["b"], t["gate"], t["post_w"], t["post_b"], t["pre_w"], t["pre_b"], x_out, n_out, post=post, pre=pre,
                           scale=0.5, rows_per_gate=per)
        w = {k: v.double() for k, v in t.items() if v is not None}
        x = w["x"] + step64(w, post, per, 0.5)
        what = "%s %s %d %d " % (kind, shape, post, pre)
        close(x_out, x, tolerance(TYPES[kind], d), what + "x'")
        # a centred row of one element is all rounding, and so is what is near it
        if pre and not (pre == LAYER and d == 1):
            close(n_out, norm64(x, pre, w.get("pre_w"), w.get("pre_b")), tolerance(TYPES[kind], d), what + "n")


@pytest.mark.parametrize("f32_grads", [False, True], ids=["own", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("kind", TYPES)
def test_backward(kind, shape, f32_grads):
    rows, d, per = shape
    dtype = TYPES[kind]
    for post, pre, gated, weights in KINDS:
        if d == 1 and LAYER in (post, pre):
            continue          # the derivative of a norm of one element is 0 but for rounding
        announce("norm backward %s %s post %d pre %d" % (kind, shape, post, pre))
        make, t = tensors(kind, shape, post, pre, gated, weights)
        gtype = torch.float32 if f32_grads else dtype
        dx_out, dnorm = make(rows, d), make(rows, d)
        dx, db = make.out(rows, d), make.out(rows, d)
        out = {k: None if t[k] is None else make.out(*t[k].shape, dtype=gtype) for k in ("gate", "post_w", "post_b", "pre_w", "pre_b")}
        dn.dn_norm_backward(t["x"], t["b"], t["gate"], t["post_w"], t["post_b"], t["pre_w"], dx_out, dnorm if pre else None, dx, db,
                            out["gate"], out["post_w"], out["post_b"], out["pre_w"], out["pre_b"], post=post, pre=pre, scale=0.5,
                            rows_per_gate=per)
        w = {k: v.double().requires_grad_() for k, v in t.items() if v is not None}
        want = {"x": dx_out.double()}
        if pre:
            n = norm64(w["x"], pre, w.get("pre_w"), w.get("pre_b"))
            names = [k for k in ("x", "pre_w", "pre_b") if k in w]
            got = dict(zip(names, torch.autograd.grad(n, [w[k] for k in names], dnorm.double())))
            want.update(got, x=got["x"] + dx_out.double())
        names = [k for k in ("b", "gate", "post_w", "post_b") if k in w]
        want.update(zip(names, torch.autograd.grad(step64(w, post, per, 0.5), [w[k] for k in names], want["x"])))
        what = "%s %s %d %d d" % (kind, shape, post, pre)
        # rows' derivatives are differences of their parts: a few more roundings of fp32 than a plain sum has
        fine = 4 * tolerance(torch.float32, d + rows)
        close(dx, want["x"], fine + (0 if kind == "f32" else tolerance(dtype, d)), what + "x")
        # the derivative of a norm is what is left of two parts of its size: all but d - 1 (layer: d - 2) of d dimensions
        if not (post and d <= 2):
            close(db, want["b"], fine + (0 if kind == "f32" else tolerance(dtype, d)), what + "b")
        for k, v in out.items():
            if v is not None:
                close(v, want[k], fine + (0 if v.dtype == torch.float32 else tolerance(dtype, rows)), what + k)


def test_pieces_by_themselves_and_in_place():
    announce("norm pieces")
    make, t = tensors("bf16", (40, 264, 40), RMS, RMS, False, True)
    n, both, n2 = make.out(40, 264), make.out(40, 264), make.out(40, 264)
    # the norm alone, and a step whose block is zero
    dn.dn_norm_forward(t["x"], None, None, None, None, t["pre_w"], None, None, n)
    zero = torch.zeros_like(t["x"])
    dn.dn_norm_forward(t["x"], zero, None, t["post_w"], None, t["pre_w"], None, both, n2)
    assert torch.equal(n, n2) and torch.equal(both, t["x"])
    # x_out over x, n_out over b
    dn.dn_norm_forward(t["x"], t["b"], None, t["post_w"], None, t["pre_w"], None, both, n2)
    dn.dn_norm_forward(t["x"], t["b"], None, t["post_w"], None, t["pre_w"], None, t["x"], t["b"])
    assert torch.equal(both, t["x"]) and torch.equal(n2, t["b"])
    # backward: dx over dn, db over b; no derivative from elsewhere
    g, dx, db = make(40, 264), make.out(40, 264), make.out(40, 264)
    w = make.out(264)
    args = lambda *o: dn.dn_norm_backward(both, t["b"], None, t["post_w"], None, t["pre_w"], None, *o, None, w, None, None, None)
    args(g, dx, db)
    first = w.clone()
    args(g, g, t["b"])
    assert torch.equal(g, dx) and torch.equal(t["b"], db) and torch.equal(first, w)


def test_rows_of_zeros_constants_and_what_is_not_finite():
    announce("norm zeros")
    for kind, dtype in TYPES.items():
        x = Make(dtype, 3)(6, 300)
        x[0] = 0
        x[1] = 3
        x[2, 5] = float("nan")
        x[3, 7] = float("inf")
        x[4] = torch.finfo(dtype).max / 1e3 if dtype == torch.float16 else 1e15
        n = torch.full_like(x, float("nan"))
        for how in (RMS, LAYER):
            dn.dn_norm_forward(x, None, None, None, None, None, None, None, n, pre=how)
            assert (n[0] == 0).all() and torch.isnan(n[2]).all()
            assert torch.isfinite(n[[0, 1, 4, 5]]).all(), (kind, how)
            assert (n[1] == 0).all() if how == LAYER else ((n[1] - 1).abs() < 1e-2).all()


def test_gradient_of_a_large_mean():
    """Layer norm of rows whose mean is a thousand times their deviation: the centred squares are formed from centred numbers."""
    announce("norm large mean")
    make = Make(torch.float32, 6)
    x = make(16, 1000, mean=1000.0)
    n = make.out(16, 1000)
    dn.dn_norm_forward(x, None, None, None, None, None, None, None, n, pre=LAYER)
    # a row's sum is 10^6, where fp32 is spaced 2^-4: some three roundings of up to 2^-5 in it, a thousandth of that in the mean
    close(n, norm64(x.double(), LAYER, None, None), 2e-4, "n")


def test_refusals_of_the_binding():
    x = torch.zeros(4, 8, device=DEV)
    n = torch.zeros(4, 8, device=DEV)
    for call in (lambda: dn.dn_norm_forward(x, None, None, None, None, None, None, None, n.half()),
                 lambda: dn.dn_norm_forward(x, x, x[:2], None, None, None, None, x, n),
                 lambda: dn.dn_norm_forward(x, None, None, None, None, x[0, :7], None, None, n),
                 lambda: dn.dn_norm_forward(x[:, :7], None, None, None, None, None, None, None, n)):
        with pytest.raises(TypeError):
            call()
    for kw in ({"pre": 3}, {"post": -1}, {"eps": -1.0}, {"scale": float("nan")}):
        with pytest.raises(dn.DnError):
            dn.dn_norm_forward(x, None, None, None, None, None, None, None, n, **kw)
    with pytest.raises(dn.DnError):   # a shift belongs to a layer norm
        dn.dn_norm_forward(x, None, None, None, None, None, x[0], None, n, pre=RMS)
