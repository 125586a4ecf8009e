"""Blocks of experts, routings and clippings of shapes that between them take every kernel that the library's rules choose for them
(test_experts_kernels.py holds the lists against the rules): each tile with each epilogue, whole and in parts of k, and each kernel for few
rows.  Against the formulas in 64 bits on the device; every tensor that a call writes starts as NaN."""
import math

import pytest
import torch

import experts_util as ex
from ffn_util import DEV, TYPES, tolerance
from paper_2001_04206_amd import dn
from parity_util import announce
from test_gpu_block_kernels import near
from test_gpu_experts import Case
from test_gpu_route import check, logits

pytestmark = pytest.mark.gpu

# rows, experts, k, d, f: of 16-bit types and of fp32
EXPERTS = {
    16: [(1, 1, 1, 16, 629), (1, 3, 1, 1, 32), (8, 8, 1, 1, 16), (16, 1, 1, 17, 2887), (16, 7, 6, 352, 2720), (24, 80, 6, 1320, 221),
         (419, 125, 3, 376, 480), (499, 8, 1, 968, 2040), (1503, 1, 1, 1751, 1), (2680, 17, 7, 136, 4080), (3363, 56, 4, 544, 80),
         (3935, 8, 5, 136, 1800), (5880, 5, 1, 56, 712), (6432, 56, 2, 523, 205)],
    32: [(1, 1, 1, 1, 1), (1, 1, 1, 8, 637), (1, 1, 1, 960, 8), (16, 1, 1, 617, 8), (24, 8, 8, 480, 112), (151, 1, 1, 121, 33),
         (319, 16, 1, 248, 560), (705, 1, 1, 384, 368), (2651, 56, 6, 79, 1291), (7007, 3, 3, 1, 1349)]}
# rows, experts, k, bias, groups
ROUTE = [(3, 60, 4, 0, 1), (8, 64, 8, 1, 4), (5, 100, 3, 0, 4), (2, 128, 8, 1, 1), (7, 200, 5, 0, 1), (1, 256, 8, 1, 8), (8, 300, 2, 0, 4), (3, 512, 8, 1, 4),
         (4, 700, 6, 0, 4), (6, 1024, 32, 1, 4), (9, 30, 2, 0, 1), (70, 64, 8, 1, 8), (90, 128, 8, 0, 4), (33, 90, 4, 1, 1), (40, 256, 8, 0, 1), (60, 200, 9, 1, 8),
         (20, 300, 8, 0, 1), (35, 400, 8, 1, 4), (25, 1000, 8, 0, 8), (12, 1024, 8, 1, 1), (2100, 24, 4, 0, 4)]
# tensors, elements of each
CLIP = [(1, 3), (80, 900), (81, 900), (3, 9000000)]


def of(shapes):
    return [pytest.param(kind, s, id="%s-%s" % (kind, "x".join(map(str, s)))) for kind in TYPES for s in shapes[32 if kind == "f32" else 16]]


@pytest.mark.parametrize("kind,shape", of(EXPERTS))
def test_experts(kind, shape):
    announce("experts' kernels %s %s" % (kind, shape))
    rows, experts, k, d, f = shape
    dtype = TYPES[kind]
    c = Case(dtype, *shape, seed=sum(shape))
    Y, GU = c.forward()
    want, G, U = ex.forward64(c.X, c.Wg, c.Wu, c.Wd, c.weight, c.expert, c.R, c.act, on=DEV)
    near(Y, want, tolerance(dtype, d + f, 3), "Y")
    # by place
    at = c.order.long()
    near(GU[:, :f], G.view(rows * k, f)[at], tolerance(dtype, d), "G")
    near(GU[:, f:], U.view(rows * k, f)[at], tolerance(dtype, d), "U")
    kept = torch.empty(rows * k, 2 * f, dtype=torch.float64, device=DEV)
    kept[at] = GU.double()
    kept = kept.view(rows, k, 2 * f)
    del G, U
    g = c.backward(GU)
    r = ex.backward64(c.X, c.Wg, c.Wu, c.Wd, c.weight, c.expert, kept[..., :f], kept[..., f:], c.dY, c.act, on=DEV)
    near(g["dX"], r[0], tolerance(dtype, d + 2 * f, 3), "dX")
    for n, w in zip(("dWg", "dWu", "dWd"), r[1:4]):
        near(g[n], w, tolerance(dtype, rows * k + d, 2), n)
    near(g["dweight"], r[4], 2.0 ** -24 * (d ** 0.5 + f ** 0.5 + 16) + (0 if dtype == torch.float32 else 3e-7), "dweight")


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("shape", ROUTE, ids=lambda s: "x".join(map(str, s)))
def test_route(kind, shape):
    rows, experts, k, bias, groups = shape
    L = logits(rows, experts, TYPES[kind], sum(shape))
    b = logits(1, experts, torch.float32, 3, std=0.1)[0].contiguous() if bias else None
    for score in (dn.DN_SCORE_SOFTMAX, dn.DN_SCORE_SIGMOID):
        check(L, b, k, score, groups, max(1, groups // 2), 1, renorm=bool(bias))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("shape", CLIP, ids=lambda s: "%dx%d" % s)
def test_clip(kind, shape):
    from test_gpu_clip import check as clipped, norm64, tensors
    before = tensors([shape[1]] * shape[0], [TYPES[kind]], 4)
    n = norm64(before)
    clipped([t.clone() for t in before], 0.3 * n, None, before)
    clipped(before, 0.3 * n, [None] * shape[0], before)


@pytest.mark.parametrize("kind,shape", of(EXPERTS))
def test_rows_apart(kind, shape):
    """NaN in rows of X, dY, G and U reaches no bit of other rows' results, nor of the gradients of experts that these rows did not choose."""
    announce("experts' rows apart %s %s" % (kind, shape))
    rows, experts, k, d, f = shape
    c = Case(TYPES[kind], *shape, seed=sum(shape))
    Y, GU = c.forward()
    clean = c.backward(GU)
    bad = torch.tensor(sorted({0, rows // 2, rows - 1}), device=DEV)
    left = torch.ones(rows, dtype=torch.bool, device=DEV)
    left[bad] = False
    others = torch.ones(experts, dtype=torch.bool, device=DEV)
    others[c.expert[bad].flatten().long()] = False
    c.X[bad], c.dY[bad] = math.nan, math.nan
    GU[c.place.view(rows, k)[bad].flatten().long()] = math.nan
    y, _ = c.forward()
    g = c.backward(GU)
    assert torch.equal(y[left], Y[left]) and y[bad].isnan().all()
    assert torch.equal(g["dX"][left], clean["dX"][left]) and torch.equal(g["dweight"][left], clean["dweight"][left])
    assert g["dX"][bad].isnan().all() and g["dweight"][bad].isnan().all()
    for n in ("dWg", "dWu", "dWd"):
        assert torch.equal(g[n][others], clean[n][others]) and g[n][~others].isnan().all(), n
