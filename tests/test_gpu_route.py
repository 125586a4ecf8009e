"""Routing to experts on the GPU: choices, weights, lists and the logits' gradient against 64 bits."""
import math

import pytest
import torch

import experts_util as ex
from ffn_util import DEV, TYPES, UNIT
from paper_2001_04206_amd import dn

pytestmark = pytest.mark.gpu
SOFTMAX, SIGMOID = dn.DN_SCORE_SOFTMAX, dn.DN_SCORE_SIGMOID
INF = math.inf

# fp32 weights: an exponential, a sum of at most 1024 terms, a division and a product, each within 2 units of 2^-24
WEIGHT = 16 * 2.0 ** -24


def logits(rows, experts, dtype, seed, pad=0, std=1.5):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(rows, experts + pad, generator=g) * std).to(dtype).to(DEV)[:, :experts]


def run(L, bias, k, score, with_lists=True, **kw):
    rows, experts = L.shape
    i32 = lambda *s: torch.full(s, 12345, dtype=torch.int32, device=DEV)
    expert, weight = i32(rows, k), torch.full((rows, k), math.nan, device=DEV)
    starts, order, place = (i32(experts + 1), i32(rows * k), i32(rows * k)) if with_lists else (None,) * 3
    dn.dn_route_forward(L, bias, expert, weight, starts, order, place, score=score, **kw)
    return expert, weight, starts, order, place


def check(L, bias, k, score, groups=1, top_groups=1, best=1, renorm=True, scale=1.0):
    expert, weight, *got = run(L, bias, k, score, groups=groups, top_groups=top_groups, group_best=best, renorm=renorm, scale=scale)
    e, w = ex.route64(L, bias, k, score, groups, top_groups, best, renorm, scale)
    assert torch.equal(expert.cpu(), e)
    off = (weight.cpu().double() - w).abs()
    assert (off <= WEIGHT * w.abs() + 2.0 ** -140).all(), (off / w.abs().clamp(min=1e-30)).max()
    for name, a, b in zip(("starts", "order", "place"), got, ex.lists(expert, L.shape[1])):
        assert torch.equal(a.cpu(), b), name
    return expert, weight


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("experts,k", [(1, 1), (2, 2), (7, 3), (63, 8), (64, 64 // 2), (65, 5), (128, 8), (129, 9), (256, 8), (257, 1), (512, 4),
                                       (513, 32), (1000, 10), (1024, 8)])
def test_choices(name, experts, k):
    """Both scores, with and without renormalised weights, at both sides of every width of a kernel; rows that do not fill a workgroup."""
    for i, (rows, score, renorm) in enumerate([(1, SOFTMAX, True), (3, SIGMOID, True), (70, SOFTMAX, False), (33, SIGMOID, False)]):
        check(logits(rows, experts, TYPES[name], experts + i, pad=(0, 3)[i % 2]), None, k, score, renorm=renorm, scale=(1.0, 2.5)[i % 2])


@pytest.mark.parametrize("score", [SOFTMAX, SIGMOID])
@pytest.mark.parametrize("groups,top,best,experts,k", [(1, 1, 1, 60, 4), (4, 2, 2, 64, 8), (8, 4, 2, 256, 8), (8, 4, 1, 256, 8), (8, 8, 2, 40, 6),
                                                       (64, 3, 1, 64, 3), (64, 20, 2, 1024, 32), (3, 1, 2, 21, 7), (5, 4, 1, 1000, 10)])
def test_bias_and_groups(score, groups, top, best, experts, k):
    """A bias, and groups that end inside a lane's experts, with and without one."""
    for bias in (True, False):
        L = logits(50, experts, torch.float32, groups + experts)
        b = logits(1, experts, torch.float32, 5, std=0.1)[0].contiguous() if bias else None
        check(L, b, k, score, groups, top, best, renorm=not bias)


def test_ties_go_to_the_lowest():
    for experts, groups, top in ((40, 1, 1), (256, 8, 3), (1024, 4, 2)):
        L = torch.zeros(5, experts, device=DEV)
        L[1] = 1.0
        L[2, ::2] = 1.0
        L[3, experts // 2:] = 1.0
        L[4, -1] = L[4, 0] = 3.0
        for bias in (None, torch.zeros(experts, device=DEV), torch.full((experts,), -2.0, device=DEV)):
            for best in (1, 2):
                check(L, bias, 8, SIGMOID, groups, top, best)
                check(L.half(), bias, 8, SOFTMAX, groups, top, best, renorm=False)


def test_experts_that_cannot_be_had():
    """Rows of padding, rows with fewer experts than choices, groups with one or none, the type's lowest value, experts taken out by the
    bias."""
    for name, dtype in TYPES.items():
        L = logits(9, 24, dtype, 3)
        L[0] = -INF
        L[1, 3:] = -INF
        L[2, :-1] = -INF
        L[3] = torch.finfo(dtype).min
        L[4, 1:] = torch.finfo(dtype).min
        L[5, :6] = -INF                  # a whole group
        L[6, :5] = -INF                  # all but one of a group
        L[7] = -INF
        L[7, 5] = L[7, 23] = 1.0
        out = torch.zeros(24, device=DEV)
        out[10:14] = -INF
        for bias in (None, torch.zeros(24, device=DEV), out):
            for score in (SOFTMAX, SIGMOID):
                for best in (1, 2):
                    for renorm in (True, False):
                        check(L, bias, 6, score, 4, 3, best, renorm)
    expert, weight, starts, order, place = run(torch.full((300, 16), -INF, device=DEV), None, 4, SOFTMAX)
    assert (expert == -1).all() and (weight == 0).all() and (starts == 0).all() and (order == -1).all() and (place == -1).all()


def test_small_scores_keep_their_ratios():
    """Scores that are 0 or all alike in 32 bits: ratios come of the logits."""
    L = torch.tensor([[-200.0, -201.0, -202.0, -203.0], [-90.0, -90.5, -120.0, -89.0], [80.0, 60.0, -80.0, -90.0], [3e4, -3e4, -3e4, -3e4],
                      [1e-30, -1e-30, 0.0, 1e-38]], device=DEV)
    for score in (SOFTMAX, SIGMOID):
        check(L, None, 3, score)
    # without a bias the order is the logits', also where the scores are one number in 64 bits
    expert, *_ = run(torch.tensor([[100.0, 200.0, 300.0, 150.0]], device=DEV), None, 4, SIGMOID)
    assert expert.tolist() == [[2, 1, 3, 0]]


def test_not_a_number():
    """NaN ranks as +inf and shows in the weights; other rows are as they were."""
    L = logits(4, 70, torch.float32, 11)
    clean = [t.clone() for t in run(L, None, 5, SOFTMAX)[:2]]
    L[1, 40] = math.nan
    L[2, 7] = INF
    for score, bias in ((SOFTMAX, None), (SIGMOID, None), (SOFTMAX, torch.zeros(70, device=DEV)), (SIGMOID, torch.zeros(70, device=DEV))):
        expert, weight = run(L, bias, 5, score)[:2]
        if score == SOFTMAX:
            assert weight[1].isnan().all() and weight[2, 0].isnan()
        else:
            assert weight[1, 0].isnan()
        assert bias is not None and score == SOFTMAX or (expert[1, 0] == 40 and expert[2, 0] == 7)
        if score == SOFTMAX and bias is None:
            assert torch.equal(expert[0::3], clean[0][0::3]) and torch.equal(weight[0::3], clean[1][0::3])
        assert ((expert >= 0) & (expert < 70)).all()


@pytest.mark.parametrize("rows,experts,k", [(1, 1, 1), (1, 1024, 32), (1024, 3, 1), (1025, 64, 1), (4000, 60, 4), (20000, 256, 8), (70000, 5, 3),
                                            (50000, 1024, 6)])
def test_lists_of_any_table(rows, experts, k):
    """Chunks of one and several thousand pairs; numbers outside the experts are none; all pairs on one expert."""
    g = torch.Generator().manual_seed(rows)
    tables = [torch.randint(-1, experts + 1, (rows, k), generator=g), torch.full((rows, k), experts - 1),
              torch.where(torch.rand(rows, k, generator=g) < 0.9, -2 ** 31, 2 ** 31 - 1), torch.arange(rows * k).view(rows, k) % experts]
    for table in tables:
        expert = table.int().to(DEV)
        starts, order, place = (torch.full((n,), 12345, dtype=torch.int32, device=DEV) for n in (experts + 1, rows * k, rows * k))
        for _ in range(2):
            dn.dn_route_lists(expert, starts, order, place)
        for name, a, b in zip(("starts", "order", "place"), (starts, order, place), ex.lists(expert, experts)):
            assert torch.equal(a.cpu(), b), name


def gradient64(L, expert, dweight, score, renorm, scale):
    l = L.double().cpu().clone().requires_grad_()
    e = expert.cpu().long()
    has = e >= 0
    if renorm:
        logs = l if score == SOFTMAX else torch.nn.functional.logsigmoid(l)
        w = torch.softmax(logs.gather(1, e.clamp(min=0)).masked_fill(~has, NEVER), 1)
    else:
        w = (torch.softmax(l, 1) if score == SOFTMAX else torch.sigmoid(l)).gather(1, e.clamp(min=0))
    w = torch.where(has, w, torch.zeros_like(w)) * scale
    return torch.autograd.grad(w, l, dweight.double().cpu())[0]


NEVER = -1e300


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("experts,k", [(2, 1), (7, 7), (64, 8), (65, 4), (256, 8), (300, 32), (1024, 10)])
def test_gradient(name, experts, k):
    """Against differentiation in 64 bits: a rounding to the type, and sums of at most 1024 fp32 terms (2^-24 each of the row's largest)."""
    for score in (SOFTMAX, SIGMOID):
        for renorm in (True, False):
            L = logits(37, experts, TYPES[name], experts + k, pad=1)
            expert = run(L, None, k, score, with_lists=False)[0]
            expert[5] = -1
            expert[6, -1] = -1
            dweight = torch.randn(37, k, generator=torch.Generator().manual_seed(k)).to(DEV)
            dL = torch.full((37, experts), math.nan, dtype=TYPES[name], device=DEV)
            dn.dn_route_backward(L, expert, dweight, dL, score=score, renorm=renorm, scale=1.5)
            want = gradient64(L, expert, dweight, score, renorm, 1.5)
            off = (dL.double().cpu() - want).abs()
            row = (dweight.double().cpu().abs().amax(1, keepdim=True) + 1) * 1.5
            small = 2.0 ** -25 if name == "f16" else 0.0     # half a step of its smallest numbers
            assert (off <= UNIT[TYPES[name]] * want.abs() * 1.01 + 40 * 2.0 ** -24 * row + small).all(), (score, renorm, off.max())


def test_gradient_against_differences():
    """dE/dL of E = sum of c w, from the forward call's weights at both sides of each logit of one row.  Steps of 2^-6: the difference is off
    by 2^-12 / 6 of the third derivative (at most about 1) and by the weights' 2^-24 over the step."""
    L = logits(1, 12, torch.float32, 2)
    for score in (SOFTMAX, SIGMOID):
        for renorm in (True, False):
            expert, weight, *_ = run(L, None, 4, score, renorm=renorm)
            c = torch.randn(1, 4, generator=torch.Generator().manual_seed(1)).to(DEV)
            dL = torch.empty_like(L)
            dn.dn_route_backward(L, expert, c, dL, score=score, renorm=renorm)
            step = 2.0 ** -6
            for e in range(12):
                value = []
                for sign in (1, -1):
                    M = L.clone()
                    M[0, e] += sign * step
                    other, w, *_ = run(M, None, 4, score, renorm=renorm)
                    # the same experts, in an order that may have changed
                    assert set(other[0].tolist()) == set(expert[0].tolist())
                    at = {int(i): float(v) for i, v in zip(other[0], w[0])}
                    value.append(sum(float(c[0, j]) * at[int(i)] for j, i in enumerate(expert[0])))
                want = (value[0] - value[1]) / (2 * step)
                assert abs(float(dL[0, e]) - want) <= 2.0 ** -12 * 2 + 8 * 2.0 ** -24 / step


def test_the_same_expert_twice():
    """A table that names an expert twice: both pairs are listed, both weights' gradients count."""
    L = logits(3, 10, torch.float32, 4)
    expert = torch.tensor([[4, 4, 1], [0, 0, 0], [9, 2, 9]], dtype=torch.int32, device=DEV)
    dweight = torch.randn(3, 3, generator=torch.Generator().manual_seed(9)).to(DEV)
    for score in (SOFTMAX, SIGMOID):
        for renorm in (True, False):
            dL = torch.empty_like(L)
            dn.dn_route_backward(L, expert, dweight, dL, score=score, renorm=renorm)
            assert (dL.double().cpu() - gradient64(L, expert, dweight, score, renorm, 1.0)).abs().max() <= 1e-6


def test_many_rows_and_the_same_bits():
    L = logits(5000, 96, torch.bfloat16, 8)
    bias = logits(1, 96, torch.float32, 9, std=0.05)[0].contiguous()
    check(L, bias, 6, SIGMOID, 8, 3, 2, scale=2.5)
    first = [t.clone() for t in run(L, bias, 6, SIGMOID, groups=8, top_groups=3, group_best=2)]
    again = run(L, bias, 6, SIGMOID, groups=8, top_groups=3, group_best=2)
    assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("experts,groups,top", [(24, 1, 1), (24, 4, 2), (64, 8, 3), (100, 5, 2), (128, 4, 3), (256, 8, 4), (300, 1, 1), (512, 16, 3), (1024, 8, 5)])
def test_few_distinct_logits(name, experts, groups, top):
    """Rows of five numbers, both zeros among them, and of -inf: equal ones everywhere, in a lane's experts and between lanes and groups.  (No two sums of
    a score and a bias, nor of two scores, are equal but those of equal numbers.)"""
    values = torch.tensor([0.0, -0.0, 0.5, 1.25, -2.0, -INF])
    k = min(16, top * (experts // groups))
    for seed, weights in enumerate(([1.0] * 6, [1, 1, 0, 0, 0, 1], [1, 1, 0.02, 0.02, 0.1, 9], [0.01, 0, 0, 0, 0, 1])):
        g = torch.Generator().manual_seed(seed)
        L = values[torch.multinomial(torch.tensor(weights).float(), 12 * experts, replacement=True, generator=g)].view(12, experts).to(TYPES[name]).to(DEV)
        steps = torch.tensor([0.0, 0.25, -0.125])[torch.randint(3, (experts,), generator=g)].to(DEV)
        for score in (SOFTMAX, SIGMOID):
            check(L, None, k, score, groups, top, 1 + seed % 2)
            check(L, steps, k, score, groups, top, 1, renorm=False)
            check(L, torch.full((experts,), 0.25, device=DEV), k, score, groups, top, 2)
