"""Routing of logits whose scores run together: beyond 37 a sigmoid is 1 in 64 bits, some 745 below the row's highest a softmax is 0, and below -690
a sigmoid comes near the smallest numbers of 64 bits."""
import math

import pytest
import torch

from ffn_util import DEV, TYPES
from paper_2001_04206_amd import dn
from test_gpu_route import SIGMOID, SOFTMAX, check, run

pytestmark = pytest.mark.gpu

# experts, groups, top groups: groups of whole lanes and of parts of them, at every width of a kernel
SHAPES = [(8, 2, 1), (8, 2, 2), (64, 8, 3), (63, 7, 4), (128, 4, 2), (120, 5, 3), (256, 8, 4), (252, 7, 3), (512, 16, 5), (500, 5, 2), (1024, 8, 4), (1000, 10, 9)]


def test_the_order_of_saturated_logits():
    """Without a bias the order is the logits', also among groups that are chosen by sums of two scores."""
    L = torch.tensor([[40.0, 50.0, 60.0, 45.0, 1.0, 1.0, 1.0, 1.0]], device=DEV)
    for dtype in TYPES.values():
        expert = run(L.to(dtype), None, 2, SIGMOID, groups=2, top_groups=1, group_best=2)[0]
        assert expert.tolist() == [[2, 1]]
    L = torch.tensor([[9000.0, 1000.0, 3000.0, 2000.0, 100.0, 100.0, 100.0, 100.0]], device=DEV)
    expert = run(L.half(), None, 4, SOFTMAX, groups=2, top_groups=1, group_best=2)[0]
    assert expert.tolist() == [[0, 2, 3, 1]]


def far(rows, experts, groups, dtype, seed, low, high):
    """Groups of logits between `low` and `high`, two of them at least from 40 on so that such groups tie, and of small ones."""
    g = torch.Generator().manual_seed(seed)
    each = experts // groups
    L = (low + (high - low) * torch.rand(rows, groups, each, generator=g)).view(rows, groups, each)
    L[:, :, :2] = 40 + (high - 40) * torch.rand(rows, groups, min(2, each), generator=g)
    L = L.gather(2, torch.rand(rows, groups, each, generator=g).argsort(2))
    small = torch.rand(rows, groups, 1, generator=g) < 0.4
    return torch.where(small, torch.randn(rows, groups, each, generator=g), L).view(rows, experts).to(dtype).to(DEV)


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("experts,groups,top", SHAPES)
def test_saturated_scores(name, experts, groups, top):
    """Sigmoids that are one number in 64 bits, some of their logits equal (ties to the lowest): one launch with the lists, and rows by themselves."""
    k = min(8, top * (experts // groups))
    for rows in (5, 40):
        L = far(rows, experts, groups, TYPES[name], rows + experts, 30, 100)
        for renorm in (True, False):
            check(L, None, k, SIGMOID, groups, top, 2, renorm)


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("experts,groups,top", SHAPES)
def test_scores_that_vanish(name, experts, groups, top):
    """Softmax scores of logits thousands apart: all but the highest are 0, so that all groups but its own tie."""
    k = min(8, top * (experts // groups))
    g = torch.Generator().manual_seed(experts)
    for rows in (5, 40):
        steps = torch.stack([torch.randperm(experts, generator=g) for _ in range(rows)])
        L = ((steps - experts // 2).float() * (60000.0 / experts)).to(TYPES[name])
        L[torch.arange(rows), steps.argmax(1)] = 60000.0
        for renorm in (True, False):
            check(L.to(DEV), None, k, SOFTMAX, groups, top, 2, renorm)


def test_not_a_number_among_groups():
    """NaN is the highest logit; the others follow by their own."""
    for experts, groups in ((64, 8), (63, 7), (256, 8), (1000, 10)):
        L = far(6, experts, groups, torch.float32, 3, 30, 100)
        at = torch.tensor([0, 1, experts // 2, experts - 1, 7, 8])
        L[torch.arange(6), at] = math.nan
        expert, weight = run(L, None, 4, SIGMOID, groups=groups, top_groups=2, group_best=2)[:2]
        assert torch.equal(expert[:, 0].cpu().long(), at) and weight.isnan().all()
        rest = L.gather(1, expert[:, 1:].long())
        assert (rest[:, :-1] >= rest[:, 1:]).all() and len(set(expert[0].tolist())) == 4


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("experts,groups,top", [(12, 1, 1), (100, 1, 1), (256, 8, 3), (1000, 10, 4)])
def test_scores_near_the_smallest_numbers(name, experts, groups, top):
    """Sigmoids of logits from -708 to -680 and a bias of zeros: their scores, 1e-296 to 3e-308, are told apart in 64 bits."""
    g = torch.Generator().manual_seed(experts)
    L = (-708 + 28 * torch.rand(20, experts, generator=g)).to(TYPES[name]).to(DEV)
    k = min(8, top * (experts // groups))
    expert, *_ = run(L, torch.zeros(experts, device=DEV), k, SIGMOID, groups=groups, top_groups=top, group_best=1)
    chosen = L.float().gather(1, expert.long())
    assert (chosen[:, :-1] >= chosen[:, 1:]).all()
    if groups == 1:
        assert torch.equal(chosen, L.float().sort(1, descending=True)[0][:, :k])
    check(L, torch.zeros(experts, device=DEV), k, SIGMOID, groups, top, 1, renorm=True)
