"""The calls of a block of experts again and again on the same tensors: what they read stays as it was, and every pass is right."""
import pytest
import torch

import experts_util as ex
from ffn_util import DEV, TYPES, close, tolerance
from paper_2001_04206_amd import dn
from test_gpu_experts import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("rows,experts,k,d,f", [(1, 4, 2, 64, 40), (3, 8, 4, 65, 33), (37, 5, 2, 101, 55), (700, 4, 2, 320, 192), (1301, 8, 2, 136, 200)])
def test_every_pass_is_the_first(name, rows, experts, k, d, f):
    c = Case(TYPES[name], rows, experts, k, d, f, none=0.1, seed=rows)
    read = {"X": c.X, "R": c.R, "Wg": c.Wg, "Wu": c.Wu, "Wd": c.Wd, "dY": c.dY, "weight": c.weight, "starts": c.starts, "order": c.order, "place": c.place}
    before = {n: t.clone() for n, t in read.items()}
    want = ex.forward64(c.X, c.Wg, c.Wu, c.Wd, c.weight, c.expert, c.R, c.act)[0]
    first = None
    for _ in range(3):
        Y, GU = c.forward()
        close(Y, want, tolerance(c.dtype, d + f, 3), "Y")
        kept = torch.where(GU.isnan(), torch.zeros_like(GU), GU)
        g = c.backward(kept)
        c.check_backward(g, kept)
        for n, t in read.items():
            assert torch.equal(t, before[n]), n
        results = [Y, kept, *g.values()]
        first = first or results
        assert all(torch.equal(a, b) for a, b in zip(first, results))


def test_routing_and_clipping():
    L = torch.randn(300, 64, generator=torch.Generator().manual_seed(1)).to(DEV)
    bias, grads = torch.linspace(-0.1, 0.1, 64, device=DEV), [torch.randn(n, device=DEV) for n in (7, 9000)]
    expert, weight, dL, norm = torch.empty(300, 4, dtype=torch.int32, device=DEV), torch.empty(300, 4, device=DEV), torch.empty_like(L), torch.empty(1, device=DEV)
    outs = [torch.empty_like(g) for g in grads]
    before = [t.clone() for t in (L, bias, *grads)]
    first = None
    for _ in range(3):
        dn.dn_route_forward(L, bias, expert, weight, score=dn.DN_SCORE_SIGMOID, groups=8, top_groups=3, group_best=2)
        dn.dn_route_backward(L, expert, weight, dL, score=dn.DN_SCORE_SIGMOID)
        dn.dn_clip(grads, 0.5, norm, outs)
        assert all(torch.equal(a, b) for a, b in zip((L, bias, *grads), before))
        results = [t.clone() for t in (expert, weight, dL, norm, *outs)]
        first = first or results
        assert all(torch.equal(a, b) for a, b in zip(first, results))
