"""The calls of a block of experts as they are used together: a classifier's step with them against 64 bits, on streams, in graphs, inside
larger buffers, and at sizes beyond 2^32 bytes."""
import ctypes as C
import math
import os
import sys

import numpy as np
import pytest
import torch

import experts_util as ex
from ffn_util import ACTS, DEV, TYPES, UNIT, Make, close, f64, tolerance
from paper_2001_04206_amd import dn, synth
from parity_util import announce
from test_gpu_experts import Case

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def rms(v, w):
    return v / (v.square().mean(1, keepdim=True) + 1e-5).sqrt() * w


def forward64(net, p, X, choices):
    """n_L with the experts that the run chose."""
    x = torch.nn.functional.gelu(X @ p["We"].t() + p["be"])
    n = rms(x, p["pre0"])
    for i in range(net.blocks):
        expert = choices[i].cpu().long()
        weight = torch.softmax((n @ p["Wr%d" % i].t()).gather(1, expert), 1)
        b = torch.zeros_like(x)
        for e in range(net.experts):
            t, j = (expert == e).nonzero(as_tuple=True)
            h = torch.nn.functional.silu(n[t] @ p["Wg%d" % i][e].t()) * (n[t] @ p["Wu%d" % i][e].t())
            b = b.index_add(0, t, (h @ p["Wd%d" % i][e].t()) * weight[t, j][:, None])
        x = x + p["gate%d" % i] * rms(b, p["post%d" % i])
        n = rms(x, p["pre%d" % (i + 1)])
    return n


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,width,hidden,experts,choose", [(1, 40, 72, 4, 2), (37, 65, 131, 5, 3), (300, 128, 264, 8, 2)])
def test_gradients_of_a_step(kind, rows, width, hidden, experts, choose):
    """Every value on the way is rounded to the type some 30 times through two blocks and back, each adding a unit roundoff, so sqrt(30)
    of them in 2-norm; a factor of 4 for what the norms and gates amplify, and of 2 for the router, whose gradients are differences
    of the choices' derivatives.  fp32: 2^-24 sqrt(terms) of sums of up to 300 terms at each of them."""
    from residual_blocks import Blocks
    announce("residual blocks of experts' gradients %s %s" % (kind, (rows, width, hidden)))
    dtype = TYPES[kind]
    net = Blocks(50, width, hidden, 5, 2, rows, dtype, experts=experts, choose=choose)
    g = torch.Generator().manual_seed(3)
    X = torch.randn(rows, 50, generator=g).to(dtype).float().cuda()
    top = torch.randn(rows, width, generator=g).to(dtype).cuda()
    n = net.forward(X, 0)
    choices = [net.kept[i + 1][4][1].clone() for i in range(2)]
    net.backward(top, 0)
    p = {k: v.double().cpu().requires_grad_() for k, v in net.w.items()}
    want = forward64(net, p, X.double().cpu(), choices)
    want.backward(top.double().cpu())
    tol = 8 * 30 ** 0.5 * (UNIT[dtype] if dtype != torch.float32 else 2.0 ** -24 * 300 ** 0.5)
    for k, got, ref in [("n", n, want)] + [(k, net.grads[k], v.grad) for k, v in p.items()]:
        off = (got.double().cpu() - ref.detach()).norm().item() / max(ref.detach().norm().item(), 1e-30)
        assert off <= tol, "%s: %.3g of %.3g" % (k, off, tol)
    # all gradients bounded together
    before = {k: v.clone() for k, v in net.grads.items()}
    whole = math.sqrt(sum((v.double() ** 2).sum().item() for v in before.values()))
    dn.dn_clip(list(net.grads.values()), 0.5 * whole, net.norm)
    assert abs(net.norm.item() - whole) <= 1.01 * 2.0 ** -24 * whole
    for k, v in before.items():
        assert ((net.grads[k].double() - 0.5 * v.double()).abs() <= 2.0 ** -22 * v.double().abs() + 2.0 ** -140).all()
    net.head.close()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_training_runs(kind):
    from residual_blocks import Blocks
    announce("residual blocks of experts' training %s" % kind)
    rows, batches = 128, 4
    task = synth.learnable((32, 8, 6), n_samples=batches * rows, batch=rows)
    X, labels = torch.from_numpy(task.X).cuda(), torch.from_numpy(task.labels).cuda()
    net = Blocks(32, 96, 80, 6, 2, rows, TYPES[kind], drop=0.1, experts=6, choose=2, clip=1.0)
    loss = torch.zeros(1, device="cuda")
    for step in range(12):
        at = step % batches * rows
        net.step(X[at:at + rows], labels[at:at + rows], step, 0.05, 0.9, loss)
        assert math.isfinite(loss.item()) and 0 < net.norm.item() < math.inf
        after = math.sqrt(sum((v.double() ** 2).sum().item() for v in net.grads.values()))
        assert after <= min(net.norm.item(), rows) * (1 + 2.0 ** -20)
    together = net.answer(X[:8])
    assert together.shape == (8, 6) and ((together.sum(1) - 1).abs() < 1e-5).all()
    net.head.close()


class Flow:
    """Routing, the block forward and backward, the router's gradient and the norm of all of it, in buffers of their own."""

    def __init__(self, dtype, rows, experts=8, k=2, d=64, f=72, shared=None):
        make = Make(dtype, rows)
        self.L, self.X, self.dY = make(rows, experts), make(rows, d), make(rows, d)
        self.bias = torch.linspace(-0.02, 0.02, experts, device=DEV)
        self.W = [make(experts, f, d, std=d ** -0.5), make(experts, f, d, std=d ** -0.5), make(experts, d, f, std=f ** -0.5)]
        whole = lambda *s: torch.full(s, -7, dtype=torch.int32, device=DEV)
        real = lambda *s: make.out(*s, dtype=torch.float32)
        self.out = {"expert": whole(rows, k), "weight": real(rows, k), "starts": whole(experts + 1), "order": whole(rows * k), "place": whole(rows * k),
                    "Y": make.out(rows, d), "GU": make.out(rows * k, 2 * f), "dX": make.out(rows, d), "dWg": make.out(experts, f, d),
                    "dWu": make.out(experts, f, d), "dWd": make.out(experts, d, f), "dweight": real(rows, k), "dL": make.out(rows, experts),
                    "norm": real(1), "c0": real(experts, f, d), "c1": real(rows, experts)}
        self.spaces = shared or [torch.empty(n, dtype=torch.uint8, device=DEV) for n in (1 << 20, 64 << 20, 64 << 20, 1 << 20)]

    def run(self):
        o, s = self.out, self.spaces
        lists = (o["weight"], o["starts"], o["order"], o["place"])
        dn.dn_route_forward(self.L, self.bias, o["expert"], *lists, score=dn.DN_SCORE_SIGMOID, groups=4, top_groups=2, group_best=2, workspace=s[0])
        dn.dn_experts_forward(self.X, *self.W, *lists, self.X, o["Y"], o["GU"], workspace=s[1])
        dn.dn_experts_backward(self.X, *self.W, *lists, o["GU"], self.dY, o["dX"], o["dWg"], o["dWu"], o["dWd"], o["dweight"], workspace=s[2])
        dn.dn_route_backward(self.L, o["expert"], o["dweight"], o["dL"], score=dn.DN_SCORE_SIGMOID)
        dn.dn_clip([o["dWg"], o["dL"]], 0.5, o["norm"], [o["c0"], o["c1"]], workspace=s[3])

    def take(self):
        torch.cuda.synchronize()
        return {k: v.clone() for k, v in self.out.items()}

    def spoil(self):
        for v in self.out.values():
            v.fill_(-7 if v.dtype == torch.int32 else math.nan)

    def same(self, want):
        torch.cuda.synchronize()
        for k, v in self.out.items():
            assert torch.equal(v, want[k]), k


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows", [1, 6, 40, 1500])
def test_streams_and_graphs(kind, rows):
    """On a side stream, two at once on two streams, and captured: two graphs that share their workspaces, replayed by turns with the
    program's own work between, every replay with other inputs against the eager result."""
    announce("experts on streams and in graphs %s %d" % (kind, rows))
    flow = Flow(TYPES[kind], rows)
    flow.run()
    want = flow.take()
    assert not any(v.isnan().any() for v in want.values() if v.is_floating_point())
    flow.spoil()
    other = Flow(TYPES[kind], rows)
    side, second = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(side):
            flow.run()
        with torch.cuda.stream(second):
            other.run()
    flow.same(want)
    other.same(want)
    twin = Flow(TYPES[kind], rows, shared=flow.spaces)
    graphs = []
    for f in (flow, twin):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            f.run()
        graphs.append(graph)
    for n in range(3):
        for f, graph in zip((flow, twin), graphs):
            for t in (f.X, f.L, f.dY):
                t.mul_(-1)
            f.run()
            want = f.take()
            f.spoil()
            graph.replay()
            f.same(want)


def test_nothing_outside_is_written():
    """Results inside larger buffers and workspaces of exactly the bytes asked for: what lies around them stays."""
    announce("experts' guards")
    for kind, rows, experts, k, d, f, none in (("bf16", 70, 5, 2, 65, 131, 0.2), ("f32", 129, 3, 2, 40, 72, 0.0), ("f16", 3, 9, 3, 33, 17, 0.3),
                                               ("bf16", 900, 2, 2, 264, 200, 0.1), ("f32", 2, 4, 2, 64, 24, 0.0)):
        c = Case(TYPES[kind], rows, experts, k, d, f, none=none, pad=3)

        def guarded(*shape, dtype=c.dtype):
            n = int(np.prod(shape))
            flat = torch.full((n + 256,), 7, dtype=dtype, device=DEV)
            return flat, flat[128:128 + n].view(*shape)

        bufs = {"Y": guarded(rows, d), "GU": guarded(rows * k, 2 * f), "dX": guarded(rows, d), "Wg": guarded(experts, f, d), "Wu": guarded(experts, f, d),
                "Wd": guarded(experts, d, f), "dw": guarded(rows, k, dtype=torch.float32), "expert": guarded(rows, k, dtype=torch.int32),
                "weight": guarded(rows, k, dtype=torch.float32), "starts": guarded(experts + 1, dtype=torch.int32), "order": guarded(rows * k, dtype=torch.int32),
                "place": guarded(rows * k, dtype=torch.int32), "dL": guarded(rows, experts), "norm": guarded(1, dtype=torch.float32)}
        v = {n: b[1] for n, b in bufs.items()}
        lib = dn.lib()
        kind_of = dn._type_of(c.X, "X")
        desc = dn.ExpertsDesc(kind_of, kind_of, dn.DN_ACT_SILU, rows, d, f, experts, k, d + 3, d + 3, 0, 1.0)
        back = dn.ExpertsDesc(kind_of, kind_of, dn.DN_ACT_SILU, rows, d, f, experts, k, d + 3, 0, d + 3, 1.0)
        spans = (dn.Span * 1)(dn.Span(c.Wg.data_ptr(), v["Wg"].data_ptr(), c.Wg.numel(), kind_of, kind_of))
        need = [lib.dn_experts_forward_workspace_bytes(C.addressof(desc)), lib.dn_experts_backward_workspace_bytes(C.addressof(back)),
                lib.dn_route_workspace_bytes(rows, experts, k), lib.dn_clip_workspace_bytes(C.addressof(spans), 1)]
        spaces = [torch.full((n + 512,), 99, dtype=torch.uint8, device=DEV) for n in need]
        ws = [s[:n] for s, n in zip(spaces, need)]
        L = c.make(rows, experts)
        dn.dn_route_forward(L, None, v["expert"], v["weight"], v["starts"], v["order"], v["place"], workspace=ws[2] if need[2] else None)
        dn.dn_route_backward(L, v["expert"], v["weight"], v["dL"])
        dn.dn_experts_forward(c.X, c.Wg, c.Wu, c.Wd, *c.lists, c.R, v["Y"], v["GU"], workspace=ws[0])
        dn.dn_experts_backward(c.X, c.Wg, c.Wu, c.Wd, *c.lists, v["GU"], c.dY, v["dX"], v["Wg"], v["Wu"], v["Wd"], v["dw"], workspace=ws[1])
        dn.dn_clip([c.Wg], 1.0, v["norm"], [v["Wg"]], workspace=ws[3])
        torch.cuda.synchronize()
        for n, (flat, _) in bufs.items():
            assert (flat[:128] == 7).all() and (flat[-128:] == 7).all(), (kind, n)
        for s, n in zip(spaces, need):
            assert (s[n:] == 99).all(), kind


def test_tensors_beyond_four_gigabytes():
    """Matrices whose later experts, and kept rows whose later places, lie past 2^32 bytes: the rows that meet them, against 64 bits."""
    announce("experts' long tensors")
    dtype, experts, d, f = torch.bfloat16, 96, 2048, 16384     # 6.4 GB a matrix
    g = torch.Generator(device=DEV).manual_seed(1)
    W = [torch.empty(s, dtype=dtype, device=DEV).normal_(0, std, generator=g) for s, std in
         (((experts, f, d), d ** -0.5), ((experts, f, d), d ** -0.5), ((experts, d, f), f ** -0.5))]
    for rows in (3, 50):
        expert = torch.tensor([[95, 3], [64, 94], [90, 0]], dtype=torch.int32).repeat(17, 1)[:rows].to(DEV)
        weight = torch.full((rows, 2), 0.5, device=DEV)
        starts, order, place = (torch.empty(n, dtype=torch.int32, device=DEV) for n in (experts + 1, 2 * rows, 2 * rows))
        dn.dn_route_lists(expert, starts, order, place)
        X = torch.empty(rows, d, dtype=dtype, device=DEV).normal_(0, 1, generator=g)
        Y, GU = torch.empty_like(X), torch.empty(2 * rows, 2 * f, dtype=dtype, device=DEV)
        dn.dn_experts_forward(X, *W, weight, starts, order, place, None, Y, GU)
        for t in range(3):
            want = torch.zeros(d, dtype=torch.float64)
            for j in range(2):
                e = int(expert[t, j])
                x = X[t].double()
                h = f64((W[0][e].double() @ x).cpu(), "silu") * (W[1][e].double() @ x).cpu()
                want += 0.5 * (W[2][e].double() @ h.to(DEV)).cpu()
            close(Y[t], want, tolerance(dtype, d + f, 3), "Y of row %d" % t)
    del W, GU
    torch.cuda.empty_cache()
    # kept rows past 2^32 bytes, and the matrices' gradients over them
    rows, experts, k, d, f = 60000, 4, 4, 32, 4800               # GU 4.6 GB, H 2.3
    c = Case.__new__(Case)
    make = Make(dtype, 3)
    expert = (torch.arange(4)[None, :] + torch.arange(rows)[:, None]).remainder(4).int().to(DEV)
    weight = torch.rand(rows, k, generator=torch.Generator().manual_seed(2)).to(DEV)
    starts, order, place = (torch.empty(n, dtype=torch.int32, device=DEV) for n in (experts + 1, rows * k, rows * k))
    dn.dn_route_lists(expert, starts, order, place)
    X, dY, Y, dX = make(rows, d), make(rows, d), make.out(rows, d), make.out(rows, d)
    W = [make(experts, f, d, std=d ** -0.5), make(experts, f, d, std=d ** -0.5), make(experts, d, f, std=f ** -0.5)]
    GU, dW, dweight = make.out(rows * k, 2 * f), [make.out(*w.shape) for w in W], torch.empty(rows, k, device=DEV)
    dn.dn_experts_forward(X, *W, weight, starts, order, place, None, Y, GU)
    dn.dn_experts_backward(X, *W, weight, starts, order, place, GU, dY, dX, *dW, dweight)
    at = torch.tensor([0, 1, 29999, 59998, 59999])
    pick = lambda t: t[at.to(DEV)]
    want, G, U = ex.forward64(pick(X), *W, pick(weight), pick(expert), None, "silu")
    close(pick(Y), want, tolerance(dtype, d + f, 3), "Y")
    rows_of = pick(place.view(rows, k)).long().cpu()
    kept = GU[rows_of.to(DEV).view(-1)].view(5, k, 2 * f).cpu().double()
    close(kept[..., :f], G, tolerance(dtype, d), "G")
    r = ex.backward64(pick(X), *W, pick(weight), pick(expert), kept[..., :f], kept[..., f:], pick(dY), "silu")
    close(pick(dX), r[0], tolerance(dtype, d + 2 * f, 3), "dX")
    close(pick(dweight), r[4], 2.0 ** -24 * (d ** 0.5 + f ** 0.5 + 16) + 3e-7, "dweight")
    # the last expert's Wd, from the kept rows, in 64 bits on the device
    a, b = int(starts[3]), int(starts[4])
    want = torch.zeros(d, f, dtype=torch.float64, device=DEV)
    for p in range(a, b, 10000):
        q = order[p:min(p + 10000, b)].long()
        gu = GU[p:p + len(q)].double()
        want += (dY[q // k].double() * weight.view(-1)[q].double()[:, None]).T @ (torch.nn.functional.silu(gu[:, :f]) * gu[:, f:])
    close(dW[2][3], want, tolerance(dtype, rows + d, 2), "dWd")


def test_refusals_of_the_binding():
    x, w = torch.zeros(4, 8, device=DEV), torch.zeros(3, 16, 8, device=DEV)
    wd, weight = torch.zeros(3, 8, 16, device=DEV), torch.zeros(4, 2, device=DEV)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)
    starts, order, place, y, gu = i32(4), i32(8), i32(8), torch.zeros(4, 8, device=DEV), torch.zeros(8, 32, device=DEV)

    def forward(**kw):
        a = dict(X=x, Wg=w, Wu=w, Wd=wd, weight=weight, starts=starts, order=order, place=place, R=None, Y=y, GU=gu)
        a.update(kw)
        return lambda: dn.dn_experts_forward(**a)

    L, expert = torch.zeros(4, 3, device=DEV), i32(4, 2)
    norm = torch.zeros(1, device=DEV)
    for call in (forward(X=x.cpu()), forward(Wg=w[0]), forward(Wu=w[:2]), forward(Wd=w), forward(weight=weight[:3]), forward(weight=weight.half()),
                 forward(starts=starts[:3]), forward(order=order.long()), forward(place=place[:4]), forward(Y=y.half()), forward(GU=gu[:4]),
                 forward(X=x.double()), forward(workspace=x),
                 lambda: dn.dn_route_forward(L.cpu(), None, expert, weight), lambda: dn.dn_route_forward(L, None, expert.long(), weight),
                 lambda: dn.dn_route_forward(L, norm, expert, weight), lambda: dn.dn_route_forward(L, None, expert, weight[:3]),
                 lambda: dn.dn_route_forward(L[0], None, expert, weight), lambda: dn.dn_route_forward(L, None, expert[:3], weight),
                 lambda: dn.dn_route_lists(expert, starts, order[:3], place), lambda: dn.dn_route_lists(expert.cpu(), starts, order, place),
                 lambda: dn.dn_route_backward(L, expert, weight, L.half()), lambda: dn.dn_route_backward(L, expert, weight[:1], L),
                 lambda: dn.dn_clip([x.double()], 1.0, norm), lambda: dn.dn_clip([x.cpu()], 1.0, norm), lambda: dn.dn_clip([x.t()], 1.0, norm),
                 lambda: dn.dn_clip([x], 1.0, norm, []), lambda: dn.dn_clip([x], 1.0, norm, [y[:2]]), lambda: dn.dn_clip([x], 1.0, norm.half()),
                 lambda: dn.dn_clip([x], 1.0, y)):
        with pytest.raises(TypeError):
            call()
    for call in (forward(act=9), forward(act=dn.DN_ACT_SOFTMAX), lambda: dn.dn_route_forward(L, None, expert, weight, starts, None, None),
                 lambda: dn.dn_route_forward(L, None, expert, weight, groups=2), lambda: dn.dn_route_forward(L, None, expert, weight, score=5),
                 lambda: dn.dn_route_forward(L, None, expert, weight, scale=math.nan), lambda: dn.dn_clip([x], -1.0, norm),
                 lambda: dn.dn_clip([x], 1.0, norm, [x.half()]), lambda: dn.dn_clip([x], math.nan, norm)):
        with pytest.raises(dn.DnError):
            call()
