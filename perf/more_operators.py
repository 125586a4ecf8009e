"""Timed cases of the block of experts: what a program that trains or serves one calls, and clipping of its gradients.

A case is one of five kinds:
  route      each row's k experts of E from the logits L, their weights, and the lists of rows by expert:
             s = softmax(l) or sigmoid(l), c = s + bias; of `groups` groups of neighbouring experts those `top_groups` stay whose
             best (or best two, added) c are highest; the k highest c of what stays, ties to the lowest index; weights s, divided
             by their sum or not, times a scale.  A logit of -inf takes its expert out; where nothing is left the choice is -1 with weight 0.
             starts [E + 1], order [rows k] (pairs by expert, -1 behind the last), place [rows k] (the other way round, -1 for none)
  route_bwd  the logits' gradient from the weights'
  experts    Y = R + sum over a row's choices of w ((f(X Wg[e]^T) * (X Wu[e]^T)) Wd[e]^T); for training the net inputs of both
             projections too, pair by pair in the order of the lists
  exp_bwd    its gradients: of the rows, the experts' matrices and the weights
  clip       gradients of many tensors times min(1, max_norm / n), n the norm of all of them together; and n
"""
import math

import torch

own = False

LINEAR, SIGMOID, TANH, RELU, SILU, GELU = 0, 1, 2, 3, 5, 6
SOFTMAX_SCORES, SIGMOID_SCORES = 0, 1
DEVICE = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}


def listed():
    return [
        # serving: one token's choice, the shortest call there is
        {"name": "route_one", "kind": "route", "type": "bf16", "rows": 1, "experts": 128, "k": 8, "score": SOFTMAX_SCORES,
         "bias": False, "groups": 1, "top_groups": 1, "best": 1, "renorm": True, "scale": 1.0, "padded": 0.0},
        # training: a batch of tokens, some of it padding, balanced by a bias, groups of experts as on several devices
        {"name": "route_large", "kind": "route", "type": "f32", "rows": 16384, "experts": 256, "k": 8, "score": SIGMOID_SCORES,
         "bias": True, "groups": 8, "top_groups": 4, "best": 2, "renorm": True, "scale": 2.5, "padded": 0.05},
        # a prompt of odd length over an odd number of experts
        {"name": "route_odd", "kind": "route", "type": "f16", "rows": 1301, "experts": 60, "k": 4, "score": SOFTMAX_SCORES,
         "bias": False, "groups": 1, "top_groups": 1, "best": 1, "renorm": False, "scale": 1.0, "padded": 0.0},
        # training, backward: every logit of a row takes part in its softmax
        {"name": "route_bwd_large", "kind": "route_bwd", "type": "bf16", "rows": 16384, "experts": 128, "k": 8,
         "score": SOFTMAX_SCORES, "renorm": False, "scale": 1.0},
        # serving: one token through 8 of 64 experts; reading their matrices is all there is
        {"name": "experts_one", "kind": "experts", "type": "bf16", "rows": 1, "experts": 64, "k": 8, "d": 2048, "f": 1024,
         "act": SILU, "res": True, "keep": False, "padded": 0.0},
        # serving: a short ragged prompt, widths that are a multiple of nothing
        {"name": "experts_few", "kind": "experts", "type": "f16", "rows": 37, "experts": 16, "k": 2, "d": 1021, "f": 555,
         "act": GELU, "res": True, "keep": False, "padded": 0.0},
        # serving: a batch of 64 tokens that meets every expert, a few rows each
        {"name": "experts_batch", "kind": "experts", "type": "bf16", "rows": 64, "experts": 64, "k": 8, "d": 2048, "f": 1024,
         "act": SILU, "res": True, "keep": False, "padded": 0.0},
        # training, forward and backward: 8192 tokens, eight experts each
        {"name": "experts_fwd_large", "kind": "experts", "type": "bf16", "rows": 8192, "experts": 64, "k": 8, "d": 2048,
         "f": 1024, "act": SILU, "res": True, "keep": True, "padded": 0.0},
        {"name": "experts_bwd_large", "kind": "exp_bwd", "type": "bf16", "rows": 8192, "experts": 64, "k": 8, "d": 2048,
         "f": 1024, "act": SILU, "padded": 0.0},
        # training, backward, fp32 at odd widths; a tenth of the rows are padding
        {"name": "experts_bwd_ragged", "kind": "exp_bwd", "type": "f32", "rows": 1301, "experts": 8, "k": 2, "d": 777,
         "f": 1021, "act": GELU, "padded": 0.1},
        # a small classifier's fp32 gradients in place, whose norm is below the bound: nothing changes but the norm
        {"name": "clip_small", "kind": "clip", "type": "f32", "out": "same", "layers": 2, "d": 256, "f": 512, "clipped": False},
        # the gradients of 48 wide blocks, 16 bits, clipped into the fp32 ones that the step of the parameters reads
        {"name": "clip_large", "kind": "clip", "type": "bf16", "out": "f32", "layers": 48, "d": 2048, "f": 2048, "clipped": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Half of the widths a multiple of 64, a quarter of 8, a quarter of nothing."""
    w = _log(rng, lo, hi)
    q = rng.choice((64, 64, 8, 1))
    return max(q, w // q * q) if q > 1 else w | 1


def draw(rng):
    kind = rng.choice(("route", "route", "route_bwd", "experts", "experts", "experts", "exp_bwd", "exp_bwd", "clip"))
    t = rng.choice(("bf16", "bf16", "f16", "f32"))
    if kind == "clip":
        same = rng.random() < 0.5
        return {"kind": kind, "type": t, "out": "same" if same else rng.choice((t, "f32")), "layers": _log(rng, 1, 48),
                "d": _width(rng, 64, 2048), "f": _width(rng, 64, 2048), "clipped": not same}
    c = {"kind": kind, "type": t, "rows": _log(rng, 1, 16384)}
    if kind[:5] == "route":
        groups = rng.choice((1, 1, 4, 8))
        experts = groups * _log(rng, 2, 256 // groups)
        top = rng.randint(1, groups)
        c.update(experts=experts, k=min(rng.randint(1, 10), experts * top // groups), score=rng.randint(0, 1),
                 renorm=rng.random() < 0.5, scale=rng.choice((1.0, 2.5)))
        if kind == "route":
            c.update(bias=rng.random() < 0.5, groups=groups, top_groups=top, best=rng.choice((1, 2)),
                     padded=rng.choice((0.0, 0.05)))
        return c
    c.update(rows=_log(rng, 1, 8192), experts=_log(rng, 2, 96), d=_width(rng, 64, 2048), f=_width(rng, 64, 2048),
             act=rng.choice((SILU, GELU, RELU)), padded=rng.choice((0.0, 0.1)))
    c["k"] = min(rng.choice((1, 2, 4, 8)), c["experts"])
    if kind == "experts":
        c.update(res=rng.random() < 0.7, keep=rng.random() < 0.5)
    while c["experts"] * c["d"] * c["f"] > 64 * 2048 * 1024:
        c["experts"] = c["experts"] * 3 // 4
    c["k"] = min(c["k"], c["experts"])
    # the largest listed pass bounds the products, and fp32's matrix rate is a tenth of that of 16 bits
    most = 8192 * 8 * 2048 * 1024 // (10 if t == "f32" else 1)
    while c["rows"] * c["k"] * c["d"] * c["f"] > most:
        c["rows"] = c["rows"] * 3 // 4
    return c


def _tensors(case):
    """The sizes of a stack of blocks' parameters, as a training step meets them."""
    d, f = case["d"], case["f"]
    return [n for _ in range(case["layers"]) for n in (f * d, f * d, d * f, d, d, f, d * d)]


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    t, kind = TYPES[case["type"]], case["kind"]

    def normal(*shape, std=1.0, dtype=None):
        return torch.empty(shape, device=DEVICE).normal_(0.0, std, generator=g).to(dtype or t)

    def out(*shape, dtype=None):
        return torch.empty(shape, dtype=dtype or t, device=DEVICE)

    s = {"case": case}
    if kind == "clip":
        # one tensor behind the other in one buffer; layers differ in the size of their gradients; the bound is half of their norm, or twice it
        sizes = _tensors(case)
        s["flat"] = torch.cat([normal(n, std=10.0 ** (-3 - i % 3)) for i, n in enumerate(sizes)])
        s["grads"] = list(s["flat"].split(sizes))
        norm = math.sqrt(sum(n * 10.0 ** (-6 - 2 * (i % 3)) for i, n in enumerate(sizes)))
        s["max_norm"] = norm * (0.5 if case["clipped"] else 2.0)
        s["norm"] = out(1, dtype=torch.float32)
        s["all"] = s["flat"] if case["out"] == "same" else out(sum(sizes), dtype=TYPES[case["out"]])
        s["outs"] = list(s["all"].split(sizes))
        return s
    rows, e, k = case["rows"], case["experts"], case["k"]
    # what a router gives: some experts are liked by all rows
    logits = normal(rows, e, std=1.5, dtype=torch.float32) + normal(e, std=0.5, dtype=torch.float32)
    if kind == "route":
        logits = logits.masked_fill(torch.rand(rows, 1, device=DEVICE, generator=g) < case["padded"], -math.inf)
    s["L"] = logits.to(t)
    if kind == "route":
        s["bias"] = normal(e, std=0.05, dtype=torch.float32) if case["bias"] else None
        s.update(expert=out(rows, k, dtype=torch.int32), weight=out(rows, k, dtype=torch.float32),
                 starts=out(e + 1, dtype=torch.int32), order=out(rows * k, dtype=torch.int32),
                 place=out(rows * k, dtype=torch.int32))
        return s
    expert = torch.sort(s["L"].float(), dim=1, descending=True, stable=True)[1][:, :k]
    if kind == "route_bwd":
        s.update(expert=expert.int().contiguous(), dweight=normal(rows, k, dtype=torch.float32), dL=out(rows, e))
        return s
    weight = torch.softmax(logits.gather(1, expert), 1)
    none = torch.rand(rows, 1, device=DEVICE, generator=g) < case["padded"]
    expert, weight = expert.masked_fill(none, -1), weight.masked_fill(none, 0.0)
    s["weight"] = weight.contiguous()
    s["starts"], s["order"], s["place"] = _lists(expert, e)
    del s["L"]
    d, f = case["d"], case["f"]
    s.update(X=normal(rows, d), Wg=normal(e, f, d, std=d ** -0.5), Wu=normal(e, f, d, std=d ** -0.5),
             Wd=normal(e, d, f, std=f ** -0.5))
    if kind == "experts":
        s.update(R=normal(rows, d) if case["res"] else None, Y=out(rows, d),
                 GU=torch.zeros(rows * k, 2 * f, dtype=t, device=DEVICE) if case["keep"] else None)
    else:
        s.update(GU=normal(rows * k, 2 * f), dY=normal(rows, d), dX=out(rows, d), dWg=out(e, f, d), dWu=out(e, f, d),
                 dWd=out(e, d, f), dweight=out(rows, k, dtype=torch.float32))
    return s


# ---- the plain forms: 32 bits (64 where choices hang on them), elementary operations, one rounding at the end

def _lists(expert, experts):
    flat = expert.reshape(-1).long()
    none = flat < 0
    order = torch.sort(torch.where(none, experts, flat), stable=True)[1]
    starts = torch.zeros(experts + 1, dtype=torch.long, device=flat.device)
    starts.index_add_(0, torch.where(none, 0, flat + 1), (~none).long())
    starts = torch.cumsum(starts, 0)
    at = torch.arange(flat.numel(), device=flat.device)
    place = torch.empty_like(flat)
    place[order] = at
    return starts.int(), torch.where(at < starts[-1], order, -1).int(), torch.where(none, -1, place).int()


def _score(l, score):
    if score == SIGMOID_SCORES:
        return 1 / (1 + torch.exp(-l))
    x = torch.exp(l - l.amax(1, keepdim=True))
    return x / x.sum(1, keepdim=True)


def _route(s):
    c = s["case"]
    rows, e, k = c["rows"], c["experts"], c["k"]
    # neighbouring scores may differ in the last bits of 32
    l = s["L"].double()
    gone = l == -math.inf
    score = torch.nan_to_num(_score(l, c["score"]))
    rank = score if s["bias"] is None else score + s["bias"].double()
    rank = rank.masked_fill(gone, -math.inf)
    if c["groups"] > 1:
        by = rank.view(rows, c["groups"], -1)
        best = torch.sort(by, dim=2, descending=True)[0][:, :, :c["best"]]
        total = torch.where(best == -math.inf, 0.0, best).sum(2).masked_fill(best[:, :, 0] == -math.inf, -math.inf)
        keep = torch.sort(total, dim=1, descending=True, stable=True)[1][:, :c["top_groups"]]
        kept = torch.zeros_like(total, dtype=torch.bool).scatter_(1, keep, True)
        rank = by.masked_fill(~kept[:, :, None], -math.inf).view(rows, e)
    rank, expert = (v[:, :k] for v in torch.sort(rank, dim=1, descending=True, stable=True))
    none = rank == -math.inf
    weight = score.gather(1, expert).masked_fill(none, 0.0)
    if c["renorm"]:
        weight = torch.where(none, 0.0, weight / weight.sum(1, keepdim=True))
    expert = expert.masked_fill(none, -1).int()
    starts, order, place = _lists(expert, e)
    return {"expert": expert, "weight": (weight * c["scale"]).float(), "starts": starts, "order": order, "place": place}


def _route_bwd(s):
    c = s["case"]
    score = _score(s["L"].float(), c["score"])
    at = s["expert"].long()
    chosen, g = score.gather(1, at), s["dweight"] * c["scale"]
    if c["renorm"]:
        total = chosen.sum(1, keepdim=True)
        g = (g - (g * chosen).sum(1, keepdim=True) / total) / total
    ds = torch.zeros_like(score).scatter_(1, at, g)
    if c["score"] == SIGMOID_SCORES:
        return {"dL": (ds * score * (1 - score)).to(s["L"].dtype)}
    return {"dL": (score * (ds - (ds * score).sum(1, keepdim=True))).to(s["L"].dtype)}


def _f(z, act):
    if act == RELU:
        return torch.where(z > 0, z, 0.0)
    if act == SILU:
        return z / (1 + torch.exp(-z))
    return 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))


def _df(z, act):
    if act == RELU:
        return (z > 0).float()
    if act == SILU:
        a = 1 / (1 + torch.exp(-z))
        return a * (1 + z * (1 - a))
    return 0.5 * (1 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5


def _experts(s):
    c = s["case"]
    t, f, k = TYPES[c["type"]], c["f"], c["k"]
    starts, order = s["starts"].tolist(), s["order"].long()
    x, weight = s["X"].float(), s["weight"].view(-1)
    y = torch.zeros_like(x) if s["R"] is None else s["R"].float()
    kept = torch.zeros(order.numel(), 2 * f, dtype=t, device=DEVICE) if c["keep"] else None
    for e in range(c["experts"]):
        p, q = starts[e], starts[e + 1]
        if p == q:
            continue
        pair = order[p:q]
        rows = x[pair // k]
        g, u = rows @ s["Wg"][e].float().t(), rows @ s["Wu"][e].float().t()
        z = (_f(g, c["act"]) * u) @ s["Wd"][e].float().t()
        y.index_add_(0, pair // k, z * weight[pair][:, None])
        if c["keep"]:
            kept[p:q, :f], kept[p:q, f:] = g.to(t), u.to(t)
    return {"Y": y.to(t), **({"GU": kept} if c["keep"] else {})}


def _exp_bwd(s):
    c = s["case"]
    t, f, k = TYPES[c["type"]], c["f"], c["k"]
    starts, order = s["starts"].tolist(), s["order"].long()
    x, dy, weight = s["X"].float(), s["dY"].float(), s["weight"].view(-1)
    dx, dweight = torch.zeros_like(x), torch.zeros_like(weight)
    r = {n: torch.zeros_like(s[n]) for n in ("dWg", "dWu", "dWd")}
    for e in range(c["experts"]):
        p, q = starts[e], starts[e + 1]
        if p == q:
            continue
        pair = order[p:q]
        rows, dz, w = x[pair // k], dy[pair // k], weight[pair][:, None]
        g, u = s["GU"][p:q].float().split(f, 1)
        a = _f(g, c["act"])
        dh = dz @ s["Wd"][e].float()
        dweight[pair] = (dh * a * u).sum(1)
        dg, du = w * dh * u * _df(g, c["act"]), w * dh * a
        dx.index_add_(0, pair // k, dg @ s["Wg"][e].float() + du @ s["Wu"][e].float())
        r["dWg"][e], r["dWu"][e], r["dWd"][e] = (dg.t() @ rows).to(t), (du.t() @ rows).to(t), (dz.t() @ (w * a * u)).to(t)
    return {"dX": dx.to(t), **r, "dweight": dweight.view(-1, k)}


def _clip(s):
    total = torch.zeros((), dtype=torch.float64, device=DEVICE)
    for v in s["grads"]:
        v = v.float()
        total += (v * v).sum(dtype=torch.float64)
    norm = torch.sqrt(total)
    factor = torch.clamp(s["max_norm"] / norm, max=1.0).float()
    for v, o in zip(s["grads"], s["outs"]):
        o.copy_(v.float() * factor)
    s["norm"].copy_(norm.view(1))
    return {"norm": s["norm"], "grads": s["all"]}


def _own(s):
    from paper_2001_04206_amd import dn
    c = s["case"]
    kind = c["kind"]

    def outputs(*names):
        return {k: s[k] for k in names if s[k] is not None}

    if kind == "route":
        dn.dn_route_forward(s["L"], s["bias"], s["expert"], s["weight"], s["starts"], s["order"], s["place"], score=c["score"],
                            groups=c["groups"], top_groups=c["top_groups"], group_best=c["best"], renorm=c["renorm"],
                            scale=c["scale"])
        return outputs("expert", "weight", "starts", "order", "place")
    if kind == "route_bwd":
        dn.dn_route_backward(s["L"], s["expert"], s["dweight"], s["dL"], score=c["score"], renorm=c["renorm"], scale=c["scale"])
        return outputs("dL")
    if kind == "experts":
        dn.dn_experts_forward(s["X"], s["Wg"], s["Wu"], s["Wd"], s["weight"], s["starts"], s["order"], s["place"], s["R"],
                              s["Y"], s["GU"], act=c["act"])
        return outputs("Y", "GU")
    if kind == "exp_bwd":
        dn.dn_experts_backward(s["X"], s["Wg"], s["Wu"], s["Wd"], s["weight"], s["starts"], s["order"], s["place"], s["GU"],
                               s["dY"], s["dX"], s["dWg"], s["dWu"], s["dWd"], s["dweight"], act=c["act"])
        return outputs("dX", "dWg", "dWu", "dWd", "dweight")
    dn.dn_clip(s["grads"], s["max_norm"], s["norm"], s["outs"])
    return {"norm": s["norm"], "grads": s["all"]}


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    return {"route": _route, "route_bwd": _route_bwd, "experts": _experts, "exp_bwd": _exp_bwd, "clip": _clip}[kind](state)


def work(case):
    e, kind = SIZE[case["type"]], case["kind"]
    if kind == "clip":
        n = sum(_tensors(case))
        # read once for the norm; read again and written where the result has to be
        write = 0 if case["out"] == "same" else e + SIZE[case["out"]]
        return {"bytes": n * (e + write), "flops": 3 * n}
    rows, n, k = case["rows"], case["experts"], case["k"]
    pairs = rows * k
    if kind == "route":
        return {"bytes": e * rows * n + 16 * pairs + 4 * n, "flops": 20 * rows * n}
    if kind == "route_bwd":
        return {"bytes": 2 * e * rows * n + 8 * pairs, "flops": 20 * rows * n}
    d, f = case["d"], case["f"]
    met = min(n, pairs)
    pairs = pairs * (1 - case["padded"])
    if kind == "experts":
        moved = 3 * met * d * f + rows * d * (2 + case["res"]) + 2 * pairs * f * case["keep"]
        return {"bytes": int(e * moved), "flops": int(6 * pairs * d * f)}
    moved = 3 * met * d * f + 3 * n * d * f + 3 * rows * d + 2 * pairs * f
    return {"bytes": int(e * moved), "flops": int(12 * pairs * d * f)}


# ---- the definitions in 64 bits: choices one after another, gradients by differentiation

def _exact_route(s, c):
    l = s["L"].double()
    rows, e = l.shape
    p = torch.sigmoid(l) if c["score"] == SIGMOID_SCORES else torch.softmax(l, 1)
    left = p.clone() if s["bias"] is None else p + s["bias"].double()
    left[torch.isinf(l)] = -math.inf
    each = e // c["groups"]
    if c["groups"] > 1:
        scores = []
        for i in range(c["groups"]):
            top = left[:, i * each:(i + 1) * each].topk(min(c["best"], each), 1).values
            scores.append(torch.where(top.isinf(), torch.zeros_like(top), top).sum(1) + torch.where(top[:, 0].isinf(), -math.inf, 0.0))
        scores = torch.stack(scores, 1)
        # a group stays if fewer than top_groups come before it
        i = torch.arange(c["groups"], device=DEVICE)
        before = (scores[:, None, :] > scores[:, :, None]) | ((scores[:, None, :] == scores[:, :, None]) & (i[None, :] < i[:, None]))
        left[(before.sum(2) >= c["top_groups"]).repeat_interleave(each, 1)] = -math.inf
    number = torch.arange(e, device=DEVICE)
    expert = torch.full((rows, c["k"]), -1, device=DEVICE)
    weight = torch.zeros(rows, c["k"], dtype=torch.float64, device=DEVICE)
    for j in range(c["k"]):
        high = left.amax(1, keepdim=True)
        first = torch.where(left == high, number, e).amin(1, keepdim=True)
        found = (high > -math.inf)[:, 0]
        expert[found, j] = first[found, 0]
        weight[found, j] = p.gather(1, first)[found, 0]
        left.scatter_(1, first, -math.inf)
    if c["renorm"]:
        total = weight.sum(1, keepdim=True)
        weight = torch.where(total > 0, weight / total, weight)
    # pairs by expert: where each pair goes is how many go before it
    flat = expert.view(-1)
    count = torch.bincount(flat[flat >= 0], minlength=e)
    starts = torch.cat((torch.zeros(1, dtype=torch.long, device=DEVICE), count.cumsum(0)))
    order, place = torch.full_like(flat, -1), torch.full_like(flat, -1)
    for i in range(e):
        mine = (flat == i).nonzero()[:, 0]
        at = starts[i] + torch.arange(mine.numel(), device=DEVICE)
        order[at], place[mine] = mine, at
    return {"expert": expert.int(), "weight": weight * c["scale"], "starts": starts.int(), "order": order.int(), "place": place.int()}


def exact(case, seed):
    s, c = prepare(case, seed), case
    kind = c["kind"]
    if kind == "route":
        return _exact_route(s, c)
    if kind == "route_bwd":
        l = s["L"].double().requires_grad_()
        p = torch.sigmoid(l) if c["score"] == SIGMOID_SCORES else torch.softmax(l, 1)
        w = torch.take_along_dim(p, s["expert"].long(), 1)
        if c["renorm"]:
            w = w / w.sum(1, keepdim=True)
        return {"dL": torch.autograd.grad(w * c["scale"], l, s["dweight"].double())[0]}
    if kind == "clip":
        parts = [torch.linalg.vector_norm(v.double()) for v in s["grads"]]
        norm = torch.linalg.vector_norm(torch.stack(parts))
        by = min(1.0, s["max_norm"] / norm.item())
        return {"norm": norm.view(1), "grads": s["flat"].double() * by}
    k, f, pairs = c["k"], c["f"], c["rows"] * c["k"]
    act = {RELU: torch.relu, SILU: torch.nn.functional.silu, GELU: lambda z: z * torch.special.ndtr(z)}[c["act"]]
    token = s["order"].long().clamp(min=0) // k
    weight = s["weight"].double().view(-1)
    bounds = s["starts"].tolist()
    x = s["X"].double()
    if kind == "experts":
        y = torch.zeros_like(x) if s["R"] is None else s["R"].double()
        gu = torch.zeros(pairs, 2 * f, dtype=torch.float64, device=DEVICE)
        for e, (a, b) in enumerate(zip(bounds, bounds[1:])):
            if a < b:
                gu[a:b] = torch.matmul(x[token[a:b]], torch.vstack((s["Wg"][e], s["Wu"][e])).double().T)
                z = torch.matmul(act(gu[a:b, :f]) * gu[a:b, f:], s["Wd"][e].double().T)
                y.index_put_((token[a:b],), z * weight[s["order"][a:b].long(), None], accumulate=True)
        return {"Y": y, **({"GU": gu} if c["keep"] else {})}
    # backward is given G and U: the derivative goes through them to the matrices and the rows
    dy = s["dY"].double()
    r = {"dX": torch.zeros_like(x), "dweight": torch.zeros_like(weight)}
    big = {n: torch.zeros(s[n].shape, dtype=torch.float64, device=DEVICE) for n in ("dWg", "dWu", "dWd")}
    for e, (a, b) in enumerate(zip(bounds, bounds[1:])):
        if a < b:
            pair = s["order"][a:b].long()
            gu = s["GU"][a:b].double().requires_grad_()
            wd, w = s["Wd"][e].double().requires_grad_(), weight[pair].requires_grad_()
            z = w[:, None] * torch.matmul(act(gu[:, :f]) * gu[:, f:], wd.T)
            dgu, big["dWd"][e], r["dweight"][pair] = torch.autograd.grad(z, (gu, wd, w), dy[token[a:b]])
            both = torch.matmul(dgu.T, x[token[a:b]])
            big["dWg"][e], big["dWu"][e] = both[:f], both[f:]
            r["dX"].index_put_((token[a:b],), torch.matmul(dgu, torch.vstack((s["Wg"][e], s["Wu"][e])).double()), accumulate=True)
    return {"dX": r["dX"], **big, "dweight": r["dweight"].view(-1, k)}
