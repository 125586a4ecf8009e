"""A block of experts in 64 bits, by its formulas and on the CPU, for the tests."""
import math

import torch

from ffn_util import df64, f64
from paper_2001_04206_amd import dn

NINF = -math.inf


def route64(L, bias, k, score, groups=1, top_groups=1, best=1, renorm=True, scale=1.0):
    """Choices and weights of every row, one row and one choice at a time: expert [rows][k], weight [rows][k] (64 bits)."""
    L = L.double().cpu()
    rows, experts = L.shape
    s = torch.softmax(L, 1) if score == dn.DN_SCORE_SOFTMAX else torch.sigmoid(L)
    expert, weight = torch.full((rows, k), -1, dtype=torch.int32), torch.zeros(rows, k, dtype=torch.float64)
    each = experts // groups
    for t in range(rows):
        # without a bias the order is the logits' own
        ranks = L[t].tolist() if bias is None else (s[t] + bias.double().cpu()).tolist()
        ranks = [NINF if l == NINF else math.inf if r != r else r for r, l in zip(ranks, L[t].tolist())]
        left = set(range(experts))
        if top_groups < groups:
            by = ranks if bias is not None or best == 1 else s[t].tolist()
            by = [NINF if r == NINF else v for v, r in zip(by, ranks)]
            total = []
            for g in range(groups):
                have = sorted((v for v in by[g * each:(g + 1) * each] if v > NINF), reverse=True)[:best]
                total.append(sum(have) if have else NINF)
            keep = sorted((g for g in range(groups) if total[g] > NINF), key=lambda g: (-total[g], g))[:top_groups]
            left = {e for g in keep for e in range(g * each, (g + 1) * each)}
        chosen = sorted((e for e in left if ranks[e] > NINF), key=lambda e: (-ranks[e], e))[:k]
        if not chosen:
            continue
        if renorm:   # ratios, from the scores' logarithms
            logs = [L[t, e].item() if score == dn.DN_SCORE_SOFTMAX else -math.log1p(math.exp(-L[t, e].item())) if L[t, e] > -700
                    else L[t, e].item() for e in chosen]
            w = torch.softmax(torch.tensor(logs, dtype=torch.float64), 0)
        else:
            w = s[t, chosen]
        expert[t, :len(chosen)] = torch.tensor(chosen, dtype=torch.int32)
        weight[t, :len(chosen)] = w * scale
    return expert, weight


def lists(expert, experts):
    """starts, order, place of a table of choices, pair by pair."""
    flat = expert.cpu().reshape(-1).tolist()
    by = [[q for q, e in enumerate(flat) if e == i] for i in range(experts)] if len(flat) * experts < 1e6 else None
    if by is None:
        by = [[] for _ in range(experts)]
        for q, e in enumerate(flat):
            if 0 <= e < experts:
                by[e].append(q)
    order = [q for b in by for q in b]
    starts = [0]
    for b in by:
        starts.append(starts[-1] + len(b))
    place = [-1] * len(flat)
    for p, q in enumerate(order):
        place[q] = p
    order += [-1] * (len(flat) - len(order))
    return tuple(torch.tensor(v, dtype=torch.int32) for v in (starts, order, place))


def forward64(X, Wg, Wu, Wd, weight, expert, R, act, on="cpu"):
    """Y, and G, U of every pair [rows][k][f]; `on`: where it is computed."""
    X, Wg, Wu, Wd, weight, expert = (t.detach().to(on) for t in (X, Wg, Wu, Wd, weight, expert))
    rows, k = expert.shape
    f, d = Wg.shape[1:]
    Y = torch.zeros(rows, d, dtype=torch.float64, device=on) if R is None else R.double().to(on).clone()
    G, U = (torch.zeros(rows, k, f, dtype=torch.float64, device=on) for _ in range(2))
    for e in range(Wg.shape[0]):
        t, j = (expert == e).nonzero(as_tuple=True)
        if len(t):
            x = X[t].double()
            G[t, j], U[t, j] = x @ Wg[e].double().T, x @ Wu[e].double().T
            z = (f64(G[t, j], act) * U[t, j]) @ Wd[e].double().T
            Y.index_add_(0, t, z * weight[t, j].double()[:, None])
    return Y, G, U


def backward64(X, Wg, Wu, Wd, weight, expert, G, U, dY, act, grad_scale=1.0, on="cpu"):
    """dX, dWg, dWu, dWd, dweight, from G and U [rows][k][f] as the forward call left them."""
    X, Wg, Wu, Wd, weight, expert, dY = (t.detach().to(on) for t in (X, Wg, Wu, Wd, weight, expert, dY))
    dX, dweight = (torch.zeros(t.shape, dtype=torch.float64, device=on) for t in (X, expert))
    dWg, dWu, dWd = (torch.zeros(w.shape, dtype=torch.float64, device=on) for w in (Wg, Wu, Wd))
    for e in range(Wg.shape[0]):
        t, j = (expert == e).nonzero(as_tuple=True)
        if not len(t):
            continue
        x, dz, w, g, u = X[t].double(), dY[t].double(), weight[t, j].double()[:, None], G[t, j].double(), U[t, j].double()
        a = f64(g, act)
        dh = dz @ Wd[e].double()
        dweight[t, j] = (dh * a * u).sum(1)
        dg, du = w * dh * u * df64(g, act), w * dh * a
        dX.index_add_(0, t, dg @ Wg[e].double() + du @ Wu[e].double())
        dWg[e], dWu[e], dWd[e] = dg.T @ x, du.T @ x, dz.T @ (w * a * u)
    return dX, dWg * grad_scale, dWu * grad_scale, dWd * grad_scale, dweight
