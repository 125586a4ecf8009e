"""Timed cases of the residual feed-forward block's operators: what a program that trains or serves such blocks calls.

A case is one of seven kinds:
  lin_fwd   Y = R + D(f(X W^T + b)): a dense layer with bias, activation, dropout and residual; Z = X W^T + b too for training
  lin_bwd   its gradients: dX, dW, db from dY (the residual's gradient is dY itself)
  ffn_fwd   Y = R + D((f(X Wg^T + bg) * (X Wu^T + bu)) Wd^T + bd): the gated feed-forward block; for training the
            net inputs of both projections too, G beside U
  ffn_bwd   its gradients: of the input, the three matrices and the three biases
  norm_fwd  x' = x + s gate * post(b),  n' = pre(x'): the norm after one block, its gate, scale and residual, and the norm
            before the next one
  norm_bwd  its gradients: of x, b, gate and the norms' weights (and shifts)
  drop      Y = D(X), dropout by itself (forward and backward are the same call)
D keeps the element in row i, column j where the 16-bit number of (seed, offset, i, j) is at least t = round(65536 p), and
multiplies it by 65536 / (65536 - t); the numbers are Philox 4x32-10's (Salmon, Moraes, Dror and Shaw, "Parallel random
numbers: as easy as 1, 2, 3", 2011) for the counter (j div 8, i, offset) and the key `seed`: number j mod 8 of the eight in
its four words, low half first.
"""
import math

import numpy as np
import torch

own = False

LINEAR, SIGMOID, TANH, RELU, SILU, GELU = 0, 1, 2, 3, 5, 6
NONE, RMS, LAYER = 0, 1, 2
DEVICE = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-5


def listed():
    return [
        # serving: one token through a projection back to the residual stream
        {"name": "lin_one", "kind": "lin_fwd", "type": "bf16", "rows": 1, "n_in": 4096, "n_out": 4096, "act": LINEAR,
         "bias": True, "res": True, "drop": 0.0, "keep": False, "pad": 0},
        # training, forward: a wide layer with everything in its epilogue
        {"name": "lin_fwd_wide", "kind": "lin_fwd", "type": "bf16", "rows": 8192, "n_in": 4096, "n_out": 4096,
         "act": GELU, "bias": True, "res": True, "drop": 0.1, "keep": True, "pad": 0},
        # training, backward: fp32 as the dense nets are, widths and rows that are a multiple of nothing, rows of X apart
        {"name": "lin_bwd_ragged", "kind": "lin_bwd", "type": "f32", "rows": 1301, "n_in": 1021, "n_out": 777,
         "act": TANH, "bias": True, "res": True, "drop": 0.1, "keep": True, "pad": 3},
        # serving: one token through the gated block; reading three matrices is all there is
        {"name": "ffn_one", "kind": "ffn_fwd", "type": "bf16", "rows": 1, "d": 4096, "f": 8192, "act": SILU,
         "bias": False, "res": True, "drop": 0.0, "keep": False},
        # serving: a short ragged prompt, nothing a multiple of anything
        {"name": "ffn_few", "kind": "ffn_fwd", "type": "f16", "rows": 37, "d": 1021, "f": 2731, "act": GELU,
         "bias": True, "res": True, "drop": 0.0, "keep": False},
        # training, forward and backward: 8192 tokens of a wide block
        {"name": "ffn_fwd_large", "kind": "ffn_fwd", "type": "bf16", "rows": 8192, "d": 4096, "f": 8192, "act": SILU,
         "bias": False, "res": True, "drop": 0.1, "keep": True},
        {"name": "ffn_bwd_large", "kind": "ffn_bwd", "type": "bf16", "rows": 8192, "d": 4096, "f": 8192, "act": SILU,
         "bias": False, "res": True, "drop": 0.1, "keep": True},
        # serving: one token between two blocks
        {"name": "norm_one", "kind": "norm_fwd", "type": "bf16", "rows": 1, "d": 4096, "post": RMS, "pre": RMS,
         "group": 1, "scale": 0.5},
        # training, forward and backward between two blocks; eight sequences with a gate each
        {"name": "norm_fwd_large", "kind": "norm_fwd", "type": "bf16", "rows": 16384, "d": 4096, "post": RMS,
         "pre": RMS, "group": 2048, "scale": 0.5},
        {"name": "norm_bwd_large", "kind": "norm_bwd", "type": "bf16", "rows": 16384, "d": 4096, "post": RMS,
         "pre": LAYER, "group": 2048, "scale": 0.5},
        # dropout by itself: a small fp32 layer of the dense nets, and a whole batch of tokens
        {"name": "drop_small", "kind": "drop", "type": "f32", "rows": 256, "cols": 777, "drop": 0.5},
        {"name": "drop_large", "kind": "drop", "type": "bf16", "rows": 16384, "cols": 4096, "drop": 0.1},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Half of the widths a multiple of 64, a quarter of 8, a quarter of nothing."""
    w = _log(rng, lo, hi)
    q = rng.choice((64, 64, 8, 1))
    return max(q, w // q * q) if q > 1 else w | 1


def draw(rng):
    kind = rng.choice(("lin_fwd", "lin_bwd", "ffn_fwd", "ffn_fwd", "ffn_bwd", "ffn_bwd", "norm_fwd", "norm_bwd", "drop"))
    t = rng.choice(("bf16", "bf16", "f16", "f32"))
    if kind == "drop":
        return {"kind": kind, "type": t, "rows": _log(rng, 1, 16384), "cols": _width(rng, 32, 4096),
                "drop": rng.choice((0.05, 0.1, 0.5))}
    if kind in ("norm_fwd", "norm_bwd"):
        rows = _log(rng, 1, 16384)
        return {"kind": kind, "type": t, "rows": rows, "d": _width(rng, 64, 4096), "post": rng.choice((NONE, RMS, LAYER)),
                "pre": rng.choice((RMS, LAYER)), "group": rng.choice((rows, max(1, rows // 4), 1)),
                "scale": rng.choice((1.0, 0.5))}
    rows = _log(rng, 1, 8192)
    act = rng.choice((SILU, GELU, RELU, TANH))
    c = {"kind": kind, "type": t, "rows": rows}
    if kind[:3] == "lin":
        c.update(n_in=_width(rng, 64, 4096), n_out=_width(rng, 64, 4096), act=rng.choice((act, LINEAR)),
                 pad=rng.choice((0, 0, 8, 3)))
    else:
        c.update(d=_width(rng, 64, 4096), f=_width(rng, 64, 8192), act=act)
    train = kind[4:] == "bwd" or rng.random() < 0.5
    c.update(bias=rng.random() < 0.5, res=rng.random() < 0.7, drop=rng.choice((0.0, 0.1)) if train else 0.0, keep=train)
    return c


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    t = TYPES[case["type"]]

    def normal(*shape, std=1.0, mean=0.0):
        return torch.empty(shape, device=DEVICE).normal_(mean, std, generator=g).to(t)

    def out(*shape):
        return torch.empty(shape, dtype=t, device=DEVICE)

    rows, kind = case["rows"], case["kind"]
    s = {"case": case, "seed": seed * 0x9E3779B97F4A7C15 % 2 ** 64, "offset": seed % 1000}
    if kind == "drop":
        s.update(X=normal(rows, case["cols"]), Y=out(rows, case["cols"]))
    elif kind[:4] == "norm":
        d = case["d"]
        groups = -(-rows // case["group"])
        # a residual stream, a block's output on it, weights around 1, gates around 1
        s.update(x=normal(rows, d, std=2.0), b=normal(rows, d), gate=normal(groups, d, std=0.2, mean=1.0),
                 post_w=normal(d, std=0.1, mean=1.0) if case["post"] else None,
                 post_b=normal(d, std=0.1) if case["post"] == LAYER else None,
                 pre_w=normal(d, std=0.1, mean=1.0), pre_b=normal(d, std=0.1) if case["pre"] == LAYER else None)
        if kind == "norm_fwd":
            s.update(x_out=out(rows, d), n_out=out(rows, d))
        else:
            s.update(dx_out=normal(rows, d), dn=normal(rows, d), dx=out(rows, d), db=out(rows, d), dgate=out(groups, d))
            for k in ("post_w", "post_b", "pre_w", "pre_b"):
                s["d" + k] = None if s[k] is None else out(d)
    elif kind[:3] == "lin":
        n, m = case["n_in"], case["n_out"]
        s.update(X=normal(rows, n + case["pad"])[:, :n], W=normal(m, n, std=n ** -0.5))
        s["bias"] = normal(m, std=0.1) if case["bias"] else None
        if kind == "lin_fwd":
            s.update(R=normal(rows, m) if case["res"] else None, Y=out(rows, m), Z=out(rows, m) if case["keep"] else None)
        else:
            s.update(Z=normal(rows, m), dY=normal(rows, m), dX=out(rows, n), dW=out(m, n),
                     dbias=out(m) if case["bias"] else None)
    else:
        d, f = case["d"], case["f"]
        s.update(X=normal(rows, d), Wg=normal(f, d, std=d ** -0.5), Wu=normal(f, d, std=d ** -0.5),
                 Wd=normal(d, f, std=f ** -0.5))
        for k, n in (("bg", f), ("bu", f), ("bd", d)):
            s[k] = normal(n, std=0.1) if case["bias"] else None
            s["d" + k] = out(n) if case["bias"] and kind == "ffn_bwd" else None
        if kind == "ffn_fwd":
            s.update(R=normal(rows, d) if case["res"] else None, Y=out(rows, d),
                     GU=out(rows, 2 * f) if case["keep"] else None)
        else:
            s.update(GU=normal(rows, 2 * f), dY=normal(rows, d), dX=out(rows, d), dWg=out(f, d), dWu=out(f, d),
                     dWd=out(d, f))
    return s


# ---- the plain forms: 32 bits, elementary operations, one rounding at the end

def _f(z, act):
    if act == SIGMOID:
        return 1 / (1 + torch.exp(-z))
    if act == TANH:
        return torch.tanh(z)
    if act == RELU:
        return torch.where(z > 0, z, 0.0)
    if act == SILU:
        return z / (1 + torch.exp(-z))
    if act == GELU:
        return 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
    return z


def _df(z, act):
    if act == SIGMOID:
        a = 1 / (1 + torch.exp(-z))
        return a * (1 - a)
    if act == TANH:
        return 1 - torch.tanh(z) ** 2
    if act == RELU:
        return (z > 0).float()
    if act == SILU:
        a = 1 / (1 + torch.exp(-z))
        return a * (1 + z * (1 - a))
    if act == GELU:
        return 0.5 * (1 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5
    return torch.ones_like(z)


def _keep(rows, cols, drop, seed, offset):
    """What dropout multiplies by: 0 or 65536 / (65536 - t)."""
    t = int(drop * 65536 + 0.5)
    low = 0xFFFFFFFF
    calls = -(-cols // 8)
    c0 = torch.arange(calls, device=DEVICE)[None, :].expand(rows, -1)
    c1 = torch.arange(rows, device=DEVICE)[:, None].expand(-1, calls)
    c2, c3 = torch.full_like(c0, offset & low), torch.full_like(c0, offset >> 32)
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        p, q = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = (q >> 32 & low) ^ c1 ^ k0, q & low, (p >> 32 & low) ^ c3 ^ k1, p & low
        k0, k1 = k0 + 0x9E3779B9 & low, k1 + 0xBB67AE85 & low
    w = torch.stack((c0, c1, c2, c3), -1)
    u = torch.stack((w & 0xFFFF, w >> 16), -1).view(rows, 8 * calls)[:, :cols]
    return torch.where(u >= t, 65536 / (65536 - t), 0.0)


def _drop(v, s):
    c = s["case"]
    return v if c["drop"] == 0 else v * _keep(v.shape[0], v.shape[1], c["drop"], s["seed"], s["offset"])


def _plus(v, w):
    return v if w is None else v + w.float()


def _normed(v, kind, w, b):
    """The norm's result, its input normalised, and the reciprocal of its deviation."""
    if kind == NONE:
        return v, v, None
    if kind == LAYER:
        v = v - v.mean(1, keepdim=True)
    r = 1 / torch.sqrt((v * v).mean(1, keepdim=True) + EPS)
    return _plus(v * r * w.float(), b), v * r, r


def _norm_back(dy, kind, w, hat, r):
    if kind == NONE:
        return dy
    q = dy * w.float()
    dv = q - hat * (q * hat).mean(1, keepdim=True)
    if kind == LAYER:
        dv = dv - q.mean(1, keepdim=True)
    return dv * r


def _plain(s):
    c = s["case"]
    t, kind = TYPES[c["type"]], c["kind"]

    def done(**v):
        return {k: x.to(t) for k, x in v.items() if x is not None}

    if kind == "drop":
        return done(Y=_drop(s["X"].float(), s))
    if kind == "lin_fwd":
        z = _plus(s["X"].float() @ s["W"].float().t(), s["bias"])
        return done(Y=_plus(_drop(_f(z, c["act"]), s), s["R"]), Z=z if c["keep"] else None)
    if kind == "lin_bwd":
        delta = _drop(s["dY"].float(), s) * _df(s["Z"].float(), c["act"])
        return done(dX=delta @ s["W"].float(), dW=delta.t() @ s["X"].float(), dbias=delta.sum(0) if c["bias"] else None)
    if kind == "ffn_fwd":
        x = s["X"].float()
        g, u = _plus(x @ s["Wg"].float().t(), s["bg"]), _plus(x @ s["Wu"].float().t(), s["bu"])
        y = _plus((_f(g, c["act"]) * u) @ s["Wd"].float().t(), s["bd"])
        return done(Y=_plus(_drop(y, s), s["R"]), GU=torch.cat((g, u), 1) if c["keep"] else None)
    if kind == "ffn_bwd":
        x, dy = s["X"].float(), _drop(s["dY"].float(), s)
        g, u = s["GU"].float().split(c["f"], 1)
        a = _f(g, c["act"])
        dh = dy @ s["Wd"].float()
        dg, du = dh * u * _df(g, c["act"]), dh * a
        r = {"dX": dg @ s["Wg"].float() + du @ s["Wu"].float(), "dWg": dg.t() @ x, "dWu": du.t() @ x, "dWd": dy.t() @ (a * u)}
        if c["bias"]:
            r.update(dbg=dg.sum(0), dbu=du.sum(0), dbd=dy.sum(0))
        return done(**r)
    rows, d, group = c["rows"], c["d"], c["group"]
    which = torch.arange(rows, device=DEVICE) // group
    gate = s["gate"].float()[which] * c["scale"]
    post, hat, r = _normed(s["b"].float(), c["post"], s["post_w"], s["post_b"])
    if kind == "norm_fwd":
        x = s["x"].float() + gate * post
        return done(x_out=x, n_out=_normed(x, c["pre"], s["pre_w"], s["pre_b"])[0])
    dn = s["dn"].float()
    _, xhat, xr = _normed(s["x"].float(), c["pre"], s["pre_w"], s["pre_b"])
    dx = s["dx_out"].float() + _norm_back(dn, c["pre"], s["pre_w"], xhat, xr)
    dc = gate * dx
    dgate = torch.zeros_like(s["gate"], dtype=torch.float32).index_add_(0, which, c["scale"] * dx * post)
    return done(dx=dx, db=_norm_back(dc, c["post"], s["post_w"], hat, r), dgate=dgate,
                dpost_w=(dc * hat).sum(0) if c["post"] else None, dpost_b=dc.sum(0) if c["post"] == LAYER else None,
                dpre_w=(dn * xhat).sum(0), dpre_b=dn.sum(0) if c["pre"] == LAYER else None)


def _own(s):
    from paper_2001_04206_amd import dn
    c = s["case"]
    kind = c["kind"]

    def outputs(*names):
        return {k: s[k] for k in names if s[k] is not None}

    if kind == "drop":
        dn.dn_dropout(s["X"], s["Y"], c["drop"], s["seed"], s["offset"])
        return outputs("Y")
    if kind == "norm_fwd":
        dn.dn_norm_forward(s["x"], s["b"], s["gate"], s["post_w"], s["post_b"], s["pre_w"], s["pre_b"], s["x_out"], s["n_out"],
                           post=c["post"], pre=c["pre"], scale=c["scale"], eps=EPS, rows_per_gate=c["group"])
        return outputs("x_out", "n_out")
    if kind == "norm_bwd":
        dn.dn_norm_backward(s["x"], s["b"], s["gate"], s["post_w"], s["post_b"], s["pre_w"], s["dx_out"], s["dn"],
                            s["dx"], s["db"], s["dgate"], s["dpost_w"], s["dpost_b"], s["dpre_w"], s["dpre_b"],
                            post=c["post"], pre=c["pre"], scale=c["scale"], eps=EPS, rows_per_gate=c["group"])
        return outputs("dx", "db", "dgate", "dpost_w", "dpost_b", "dpre_w", "dpre_b")
    drop = {"drop": c["drop"], "seed": s["seed"], "offset": s["offset"]}
    if kind == "lin_fwd":
        dn.dn_linear_forward(s["X"], s["W"], s["bias"], s["R"], s["Y"], s["Z"], act=c["act"], **drop)
        return outputs("Y", "Z")
    if kind == "lin_bwd":
        dn.dn_linear_backward(s["X"], s["W"], s["Z"], s["dY"], s["dX"], s["dW"], s["dbias"], act=c["act"], **drop)
        return outputs("dX", "dW", "dbias")
    if kind == "ffn_fwd":
        dn.dn_ffn_forward(s["X"], s["Wg"], s["bg"], s["Wu"], s["bu"], s["Wd"], s["bd"], s["R"], s["Y"], s["GU"],
                          act=c["act"], **drop)
        return outputs("Y", "GU")
    dn.dn_ffn_backward(s["X"], s["Wg"], s["Wu"], s["Wd"], s["GU"], s["dY"], s["dX"], s["dWg"], s["dbg"], s["dWu"],
                       s["dbu"], s["dWd"], s["dbd"], act=c["act"], **drop)
    return outputs("dX", "dWg", "dWu", "dWd", "dbg", "dbu", "dbd")


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    e, rows, kind = SIZE[case["type"]], case["rows"], case["kind"]
    if kind == "drop":
        n = rows * case["cols"]
        return {"bytes": 2 * e * n, "flops": n}
    if kind[:4] == "norm":
        d = case["d"]
        n, groups = rows * d, -(-rows // case["group"])
        small = e * d * (groups + 2 * bool(case["post"]) + 2)
        if kind == "norm_fwd":
            return {"bytes": 4 * e * n + small, "flops": 12 * n}
        return {"bytes": 6 * e * n + 2 * small, "flops": 30 * n}
    if kind[:3] == "lin":
        n, m = case["n_in"], case["n_out"]
        x, y, w = rows * n, rows * m, n * m
        if kind == "lin_fwd":
            moved = x + w + y * (1 + case["res"] + case["keep"]) + m * case["bias"]
            return {"bytes": e * moved, "flops": 2 * rows * w}
        return {"bytes": e * (2 * x + 2 * w + 2 * y + m * case["bias"]), "flops": 4 * rows * w}
    d, f = case["d"], case["f"]
    x, h, w, b = rows * d, rows * f, 3 * d * f, (2 * f + d) * case["bias"]
    if kind == "ffn_fwd":
        return {"bytes": e * (x * (2 + case["res"]) + 2 * h * case["keep"] + w + b), "flops": 2 * rows * w}
    return {"bytes": e * (3 * x + 2 * h + 2 * w + b), "flops": 4 * rows * w}


# ---- the definitions in 64 bits, by differentiation

def _numbers(rows, cols, seed, offset):
    """The 16-bit number of every element, in numpy: the calls' words, then each column's half of one."""
    m32, s32 = np.uint64(0xFFFFFFFF), np.uint64(32)
    calls = -(-cols // 8)
    x = [np.tile(np.arange(calls, dtype=np.uint64), rows), np.repeat(np.arange(rows, dtype=np.uint64), calls),
         np.full(rows * calls, offset & 0xFFFFFFFF, np.uint64), np.full(rows * calls, offset >> 32, np.uint64)]
    key = [seed & 0xFFFFFFFF, seed >> 32]
    for r in range(10):
        a, b = np.uint64(0xD2511F53) * x[0], np.uint64(0xCD9E8D57) * x[2]
        x = [(b >> s32) ^ x[1] ^ np.uint64(key[0]), b & m32, (a >> s32) ^ x[3] ^ np.uint64(key[1]), a & m32]
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    found = np.empty((rows, calls, 8), np.int64)
    for n in range(8):
        found[:, :, n] = (x[n // 2] >> np.uint64(16 * (n % 2)) & np.uint64(0xFFFF)).reshape(rows, calls)
    return found.reshape(rows, 8 * calls)[:, :cols]


def exact(case, seed):
    s, c = prepare(case, seed), case
    kind, rows = c["kind"], c["rows"]
    wide = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    get = wide.get

    def dropped(v):
        if c["drop"] == 0:
            return v
        t = round(c["drop"] * 65536)
        kept = torch.from_numpy(_numbers(rows, v.shape[1], s["seed"], s["offset"]) >= t).to(DEVICE)
        return torch.where(kept, v * (65536 / (65536 - t)), torch.zeros_like(v))

    def act(z):
        return {LINEAR: lambda: z, SIGMOID: lambda: torch.sigmoid(z), TANH: lambda: torch.tanh(z),
                RELU: lambda: torch.clamp(z, min=0), SILU: lambda: z * torch.sigmoid(z),
                GELU: lambda: z * torch.special.ndtr(z)}[c["act"]]()

    def norm(v, how, w, b):
        if how == NONE:
            return v
        if how == LAYER:
            return (v - v.mean(1, True)) / torch.sqrt(v.var(1, keepdim=True, unbiased=False) + EPS) * w + b
        return v / torch.sqrt(v.square().mean(1, keepdim=True) + EPS) * w

    def add(v, k):
        return v if get(k) is None else v + wide[k]

    if kind == "drop":
        return {"Y": dropped(wide["X"])}
    if kind == "lin_fwd":
        z = add(torch.matmul(wide["X"], wide["W"].T), "bias")
        return {"Y": add(dropped(act(z)), "R"), **({"Z": z} if c["keep"] else {})}
    if kind == "lin_bwd":
        z = wide["Z"].requires_grad_()
        delta, = torch.autograd.grad(dropped(act(z)), z, wide["dY"])
        return {"dX": torch.matmul(delta, wide["W"]), "dW": torch.matmul(delta.T, wide["X"]),
                **({"dbias": delta.sum(0)} if c["bias"] else {})}
    if kind == "ffn_fwd":
        g, u = (add(torch.matmul(wide["X"], wide["W" + k].T), "b" + k) for k in "gu")
        y = add(dropped(add(torch.matmul(act(g) * u, wide["Wd"].T), "bd")), "R")
        return {"Y": y, **({"GU": torch.hstack((g, u))} if c["keep"] else {})}
    if kind == "ffn_bwd":
        g, u = (v.clone().requires_grad_() for v in wide["GU"].chunk(2, 1))
        h, dz = act(g) * u, dropped(wide["dY"])
        dg, du = torch.autograd.grad(h, (g, u), torch.matmul(dz, wide["Wd"]))
        r = {"dX": torch.matmul(dg, wide["Wg"]).addmm_(du, wide["Wu"]), "dWg": torch.matmul(dg.T, wide["X"]),
             "dWu": torch.matmul(du.T, wide["X"]), "dWd": torch.matmul(dz.T, h.detach())}
        return {**r, **({"dbg": dg.sum(0), "dbu": du.sum(0), "dbd": dz.sum(0)} if c["bias"] else {})}
    names = [k for k in ("x", "b", "gate", "post_w", "post_b", "pre_w", "pre_b") if k in wide]
    if kind == "norm_bwd":
        for k in names:
            wide[k].requires_grad_()
    gate = wide["gate"].repeat_interleave(c["group"], 0)[:rows]
    step = c["scale"] * gate * norm(wide["b"], c["post"], get("post_w"), get("post_b"))
    if kind == "norm_fwd":
        x = wide["x"] + step
        return {"x_out": x, "n_out": norm(x, c["pre"], get("pre_w"), get("pre_b"))}
    # backward is given x' itself: its own gradient first, which then goes on to the step that was added
    n = norm(wide["x"], c["pre"], get("pre_w"), get("pre_b"))
    first = [k for k in names if k in ("x", "pre_w", "pre_b")]
    r = dict(zip(first, torch.autograd.grad(n, [wide[k] for k in first], wide["dn"])))
    r["x"] = r["x"] + wide["dx_out"]
    then = [k for k in names if k not in first]
    r.update(zip(then, torch.autograd.grad(step, [wide[k] for k in then], r["x"])))
    return {"d" + k: v for k, v in r.items()}
