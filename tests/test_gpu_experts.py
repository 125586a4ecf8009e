"""A block of experts on the GPU, forward and backward, against 64 bits."""
import math

import pytest
import torch

import experts_util as ex
from ffn_util import ACTS, DEV, TYPES, UNIT, Make, close, tolerance
from paper_2001_04206_amd import dn

pytestmark = pytest.mark.gpu


def table(rows, experts, k, seed, none=0.0, hot=None):
    """Choices and weights of every row: k different experts (all rows on the first `hot` ones), a share of them none."""
    g = torch.Generator().manual_seed(seed)
    score = torch.randn(rows, experts, generator=g)
    if hot:
        score[:, hot:] -= 100.0
    expert = score.topk(k, 1).indices.int()
    expert[torch.rand(rows, k, generator=g) < none] = -1
    weight = torch.rand(rows, k, generator=g) + 0.1
    weight[expert < 0] = 0.0
    return expert.to(DEV), weight.to(DEV)


class Case:
    def __init__(self, dtype, rows, experts, k, d, f, seed=1, none=0.0, hot=None, pad=0, act="silu", res=True):
        self.dtype, self.act, self.shape = dtype, act, (rows, experts, k, d, f)
        make = self.make = Make(dtype, seed)
        self.expert, self.weight = table(rows, experts, k, seed, none, hot)
        self.starts, self.order, self.place = (torch.empty(n, dtype=torch.int32, device=DEV) for n in (experts + 1, rows * k, rows * k))
        dn.dn_route_lists(self.expert, self.starts, self.order, self.place)
        self.X, self.R = make(rows, d, pad=pad), make(rows, d, pad=pad) if res else None
        self.Wg, self.Wu = (make(experts, f, d, std=d ** -0.5) for _ in range(2))
        self.Wd = make(experts, d, f, std=f ** -0.5)
        self.dY = make(rows, d, pad=pad)
        self.lists = (self.weight, self.starts, self.order, self.place)

    def forward(self, keep=True, pad=0, workspace=None):
        rows, experts, k, d, f = self.shape
        Y = self.make.out(rows, d + pad)[:, :d]
        GU = self.make.out(rows * k, 2 * f) if keep else None
        dn.dn_experts_forward(self.X, self.Wg, self.Wu, self.Wd, *self.lists, self.R, Y, GU, act=ACTS[self.act], workspace=workspace)
        return Y, GU

    def by_pair(self, GU):
        """G and U [rows][k][f] of what was kept by place; zeros for pairs without an expert."""
        rows, experts, k, d, f = self.shape
        place = self.place.cpu().long()
        gu = torch.where((place >= 0)[:, None], GU.cpu()[place.clamp(min=0)].double(), 0.0).view(rows, k, 2 * f)
        return gu[..., :f], gu[..., f:]

    def backward(self, GU, grad_dtype=None, grad_scale=1.0, dX=True, dweight=True, workspace=None):
        rows, experts, k, d, f = self.shape
        out = lambda *s, t=None: self.make.out(*s, dtype=t)
        g = {"dX": out(rows, d) if dX else None, "dWg": out(experts, f, d, t=grad_dtype), "dWu": out(experts, f, d, t=grad_dtype),
             "dWd": out(experts, d, f, t=grad_dtype), "dweight": out(rows, k, t=torch.float32) if dweight else None}
        dn.dn_experts_backward(self.X, self.Wg, self.Wu, self.Wd, *self.lists, GU, self.dY, g["dX"], g["dWg"], g["dWu"], g["dWd"], g["dweight"],
                               act=ACTS[self.act], grad_scale=grad_scale, workspace=workspace)
        return g

    def check_forward(self, Y, GU):
        """H and z are rounded once each before Y is: three roundings where nothing hides them, and G and U one."""
        rows, experts, k, d, f = self.shape
        want, G, U = ex.forward64(self.X, self.Wg, self.Wu, self.Wd, self.weight, self.expert, self.R, self.act)
        close(Y, want, tolerance(self.dtype, d + f, 3), "Y")
        if GU is not None:
            n = int(self.starts[-1])
            assert GU[n:].isnan().all(), "rows behind the last pair"
            if n:
                g, u = self.by_pair(GU)
                has = (self.expert >= 0).cpu()
                close(g[has], G[has], tolerance(self.dtype, d), "G")
                close(u[has], U[has], tolerance(self.dtype, d), "U")

    def check_backward(self, g, GU, grad_scale=1.0):
        """dG, dU and w H are rounded, then each result; dX also each pair's part.  dweight is fp32: sums of d and of f terms, and
        the 16-bit activations' 3e-7."""
        rows, experts, k, d, f = self.shape
        G, U = self.by_pair(GU)
        want = dict(zip(("dX", "dWg", "dWu", "dWd", "dweight"),
                        ex.backward64(self.X, self.Wg, self.Wu, self.Wd, self.weight, self.expert, G, U, self.dY, self.act, grad_scale)))
        if g["dX"] is not None:
            close(g["dX"], want["dX"], tolerance(self.dtype, d + 2 * f, 3), "dX")
        for n in ("dWg", "dWu", "dWd"):
            t = g[n].dtype
            tol = tolerance(self.dtype, rows * k + d, 1 + (t != torch.float32))
            close(g[n] / grad_scale, want[n] / grad_scale, tol, n)
            for e in range(experts):
                if not (self.expert == e).any():
                    assert (g[n][e] == 0).all(), "an expert without rows"
        if g["dweight"] is not None:
            assert (g["dweight"][self.expert < 0] == 0).all()
            close(g["dweight"], want["dweight"], 2.0 ** -24 * (d ** 0.5 + f ** 0.5 + 16) + (0 if self.dtype == torch.float32 else 3e-7), "dweight")

    def check(self):
        Y, GU = self.forward()
        self.check_forward(Y, GU)
        GU = torch.where(GU.isnan(), torch.zeros_like(GU), GU)
        self.check_backward(self.backward(GU), GU)


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("rows,experts,k,d,f", [
    (1, 1, 1, 64, 64), (1, 8, 2, 64, 48), (1, 64, 8, 256, 96), (2, 5, 3, 40, 24), (7, 4, 4, 33, 17), (17, 3, 1, 8, 8),
    (37, 16, 2, 101, 55), (130, 2, 1, 128, 256), (300, 4, 2, 264, 130), (65, 7, 3, 512, 129), (1000, 70, 5, 72, 40)])
def test_shapes(name, rows, experts, k, d, f):
    """Experts of one row and of many, odd widths that make the calls copy their matrices, more than 64 experts."""
    Case(TYPES[name], rows, experts, k, d, f, seed=rows + d).check()


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("rows,experts,k,d,f", [(700, 2, 2, 320, 192), (2048, 4, 2, 256, 512), (1500, 3, 2, 1024, 520)])
def test_tiles(name, rows, experts, k, d, f):
    """Enough rows an expert for every size of tile, several of them, with last ones that end inside."""
    Case(TYPES[name], rows, experts, k, d, f, seed=rows).check()


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("rows", [959, 960, 961, 1919, 1920, 1921, 3841, 5000])
def test_long_runs(name, rows):
    """Experts with more rows than a workgroup of the matrices' gradients looks up at a time (960 in fp32, 1920 in 16 bits), to a row."""
    Case(TYPES[name], rows, 2, 2, 24, 40, seed=rows, pad=rows % 3).check()


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("act", ACTS)
def test_activations(name, act):
    Case(TYPES[name], 50, 4, 2, 96, 80, act=act, seed=7).check()


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("rows,d,f", [(3, 64, 40), (200, 96, 264), (90, 51, 33)])
def test_none_hot_and_empty(name, rows, d, f):
    """Pairs without an expert, experts without a row (their gradients are zeros), all rows on two experts, nothing at all; rows of X, R
    and Y apart; no residual."""
    Case(TYPES[name], rows, 6, 3, d, f, none=0.4, pad=5, seed=2).check()
    Case(TYPES[name], rows, 9, 2, d, f, hot=2, pad=8, seed=3, res=False).check()
    c = Case(TYPES[name], rows, 4, 2, d, f, none=1.1, seed=4)
    Y, GU = c.forward(pad=3)
    assert torch.equal(Y, c.R) and GU.isnan().all()
    g = c.backward(torch.zeros_like(GU))
    assert all((g[n] == 0).all() for n in g)
    c.R = None
    assert (c.forward(keep=False)[0] == 0).all()


@pytest.mark.parametrize("name", ["f16", "bf16"])
def test_gradients_in_fp32(name):
    c = Case(TYPES[name], 120, 5, 2, 72, 136, seed=5)
    _, GU = c.forward()
    c.check_backward(c.backward(GU, grad_dtype=torch.float32, grad_scale=0.25), GU, 0.25)
    whole = c.backward(GU)
    part = c.backward(GU, dX=False, dweight=False)
    assert all(torch.equal(whole[n], part[n]) for n in ("dWg", "dWu", "dWd"))


def test_gradients_against_differences():
    """dE of E = sum of dY * Y along a random direction of every input, fp32, from forward calls at both sides.  Steps of 2^-6 of inputs of
    size 1: the third derivative leaves about 2^-12, the sums' rounding 2^-24 sqrt(terms) of E over the step; 2e-3 of each is allowed."""
    c = Case(torch.float32, 9, 4, 2, 24, 20, seed=6, act="gelu")
    _, GU = c.forward()
    g = c.backward(GU)

    def E():
        return (c.dY.double() * c.forward()[0].double()).sum().item()

    for name, t, grad in (("X", c.X, g["dX"]), ("Wg", c.Wg, g["dWg"]), ("Wu", c.Wu, g["dWu"]), ("Wd", c.Wd, g["dWd"]), ("weight", c.weight, g["dweight"])):
        v = torch.randn(t.shape, generator=torch.Generator().manual_seed(3)).to(DEV) * (1.0 if name in ("X", "weight") else 0.2)
        before, step = t.clone(), 2.0 ** -6
        t.copy_(before + step * v)
        up = E()
        t.copy_(before - step * v)
        down = E()
        t.copy_(before)
        want, got = (up - down) / (2 * step), (grad.double() * v.double()).sum().item()
        scale = (grad.double() * v.double()).norm().item()
        assert abs(got - want) <= 2e-3 * max(scale, 1.0), (name, got, want)


def test_against_the_dense_block():
    """One expert that every row takes with weight 1 is the gated block: the same G and U, and Y within the roundings of z."""
    for dtype in TYPES.values():
        c = Case(dtype, 200, 1, 1, 128, 192, seed=8)
        c.weight.fill_(1.0)
        Y, GU = c.forward()
        dense, kept = torch.empty_like(Y), torch.empty_like(GU)
        dn.dn_ffn_forward(c.X, c.Wg[0], None, c.Wu[0], None, c.Wd[0], None, c.R, dense, kept, act=ACTS["silu"])
        close(GU, kept.double(), 2 * tolerance(dtype, 128), "GU")
        close(Y, dense.double(), tolerance(dtype, 320, 4), "Y")


def test_the_same_bits_and_other_rows():
    """The same call gives the same bits; a row's result does not depend on what other rows hold, NaN and infinities among them."""
    for name, dtype in TYPES.items():
        for rows in (5, 400):
            c = Case(dtype, rows, 6, 2, 64, 72, seed=9)
            Y, GU = c.forward()
            again, _ = c.forward()
            assert torch.equal(Y, again)
            g, h = c.backward(GU), c.backward(GU)
            assert all(torch.equal(g[n], h[n]) for n in g)
            c.X[1] = math.nan
            c.X[3] = math.inf
            bad, _ = c.forward()
            keep = [i for i in range(rows) if i not in (1, 3)]
            assert torch.equal(bad[keep], Y[keep]) and bad[1].isnan().all()


def test_the_residual_itself():
    """Y may be R, and both X: every row is read before it is written."""
    for name, dtype in TYPES.items():
        for rows in (2, 30, 700):
            c = Case(dtype, rows, 6, 2, 64, 72, seed=11)
            Y, _ = c.forward()
            R = c.R.clone()
            dn.dn_experts_forward(c.X, c.Wg, c.Wu, c.Wd, *c.lists, R, R)
            assert torch.equal(R, Y)
            c.R = c.X
            Y, _ = c.forward()
            X = c.X.clone()
            dn.dn_experts_forward(X, c.Wg, c.Wu, c.Wd, *c.lists, X, X)
            assert torch.equal(X, Y)


def test_lists_that_are_wrong_stay_inside():
    """Numbers out of range in the lists: no access outside the tensors (what is computed has no meaning), and the next call is right."""
    for rows in (4, 300):
        c = Case(torch.bfloat16, rows, 5, 2, 64, 64, seed=10)
        good, GU = c.forward()
        n = rows * 2
        for starts, order, place in (([0, 5 * n, -7, 2 ** 31 - 1, 3, 9 * n], 2 ** 31 - 1, 2 ** 31 - 1), ([-5] * 6, -2 ** 31, -2 ** 31),
                                     ([9 * n] * 6, n, n), ([n, 0, n, 0, n, 0], -1, 0)):
            lists = (c.weight, torch.tensor(starts, dtype=torch.int32, device=DEV), torch.full((n,), order, dtype=torch.int32, device=DEV),
                     torch.full((n,), place, dtype=torch.int32, device=DEV))
            keep, c.lists = c.lists, lists
            c.forward()
            c.backward(GU)
            c.lists = keep
        assert torch.equal(c.forward()[0], good)


WHERE = [(3, 6, 1, 40, 24), (5, 6, 2, 72, 40), (60, 7, 2, 33, 17), (400, 6, 2, 72, 136), (700, 8, 1, 264, 130), (2500, 5, 2, 328, 200), (2048, 4, 1, 64, 264)]


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("rows,experts,k,d,f", WHERE)
def test_the_weights_derivatives_alone(name, rows, experts, k, d, f):
    """Without dX they come from a launch of their own, and are the same; so are the matrices' gradients."""
    c = Case(TYPES[name], rows, experts, k, d, f, none=0.2, seed=12)
    _, GU = c.forward()
    GU = torch.where(GU.isnan(), torch.zeros_like(GU), GU)
    whole, alone, rest = c.backward(GU), c.backward(GU, dX=False), c.backward(GU, dweight=False)
    c.check_backward(alone, GU)
    assert all(torch.equal(whole[n], alone[n]) for n in alone if n != "dX")
    assert all(torch.equal(whole[n], rest[n]) for n in rest if n != "dweight")


def filled():
    return torch.full((64 << 20,), 255, dtype=torch.uint8, device=DEV)


@pytest.mark.parametrize("what", ["NaN", "inf"])
@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("rows,experts,k,d,f", WHERE)
def test_what_one_row_holds_stays_with_it(name, what, rows, experts, k, d, f):
    """A row's NaN or infinity in X, dY or its G and U reaches its own results and its experts' gradients, and no bit of others; a row without
    an expert reaches nothing, nor do the places behind the last pair.  In workspaces whose every byte is FF."""
    c = Case(TYPES[name], rows, experts, k, d, f, none=0.3, seed=13)
    c.expert[rows // 2], c.weight[rows // 2] = -1, 0.0
    dn.dn_route_lists(c.expert, c.starts, c.order, c.place)
    Y, GU = c.forward(workspace=filled())
    c.check_forward(Y, GU)
    clean = c.backward(torch.where(GU.isnan(), torch.zeros_like(GU), GU))
    dirty = c.backward(GU, workspace=filled())
    assert all(torch.equal(clean[n], dirty[n]) for n in clean), "places behind the last pair"
    value = math.nan if what == "NaN" else math.inf
    X, dY = c.X.clone(), c.dY.clone()
    for t in (rows // 2, 0, rows - 1):
        mine = [int(e) for e in c.expert[t] if e >= 0]
        others = [e for e in range(experts) if e not in mine]
        left = [i for i in range(rows) if i != t]
        c.X[t], c.dY[t] = value, value
        spoilt = GU.clone()
        for p in c.place.view(rows, k)[t].tolist():
            if p >= 0:
                spoilt[p] = value
        y, _ = c.forward(workspace=filled())
        g = c.backward(spoilt, workspace=filled())
        assert torch.equal(y[left], Y[left])
        assert torch.equal(g["dX"][left], clean["dX"][left]) and torch.equal(g["dweight"][left], clean["dweight"][left])
        for n in ("dWg", "dWu", "dWd"):
            assert torch.equal(g[n][others], clean[n][others]), n
        if not mine:
            assert torch.equal(y, Y) and all(torch.equal(g[n], clean[n]) for n in g)
        c.X.copy_(X)
        c.dY.copy_(dY)


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("rows,experts,k,d,f", WHERE)
def test_what_one_expert_holds_stays_with_it(name, rows, experts, k, d, f):
    """NaN in an expert's matrices reaches the rows that chose it, and no bit of others."""
    c = Case(TYPES[name], rows, experts, k, d, f, none=0.1, seed=14)
    Y, GU = c.forward()
    GU = torch.where(GU.isnan(), torch.zeros_like(GU), GU)
    clean = c.backward(GU)
    for e in (0, experts // 2, experts - 1):
        W = [w[e].clone() for w in (c.Wg, c.Wu, c.Wd)]
        for w in (c.Wg, c.Wu, c.Wd):
            w[e] = math.nan
        y, _ = c.forward()
        g = c.backward(GU)
        for w, was in zip((c.Wg, c.Wu, c.Wd), W):
            w[e] = was
        off = (c.expert == e).any(1)
        assert torch.equal(y[~off], Y[~off]) and y[off].isnan().all()
        assert torch.equal(g["dX"][~off], clean["dX"][~off]) and g["dX"][off].isnan().all()
        assert torch.equal(g["dweight"][c.expert != e], clean["dweight"][c.expert != e])
        others = [i for i in range(experts) if i != e]
        assert all(torch.equal(g[n][others], clean[n][others]) for n in ("dWg", "dWu", "dWd"))


@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("rows,d,f", [(2, 40, 24), (9, 33, 17), (300, 72, 136), (1500, 264, 130)])
def test_the_same_expert_twice(name, rows, d, f):
    """A row that names an expert more than once has its output with each of the weights, and a gradient for each."""
    c = Case(TYPES[name], rows, 4, 3, d, f, seed=15)
    c.expert[::2, 1] = c.expert[::2, 0]
    c.expert[::3] = c.expert[::3, :1]
    _, starts, order, place = c.lists
    dn.dn_route_lists(c.expert, starts, order, place)
    c.check()
