"""Clipping by the norm of many tensors on the GPU, against 64 bits."""
import math

import pytest
import torch

from ffn_util import DEV, TYPES, UNIT
from paper_2001_04206_amd import dn

pytestmark = pytest.mark.gpu

SIZES = [[1], [7], [8, 1, 9], [8191, 8192, 8193], [100003], [0, 5, 0], [3] * 79, [5] * 80, [300] * 81, [257, 70000] * 100, [3000001, 2]]


def tensors(sizes, dtypes, seed):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(n, generator=g) * 10.0 ** (-(i % 3))).to(dtypes[i % len(dtypes)]).to(DEV) for i, n in enumerate(sizes)]


def norm64(grads):
    return math.sqrt(sum((t.double() ** 2).sum().item() for t in grads))


def check(grads, max_norm, outs, before):
    """The norm is rounded once (its sums are in 64 bits); a result is g times a rounded factor, rounded."""
    n = norm64(before)
    norm = torch.full((1,), math.nan, device=DEV)
    dn.dn_clip(grads, max_norm, norm, outs)
    assert abs(norm.item() - n) <= 1.01 * 2.0 ** -24 * n
    by = min(1.0, max_norm / n) if n else 1.0
    for g, b, o in zip(grads, before, grads if outs is None else outs):
        if o is None:
            assert torch.equal(g, b)
            continue
        want = b.double() * by
        small = {torch.float16: 2.0 ** -25}.get(o.dtype, 2.0 ** -140)
        assert ((o.double() - want).abs() <= (UNIT[o.dtype] + 2.0 ** -22) * want.abs() + small).all()
        if by == 1.0:
            assert torch.equal(o, b.to(o.dtype))
        if o is not g:
            assert torch.equal(g, b)


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "%dx%d" % (len(s), s[0]))
@pytest.mark.parametrize("names", [("f32",), ("f16",), ("bf16",), ("bf16", "f32", "f16")], ids="-".join)
def test_clip(sizes, names):
    """In place, into tensors of the type, into fp32; clipped, not clipped, and the norm only."""
    dtypes = [TYPES[n] for n in names]
    before = tensors(sizes, dtypes, len(sizes))
    n = norm64(before)
    for bound in (0.25 * n, 4 * n, 0.0):
        grads = [t.clone() for t in before]
        check(grads, bound, None, before)
        grads = [t.clone() for t in before]
        check(grads, bound, [torch.full_like(t, math.nan, dtype=torch.float32) for t in grads], before)
        check(grads, bound, [torch.full_like(t, math.nan) for t in grads], before)
    check(before, 0.25 * n, [None] * len(before), before)
    check(before, math.inf, None, [t.clone() for t in before])


def test_odd_places():
    """Tensors that begin anywhere in a buffer, results too; what lies between them stays."""
    for name, dtype in TYPES.items():
        for out in (dtype, torch.float32):
            buffer = torch.randn(50000, generator=torch.Generator().manual_seed(3)).to(dtype).to(DEV)
            result = torch.full((50000,), 7.0, dtype=out, device=DEV)
            cuts = [(1, 700), (703, 9000), (9001, 9002), (9005, 30011), (30012, 49999)]
            grads, outs = [buffer[a:b] for a, b in cuts], [result[a:b] for a, b in cuts]
            check(grads, 3.0, outs, [g.clone() for g in grads])
            inside = torch.zeros(50000, dtype=torch.bool, device=DEV)
            for a, b in cuts:
                inside[a:b] = True
            assert (result[~inside] == 7.0).all()
            whole = buffer.clone()
            dn.dn_clip(grads, 3.0, torch.empty(1, device=DEV))
            assert torch.equal(buffer[~inside], whole[~inside])


def test_large_and_small_numbers():
    """Squares beyond fp32's range at both ends; a norm beyond it whose factor is not."""
    for v in (1e30, 1e-30, 3e38):
        g = [torch.full((1000,), v, device=DEV), torch.full((3,), v, device=DEV)]
        before = [t.clone() for t in g]
        norm = torch.empty(1, device=DEV)
        n = norm64(before)
        dn.dn_clip(g, v, norm)
        assert math.isinf(norm.item()) if n > 3.4028235e38 else abs(norm.item() - n) <= 2.0 ** -23 * n
        for t, b in zip(g, before):
            want = b.double() * (v / n)
            assert ((t.double() - want).abs() <= 2.0 ** -22 * want).all()


def test_norms_that_are_not_finite():
    for bad in (math.nan, math.inf, -math.inf):
        g = [torch.randn(5000, device=DEV), torch.randn(70, device=DEV, dtype=torch.bfloat16)]
        g[0][4321] = bad
        before, norm, outs = [t.clone() for t in g], torch.empty(1, device=DEV), [torch.zeros(5000, device=DEV), torch.zeros(70, device=DEV)]
        dn.dn_clip(g, 1e-3, norm, outs)
        assert not math.isfinite(norm.item())
        for a, b, o in zip(g, before, outs):
            assert torch.equal(a.float().nan_to_num(0.5), b.float().nan_to_num(0.5)) and torch.equal(o.nan_to_num(0.5), b.float().nan_to_num(0.5))
        dn.dn_clip(g, 1e-3, norm)
        assert torch.equal(g[0].nan_to_num(0.5), before[0].nan_to_num(0.5))


def test_nothing_at_all():
    norm = torch.full((1,), math.nan, device=DEV)
    dn.dn_clip([], 1.0, norm)
    assert norm.item() == 0
    norm.fill_(math.nan)
    dn.dn_clip([torch.empty(0, device=DEV)], 1.0, norm)
    assert norm.item() == 0
    z = torch.zeros(9, device=DEV)
    dn.dn_clip([z], 0.0, norm)
    assert norm.item() == 0 and (z == 0).all()


def test_the_same_bits():
    a = tensors([100000, 3, 2000000, 77] * 30, [torch.bfloat16, torch.float32], 5)
    norm, again = torch.empty(1, device=DEV), torch.empty(1, device=DEV)
    b = [t.clone() for t in a]
    dn.dn_clip(a, 0.5, norm)
    dn.dn_clip(b, 0.5, again)
    assert torch.equal(norm, again) and all(torch.equal(x, y) for x, y in zip(a, b))


def test_results_that_overlap_are_refused():
    t = torch.randn(100, device=DEV)
    norm = torch.empty(1, device=DEV)
    before = t.clone()
    for grads, outs in (([t, t], None), ([t[:60], t[50:]], None), ([t[:50]], [t[1:51]]), ([t[:50], t[50:]], [t[50:], t[:50]])):
        with pytest.raises(dn.DnError) as e:
            dn.dn_clip(grads, 0.1, norm, outs)
        assert e.value.status == dn.DN_ERR_INVALID_ARG
    h = torch.randn(100, device=DEV).half()
    with pytest.raises(dn.DnError):
        dn.dn_clip([h[:50]], 0.1, norm, [h.view(torch.float32)])
    assert torch.equal(t, before)
    dn.dn_clip([t, t], math.inf, norm, [None, None])
    assert abs(norm.item() - norm64([t, t])) <= 2.0 ** -23 * norm64([t, t])
