"""The shapes of test_gpu_experts_kernels.py reach every kernel that the library's own rules take over a wide sample of sizes, so that a
change of a rule cannot leave one untested; and launches stay within what a device takes (no GPU: tests/fake_experts.cpp stands in)."""
import random

import pytest

import test_gpu_experts_kernels as gpu
from block_launches import TYPE, sizes
from experts_launches import ask, compile_program, kernels
from paper_2001_04206_amd import dn


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    return compile_program(tmp_path_factory.mktemp("fake_experts"))


def sample(kind, n, seed):
    rng, out = random.Random(seed), []
    while len(out) < n:
        e = sizes(rng, 1, 200)
        k, r = rng.randint(1, min(8, e)), sizes(rng, rng.choice((1, 17, 65, 1000)), 12000)
        d, f = sizes(rng, 1, 5000), sizes(rng, 1, 5000)
        if e * d * f <= 2 ** 27 and r * k * d * f <= 2 ** 37:
            out.append(("experts", kind, r, e, k, d, f, rng.choice((0, 0, 4, 16))))
    return out


@pytest.mark.parametrize("kind", TYPE)
def test_every_product(exe, kind):
    bits = 32 if kind == "f32" else 16
    mine = set().union(*kernels(exe, [("experts", kind) + s + (0,) for s in gpu.EXPERTS[bits]]))
    cases = sample(kind, 8000, 5)
    missing = {k: c for c, found in zip(cases, kernels(exe, cases)) for k in found if k not in mine}
    assert not missing, missing
    tiles = {k[2] for k in mine if len(k) == 5}
    assert tiles == ({"small", "tiny"} if bits == 32 else {"small", "medium", "large"})
    assert {k[1] for k in mine if len(k) == 5} == {"gated", "store", "dexpert"} | ({"pair"} if bits == 16 else set())


@pytest.mark.parametrize("kind", TYPE)
def test_every_routing(exe, kind):
    mine = set().union(*kernels(exe, [("route", kind) + s + (0,) for s in gpu.ROUTE]))
    rng, cases = random.Random(6), []
    while len(cases) < 3000:
        g = rng.choice((1, 1, 4, 8))
        e = g * rng.randint(1, 1024 // g)
        k = rng.randint(1, min(32, max(1, e // 2)))
        cases.append(("route", kind, sizes(rng, 1, 20000), e, k, rng.randint(0, 1), g, 0))
    missing = {k: c for c, found in zip(cases, kernels(exe, cases)) for k in found if k not in mine}
    assert not missing, missing


def test_sizes_at_the_limits(exe):
    """The largest calls are launched whole, the next larger ones refused: nothing fails in a launch."""
    ok = [("experts", "bf16", (1 << 24) // 8 - 1, 64, 8, 64, 64, 0), ("experts", "f32", 1 << 20, 1024, 15, 256, 64, 0), ("experts", "bf16", 1, 1024, 32, 1, 1, 0),
          ("experts", "f16", 3, 1, 32, 131072, 8, 0), ("experts", "f32", 5, 1024, 2, 8, 65536, 0), ("experts", "bf16", 100000, 2, 2, 4096, 8192, 0),
          ("route", "f32", (1 << 25) - 1, 64, 8, 1, 8, 0), ("route", "bf16", (1 << 25) - 1, 1024, 31, 0, 1, 0), ("clip", "f32", 3, 2000000000, 1, 0, 0, 0)]
    for call, passes in zip(ok, ask(exe, ok)):
        for status, launches in passes:
            assert status == dn.DN_OK and launches, (call, status)
            for name, x, y, threads in launches:
                assert 0 < x * threads < 1 << 32 and 0 < y < 1 << 16, (call, name, x, y, threads)
    rng = random.Random(8)
    wild = [("experts", rng.choice(list(TYPE)), sizes(rng, 1, 1 << 26), sizes(rng, 1, 1100), rng.randint(1, 32), sizes(rng, 1, 1 << 21), sizes(rng, 1, 1 << 21), 0)
            for _ in range(4000)]
    statuses = set()
    for call, passes in zip(wild, ask(exe, wild)):
        for status, launches in passes:
            statuses.add(status)
            assert status in (dn.DN_OK, dn.DN_ERR_SHAPE), (call, status)
            assert (status == dn.DN_OK) == bool(launches), call
            for name, x, y, threads in launches:
                assert 0 < x * threads < 1 << 32 and 0 < y < 1 << 16, (call, name, x, y, threads)
    assert statuses == {dn.DN_OK, dn.DN_ERR_SHAPE}
