"""The shapes of test_gpu_block_kernels.py reach every kernel that the library's own rule takes over a wide sample of sizes, so that a
change of the rule cannot leave one untested (no GPU: tests/fake_block.cpp stands in for the device)."""
import random

import pytest

import test_gpu_block_kernels as gpu
from block_launches import TYPE, compile_program, kernels, sizes


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    return compile_program(tmp_path_factory.mktemp("fake_block"))


@pytest.mark.parametrize("kind", TYPE)
def test_every_product(exe, kind):
    bits = 32 if kind == "f32" else 16
    mine = kernels(exe, [("linear", kind) + s + (0,) for s in gpu.LINEAR[bits]] + [("block", kind) + s + (0,) for s in gpu.BLOCK[bits]])
    rng = random.Random(5)
    sample = [(rng.choice(("linear", "block")), kind, sizes(rng, rng.choice((1, 17, 65)), 9000), sizes(rng, 8, 9000), sizes(rng, 8, 9000), 0)
              for _ in range(8000)]
    missing = {k: c for c, found in zip(sample, kernels(exe, sample)) for k in found if k not in set().union(*mine)}
    assert not missing, missing
    tiles = {k[3] for found in mine for k in found if len(k) == 7}
    assert tiles == ({"small", "tiny"} if bits == 32 else {"small", "medium", "large"})
