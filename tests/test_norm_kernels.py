"""The shapes of test_gpu_norm_widths.py reach every kernel of the norms that a wide sample of sizes does (no GPU: tests/fake_block.cpp
stands in for the device)."""
import random

import pytest

import test_gpu_norm_widths as gpu
from block_launches import TYPE, compile_program, kernels, sizes


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    return compile_program(tmp_path_factory.mktemp("fake_block"))


@pytest.mark.parametrize("kind", TYPE)
def test_every_norm(exe, kind):
    mine = kernels(exe, [("norm", kind) + s + (0,) for s in gpu.WIDTHS + gpu.MANY])
    rng = random.Random(6)
    sample = [("norm", kind, sizes(rng, 1, 9000), sizes(rng, 1, 16384), sizes(rng, 1, 9000), 0) for _ in range(2000)]
    missing = {k: c for c, found in zip(sample, kernels(exe, sample)) for k in found if k not in set().union(*mine)}
    assert not missing, missing
