"""Clipping of gradients so large that max_norm / n lies below the normal numbers of fp32, which results do not."""
import math

import pytest
import torch

from ffn_util import DEV, TYPES, UNIT
from paper_2001_04206_amd import dn
from test_gpu_clip import norm64

pytestmark = pytest.mark.gpu

# half of the smallest number of each type: what rounding may take from a result below its normal numbers
HALF = {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("max_norm", [1.0, 1e-3, 1e-6, 1e-20, 1e-37, 1e-44, 0.0])
@pytest.mark.parametrize("size", [1e38, 3e37, 1e30])
def test_small_factors(name, max_norm, size):
    """In place, into the type and into fp32: the product is rounded to fp32 (2^-24) and then to the type; where the factor is a normal number of fp32 it has
    been rounded, too."""
    g = torch.Generator().manual_seed(3)
    sizes = (1000, 8193, 3, 40000)
    before = [(torch.randn(n, generator=g).clamp(-3, 3) * size * 10.0 ** (-3 * (i % 2))).to(TYPES[name]).to(DEV) for i, n in enumerate(sizes)]
    n = norm64(before)
    norm = torch.full((1,), math.nan, device=DEV)
    for out in (None, TYPES[name], torch.float32):
        grads = [t.clone() for t in before]
        outs = None if out is None else [torch.full_like(t, math.nan, dtype=out) for t in grads]
        dn.dn_clip(grads, max_norm, norm, outs)
        assert math.isinf(norm.item()) if n >= 2.0 ** 128 else abs(norm.item() - n) <= 1.01 * 2.0 ** -24 * n
        for b, o in zip(before, grads if outs is None else outs):
            bound = torch.tensor(max_norm, dtype=torch.float32).double().item()     # what the call gets
            want = b.double() * (bound / n)
            off = (o.double() - want).abs()
            assert (off <= (UNIT[o.dtype] + 2.0 ** -22) * want.abs() + HALF[o.dtype] + HALF[torch.float32]).all(), (max_norm, size, off.max().item())
