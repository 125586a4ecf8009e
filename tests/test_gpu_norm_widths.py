"""dn_norm_* at both sides of every width at which another kernel begins, and of more rows than workgroups run at once, so that one takes
several rows with the next one's loads under way.  The cases and tolerances are test_gpu_norm.py's."""
import pytest

import test_gpu_norm
from ffn_util import TYPES

pytestmark = pytest.mark.gpu

# rows, d, rows of a gate: three (a workgroup takes whole gates) and ten (a gate's rows are divided, and the last one is short)
WIDTHS = [(37, d, per) for d in (512, 513, 1024, 1025, 1536, 1537, 2048, 2049, 3071, 3073, 4096, 4097, 8192, 8193, 16383) for per in (3, 10)]
MANY = [(9001, 509, 2), (9001, 509, 1700), (6001, 1021, 2), (6001, 1021, 1700), (3001, 1400, 1), (3001, 1400, 3001), (3001, 2041, 3), (3001, 2041, 700),
        (2001, 2600, 1), (2001, 2600, 900), (1501, 4093, 4), (1501, 4093, 400), (1301, 5003, 2), (1301, 5003, 500), (701, 9001, 1), (701, 9001, 300)]


@pytest.mark.parametrize("shape", WIDTHS + MANY, ids=str)
@pytest.mark.parametrize("kind", TYPES)
def test_forward(kind, shape):
    test_gpu_norm.test_forward(kind, shape)


@pytest.mark.parametrize("shape", WIDTHS + MANY, ids=str)
@pytest.mark.parametrize("kind", TYPES)
def test_backward(kind, shape):
    test_gpu_norm.test_backward(kind, shape, f32_grads=kind != "f16")
