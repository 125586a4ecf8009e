"""A copy to 16-byte rows that takes several launches: 1100001 rows of 15629 (34 GB, and as much for the copy in the workspace)."""
import pytest
import torch

from ffn_util import DEV, close, tolerance
from paper_2001_04206_amd import dn
from parity_util import announce
from test_gpu_ffn_long import BF16, filled

pytestmark = pytest.mark.gpu


def test_rows_on_both_sides_of_a_launch():
    rows, n, m = 1100001, 15629, 8
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("needs 80 GB of device memory")
    announce("copy in several launches")
    X, W = filled(rows, n, 1), (torch.randn(m, n, device=DEV) * n ** -0.5).to(BF16)
    Y = torch.full((rows, m), float("nan"), dtype=BF16, device=DEV)
    dn.dn_linear_forward(X, W, None, None, Y)
    first = (1 << 31) // -(-n // 8)      # the row in which the second launch begins
    at = torch.tensor([0, 1, 65536, first - 1, first, first + 1, rows - 2, rows - 1], device=DEV)
    close(Y[at], X[at].double() @ W.double().t(), tolerance(BF16, n), "Y")
    del X
    torch.cuda.empty_cache()
