"""Sizes that a launch could not hold are refused before anything is launched (no GPU needed)."""
import ctypes as C

import pytest

from paper_2001_04206_amd import dn
from test_ffn_abi import A, BAD, ffn, linear

FITS = [(1 << 28, 8), ((1 << 29) - 64, 8), (1 << 20, 1 << 12)]
TOO_MANY = [(1 << 29, 8), (0x7fffffff, 1), (1 << 25, 1 << 10), (1 << 15, 1 << 20)]


@pytest.mark.parametrize("rows,cols", TOO_MANY)
def test_too_many(rows, cols):
    lib, at = dn.lib(), C.addressof
    for d in (linear(rows=rows, n_in=cols, n_out=8), linear(rows=rows, n_in=8, n_out=cols)):
        assert lib.dn_linear_forward_workspace_bytes(at(d)) == BAD and lib.dn_linear_backward_workspace_bytes(at(d)) == BAD
        assert lib.dn_linear_forward(at(d), A, A, A, A, A, A, A, BAD - 1, None) == dn.DN_ERR_SHAPE
    d = ffn(rows=rows, d=cols, f=8)
    assert lib.dn_ffn_forward_workspace_bytes(at(d)) == BAD and lib.dn_ffn_backward_workspace_bytes(at(d)) == BAD
    assert lib.dn_dropout(dn.DN_BF16, A, A, rows, cols, 0, 0, 0.5, 1, 2, None) == dn.DN_ERR_SHAPE


def test_wide_weights_are_refused_too():
    d = linear(n_in=1 << 20, n_out=1 << 20)
    assert dn.lib().dn_linear_forward_workspace_bytes(C.addressof(d)) == BAD


@pytest.mark.parametrize("rows,cols", FITS)
def test_large_ones_are_not(rows, cols):
    d = linear(rows=rows, n_in=cols, n_out=8)
    need = dn.lib().dn_linear_backward_workspace_bytes(C.addressof(d))
    assert rows * 8 * 2 <= need < BAD
