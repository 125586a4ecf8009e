"""A norm's weight where there is no norm takes no part: dn_norm_* then give, bit for bit, what they give without it."""
import pytest
import torch

from ffn_util import TYPES, Make, close, tolerance
from paper_2001_04206_amd import dn
from parity_util import announce

pytestmark = pytest.mark.gpu
NONE, RMS = dn.DN_NORM_NONE, dn.DN_NORM_RMS


# rows a gate: one, a few (a workgroup takes whole gates), all of many (a gate's rows are divided)
@pytest.mark.parametrize("per", [1, 3, 600])
@pytest.mark.parametrize("kind", TYPES)
def test_block_without_a_norm(kind, per):
    announce("norm weights without a norm %s %d" % (kind, per))
    dtype, rows, d = TYPES[kind], 600, 72
    make = Make(dtype, 11)
    x, b, gate, w, pre_w = make(rows, d), make(rows, d), make(rows // per, d, mean=1.0), make(d, mean=2.0), make(d, mean=1.0)
    dx_out, dnorm = make(rows, d), make(rows, d)
    found = []
    for post_w in (None, w):
        x_out, n_out, dx, db = (make.out(rows, d) for _ in range(4))
        dgate = make.out(rows // per, d, dtype=torch.float32)
        dn.dn_norm_forward(x, b, gate, post_w, None, pre_w, None, x_out, n_out, post=NONE, pre=RMS, scale=0.5, rows_per_gate=per)
        dn.dn_norm_backward(x_out, b, gate, post_w, None, pre_w, dx_out, dnorm, dx, db, dgate, None, None, None, None, post=NONE, pre=RMS,
                            scale=0.5, rows_per_gate=per)
        found.append((x_out, n_out, dx, db, dgate))
    for name, a, c in zip(("x_out", "n_out", "dx", "db", "dgate"), *found):
        assert torch.equal(a, c), name
    x_out, _, dx, _, dgate = found[1]
    # dx as it was stored carries one rounding of its type into every term
    want = (0.5 * dx.double() * b.double()).view(rows // per, per, d).sum(1)
    close(dgate, want, 2 * tolerance(dtype, per), "dgate")


@pytest.mark.parametrize("kind", TYPES)
def test_nothing_before_the_next_block(kind):
    announce("norm weights before no norm %s" % kind)
    dtype, rows, d = TYPES[kind], 37, 520
    make = Make(dtype, 12)
    x, b, post_w, w, dx_out = make(rows, d), make(rows, d), make(d, mean=1.0), make(d, mean=2.0), make(rows, d)
    found = []
    for pre_w in (None, w):
        x_out, dx, db, dpost = (make.out(*s) for s in ((rows, d),) * 3 + ((d,),))
        dn.dn_norm_forward(x, b, None, post_w, None, pre_w, None, x_out, None, post=RMS, pre=NONE)
        dn.dn_norm_backward(x_out, b, None, post_w, None, pre_w, dx_out, None, dx, db, None, dpost, None, None, None, post=RMS, pre=NONE)
        found.append((x_out, dx, db, dpost))
    for name, a, c in zip(("x_out", "dx", "db", "dpost_w"), *found):
        assert torch.equal(a, c), name
