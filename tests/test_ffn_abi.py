"""Host-side checks of the residual feed-forward block's calls that need no GPU: workspace queries and refusals, all before
anything is launched."""
import ctypes as C

import pytest

from paper_2001_04206_amd import dn

A = 0x10000           # an aligned address that no call below gets to
BAD = C.c_size_t(-1).value


@pytest.fixture(scope="module")
def lib():
    return dn.lib()


def linear(**kw):
    d = dict(type=dn.DN_BF16, grad_type=dn.DN_BF16, act=dn.DN_ACT_GELU, rows=100, n_in=64, n_out=48, ldx=0, ldw=0, ldr=0, ldy=0, drop=0.1,
             grad_scale=1.0, seed=1, offset=2)
    d.update(kw)
    return dn.LinearDesc(**d)


def ffn(**kw):
    d = dict(type=dn.DN_BF16, grad_type=dn.DN_F32, act=dn.DN_ACT_SILU, rows=100, d=64, f=48, ldx=0, ldr=0, ldy=0, drop=0.1, grad_scale=1.0,
             seed=1, offset=2)
    d.update(kw)
    return dn.FfnDesc(**d)


def norm(**kw):
    d = dict(type=dn.DN_F16, grad_type=dn.DN_F16, rows=100, d=64, post=dn.DN_NORM_RMS, pre=dn.DN_NORM_LAYER, rows_per_gate=100, scale=1.0, eps=1e-5)
    d.update(kw)
    return dn.NormDesc(**d)


WRONG = [({"type": 3}, dn.DN_ERR_INVALID_ARG), ({"type": dn.DN_F16, "grad_type": dn.DN_BF16}, dn.DN_ERR_INVALID_ARG),
         ({"act": -1}, dn.DN_ERR_INVALID_ARG), ({"act": 7}, dn.DN_ERR_INVALID_ARG), ({"act": dn.DN_ACT_SOFTMAX}, dn.DN_ERR_UNSUPPORTED),
         ({"rows": 0}, dn.DN_ERR_SHAPE), ({"rows": -5}, dn.DN_ERR_SHAPE), ({"ldx": 63}, dn.DN_ERR_SHAPE), ({"ldx": -64}, dn.DN_ERR_SHAPE),
         ({"ldx": 1 << 23}, dn.DN_ERR_SHAPE), ({"drop": 1.0}, dn.DN_ERR_INVALID_ARG), ({"drop": -0.1}, dn.DN_ERR_INVALID_ARG),
         ({"drop": float("nan")}, dn.DN_ERR_INVALID_ARG), ({"grad_scale": float("inf")}, dn.DN_ERR_INVALID_ARG)]


def test_linear_refuses(lib):
    at = C.addressof
    ok = linear()
    need = lib.dn_linear_backward_workspace_bytes(at(ok))
    assert 0 < need < BAD and need % 256 == 0 and need >= 100 * 48 * 2
    assert lib.dn_linear_forward_workspace_bytes(None) == BAD and lib.dn_linear_forward(None, A, A, A, A, A, A, A, 1 << 30, None) == dn.DN_ERR_INVALID_ARG
    for kw, status in WRONG + [({"n_in": 0}, dn.DN_ERR_SHAPE), ({"n_out": 0}, dn.DN_ERR_SHAPE), ({"n_out": 1 << 23}, dn.DN_ERR_SHAPE),
                               ({"ldw": 1}, dn.DN_ERR_SHAPE), ({"ldr": 1}, dn.DN_ERR_SHAPE), ({"ldy": 47}, dn.DN_ERR_SHAPE)]:
        d = linear(**kw)
        assert lib.dn_linear_forward_workspace_bytes(at(d)) == BAD and lib.dn_linear_backward_workspace_bytes(at(d)) == BAD, kw
        assert lib.dn_linear_forward(at(d), A, A, A, A, A, A, A, 1 << 30, None) == status, kw
        assert lib.dn_linear_backward(at(d), A, A, A, A, A, A, A, A, 1 << 30, None) == status, kw
    full = [A] * 6
    for k in (0, 1, 4):
        assert lib.dn_linear_forward(at(ok), *[None if i == k else v for i, v in enumerate(full)], A, 1 << 30, None) == dn.DN_ERR_INVALID_ARG
    for k in range(6):
        assert lib.dn_linear_forward(at(ok), *[A + 1 if i == k else v for i, v in enumerate(full)], A, 1 << 30, None) == dn.DN_ERR_INVALID_ARG
    back = [A] * 7
    for k in (0, 1, 2, 3):
        assert lib.dn_linear_backward(at(ok), *[None if i == k else v for i, v in enumerate(back)], A, need, None) == dn.DN_ERR_INVALID_ARG
    assert lib.dn_linear_backward(at(ok), A, A, A, A, A, None, A, A, need, None) == dn.DN_ERR_INVALID_ARG     # dbias without dW
    assert lib.dn_linear_backward(at(ok), *back, None, need, None) == dn.DN_ERR_INVALID_ARG
    assert lib.dn_linear_backward(at(ok), *back, A + 16, need, None) == dn.DN_ERR_INVALID_ARG
    assert lib.dn_linear_backward(at(ok), *back, A, need - 1, None) == dn.DN_ERR_SHAPE


def test_ffn_refuses(lib):
    at = C.addressof
    ok = ffn()
    need = [lib.dn_ffn_forward_workspace_bytes(at(ok)), lib.dn_ffn_backward_workspace_bytes(at(ok))]
    assert all(0 < n < BAD and n % 256 == 0 for n in need) and need[0] >= 100 * 48 * 2 and need[1] >= 100 * (3 * 48 + 64) * 2
    fwd, bwd = [A] * 10, [A] * 13
    for kw, status in WRONG + [({"d": 0}, dn.DN_ERR_SHAPE), ({"f": 0}, dn.DN_ERR_SHAPE), ({"f": 1 << 22}, dn.DN_ERR_SHAPE)]:
        d = ffn(**kw)
        assert lib.dn_ffn_forward_workspace_bytes(at(d)) == BAD and lib.dn_ffn_backward_workspace_bytes(at(d)) == BAD, kw
        assert lib.dn_ffn_forward(at(d), *fwd, A, 1 << 40, None) == status, kw
        assert lib.dn_ffn_backward(at(d), *bwd, A, 1 << 40, None) == status, kw
    for k in (0, 1, 3, 5, 8):
        assert lib.dn_ffn_forward(at(ok), *[None if i == k else v for i, v in enumerate(fwd)], A, 1 << 40, None) == dn.DN_ERR_INVALID_ARG
    for k in (0, 1, 2, 3, 4, 5, 7, 9, 11):
        assert lib.dn_ffn_backward(at(ok), *[None if i == k else v for i, v in enumerate(bwd)], A, 1 << 40, None) == dn.DN_ERR_INVALID_ARG
    for k in range(10):
        assert lib.dn_ffn_forward(at(ok), *[A + 1 if i == k else v for i, v in enumerate(fwd)], A, 1 << 40, None) == dn.DN_ERR_INVALID_ARG
    for k in range(13):
        assert lib.dn_ffn_backward(at(ok), *[A + 1 if i == k else v for i, v in enumerate(bwd)], A, 1 << 40, None) == dn.DN_ERR_INVALID_ARG
    assert lib.dn_ffn_forward(at(ok), *fwd, A, need[0] - 1, None) == dn.DN_ERR_SHAPE
    assert lib.dn_ffn_backward(at(ok), *bwd, A, need[1] - 1, None) == dn.DN_ERR_SHAPE
    assert lib.dn_ffn_forward(at(ok), *fwd, None, need[0], None) == dn.DN_ERR_INVALID_ARG


def test_norm_and_dropout_refuse(lib):
    at = C.addressof
    ok = norm()
    need = lib.dn_norm_backward_workspace_bytes(at(ok))
    assert 0 < need < BAD and need % 256 == 0
    fwd, bwd = [A] * 9, [A] * 15
    fwd[4] = bwd[4] = bwd[12] = None       # shifts belong to layer norms only
    for kw, status in [({"type": -1}, dn.DN_ERR_INVALID_ARG), ({"grad_type": dn.DN_BF16}, dn.DN_ERR_INVALID_ARG), ({"post": 3}, dn.DN_ERR_INVALID_ARG),
                       ({"pre": -1}, dn.DN_ERR_INVALID_ARG), ({"rows": 0}, dn.DN_ERR_SHAPE), ({"d": 0}, dn.DN_ERR_SHAPE), ({"d": 16385}, dn.DN_ERR_SHAPE),
                       ({"rows_per_gate": 0}, dn.DN_ERR_SHAPE), ({"scale": float("inf")}, dn.DN_ERR_INVALID_ARG), ({"eps": -1e-5}, dn.DN_ERR_INVALID_ARG)]:
        d = norm(**kw)
        assert lib.dn_norm_backward_workspace_bytes(at(d)) == BAD, kw
        assert lib.dn_norm_forward(at(d), *fwd, None) == status, kw
        assert lib.dn_norm_backward(at(d), *bwd, A, 1 << 40, None) == status, kw
    for k, v in ((0, None), (7, None), (8, None), (4, A), (0, A + 1)):
        assert lib.dn_norm_forward(at(ok), *[v if i == k else w for i, w in enumerate(fwd)], None) == dn.DN_ERR_INVALID_ARG, k
    assert lib.dn_norm_forward(at(norm(pre=0)), A, None, None, None, None, None, None, None, None, None) == dn.DN_ERR_INVALID_ARG
    for k, v in ((0, None), (7, None), (8, None), (9, None), (4, A), (12, A), (8, A + 1)):
        assert lib.dn_norm_backward(at(ok), *[v if i == k else w for i, w in enumerate(bwd)], A, need, None) == dn.DN_ERR_INVALID_ARG, k
    assert lib.dn_norm_backward(at(ok), *bwd, A, need - 1, None) == dn.DN_ERR_SHAPE
    assert lib.dn_norm_backward(at(ok), *bwd, A + 8, need, None) == dn.DN_ERR_INVALID_ARG
    drop = lambda t=dn.DN_F32, x=A, y=A, rows=4, cols=8, ldx=0, ldy=0, p=0.5: lib.dn_dropout(t, x, y, rows, cols, ldx, ldy, p, 1, 2, None)
    assert drop(x=None) == drop(y=None) == drop(t=5) == drop(p=1.0) == drop(p=-1.0) == drop(x=A + 2) == dn.DN_ERR_INVALID_ARG
    assert drop(rows=0) == drop(cols=0) == drop(ldx=7) == drop(ldy=-8) == drop(cols=1 << 22) == dn.DN_ERR_SHAPE


def test_nets_refuse_the_new_activations(lib):
    import numpy as np
    w, a = np.array([4, 3], np.int32), np.array([dn.DN_ACT_SILU], np.int32)
    h = C.c_void_p()
    st = lib.dn_net_create(w.ctypes.data_as(C.c_void_p), 2, a.ctypes.data_as(C.c_void_p), dn.DN_LOSS_MSE, 4, C.c_void_p(A), 1 << 40, None, C.byref(h))
    assert st == dn.DN_ERR_INVALID_ARG
