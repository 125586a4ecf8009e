"""Sizes that do not fit the descriptors' 32-bit fields, through the Python binding with stand-in tensors (no GPU): they are refused, not
cut to their low 32 bits."""
import pytest
import torch

from paper_2001_04206_amd import dn


class Tensor:
    """What the binding asks of a contiguous bf16 tensor on device 0."""
    dtype, is_cuda, device = torch.bfloat16, True, torch.device("cuda:0")

    def __init__(self, *shape):
        self.shape = torch.Size(shape)

    def dim(self):
        return len(self.shape)

    def get_device(self):
        return 0

    def stride(self):
        return (self.shape[1], 1)

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 0x10000


@pytest.fixture
def seen(monkeypatch):
    """The descriptors' fields (dn_dropout: its arguments) that get to the library."""
    got = []

    class Library:
        def __getattr__(self, name):
            def call(*args):
                if name == "dn_status_string":
                    return b"shape"
                kind = {"dn_linear": dn.LinearDesc, "dn_ffn": dn.FfnDesc, "dn_norm": dn.NormDesc}.get("_".join(name.split("_")[:2]))
                if kind:
                    at = kind.from_address(args[0])
                    got.append({k: getattr(at, k) for k, _ in kind._fields_})
                else:
                    got.append({"rows": args[3], "cols": args[4]})
                return 0
            return call

    monkeypatch.setattr(dn, "lib", Library)
    monkeypatch.setattr(dn, "_on", lambda dev: dn._here)
    monkeypatch.setattr(dn, "_stream", lambda dev: 0)
    return got


MANY = (1 << 32) + 5


def calls(rows):
    T = Tensor
    return {
        "linear forward": lambda: dn.dn_linear_forward(T(rows, 8), T(4, 8), None, None, T(rows, 4)),
        "linear backward": lambda: dn.dn_linear_backward(T(rows, 8), T(4, 8), None, T(rows, 4), None, T(4, 8), None),
        "linear outputs": lambda: dn.dn_linear_forward(T(3, 8), T(rows, 8), None, None, T(3, rows)),
        "block forward": lambda: dn.dn_ffn_forward(T(rows, 8), T(4, 8), None, T(4, 8), None, T(8, 4), None, None, T(rows, 8)),
        "block hidden": lambda: dn.dn_ffn_forward(T(3, 8), T(rows, 8), None, T(rows, 8), None, T(8, rows), None, None, T(3, 8)),
        "block backward": lambda: dn.dn_ffn_backward(T(rows, 8), T(4, 8), T(4, 8), T(8, 4), T(rows, 8), T(rows, 8), None, T(4, 8), None, T(4, 8),
                                                     None, T(8, 4), None),
        "norm forward": lambda: dn.dn_norm_forward(T(rows, 8), None, None, None, None, None, None, None, T(rows, 8)),
        "norm backward": lambda: dn.dn_norm_backward(T(rows, 8), None, None, None, None, None, None, T(rows, 8), T(rows, 8), None, None, None, None,
                                                     None, None),
        "dropout": lambda: dn.dn_dropout(T(rows, 8), T(rows, 8), 0.5, 1),
        "dropout columns": lambda: dn.dn_dropout(T(3, rows), T(3, rows), 0.5, 1),
    }


@pytest.mark.parametrize("name", calls(1))
def test_too_many_rows_or_columns(seen, name):
    with pytest.raises(dn.DnError) as e:
        calls(MANY)[name]()
    assert e.value.status == dn.DN_ERR_SHAPE and not seen
    calls(7)[name]()
    assert seen and 7 in seen[-1].values()


@pytest.mark.parametrize("per,field", [(1 << 32, 6), (MANY, 6), (1 << 31, 6), (7, 6), (6, 6), (2, 2), (0, 0), (-1, 0)])
def test_rows_of_a_gate(seen, per, field):
    """More rows a gate than there are rows is one gate, however many."""
    x, gate = Tensor(6, 8), Tensor(-(-6 // per) if per > 0 else 0, 8)
    dn.dn_norm_forward(x, x, gate, None, None, None, None, x, x, rows_per_gate=per)
    assert seen[-1]["rows_per_gate"] == field
