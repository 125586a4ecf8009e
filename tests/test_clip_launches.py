"""What dn_clip launches, asked of the library on a device that does not exist (fake_experts.cpp): the parts of the sum are added up once a call, not
by every workgroup of every launch (no GPU)."""
import pytest

from experts_launches import ask, compile_program, kernel


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    return compile_program(tmp_path_factory.mktemp("clip_launches"))


@pytest.mark.parametrize("tensors", [1, 80, 81, 160, 161, 400, 5000])
def test_the_sum_is_formed_once(exe, tensors):
    runs = -(-tensors // 80)
    (written, launches), (_, alone) = ask(exe, [("clip", "bf16", tensors, 9000, 1, 0, 0, 0)])[0]
    names = [kernel(l)[0] for l in launches]
    only = [kernel(l)[0] for l in alone]
    assert written == 0
    if runs == 1:   # few parts, which the launch that needs their sum adds up itself
        assert names == only == ["squares_kernel", "times_kernel"]
        return
    assert names == ["squares_kernel"] * runs + ["total_kernel"] + ["times_kernel"] * runs
    assert only == ["squares_kernel"] * runs + ["total_kernel"]
    assert [l[1] for l in launches if "total_kernel" in l[0]] == [1]
