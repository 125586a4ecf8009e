"""Every kernel of a block of experts that the library holds is one that its rules take for some call (no GPU: the library's own symbols, and
fake_experts.cpp in the place of a device)."""
import re
import subprocess

import pytest

import test_gpu_experts_kernels as gpu
from block_launches import TYPE
from experts_launches import ask, compile_program
from paper_2001_04206_amd import dn
from test_experts_kernels import sample


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    return compile_program(tmp_path_factory.mktemp("experts_compiled"))


def compiled():
    """Mangled names of the kernels, from those of the functions that launch them."""
    names = set()
    for line in subprocess.run(["nm", dn.LIB_PATH], check=True, capture_output=True, text=True).stdout.splitlines():
        m = re.fullmatch(r".* (\S*?)\d+__device_stub__(\w+?_kernel)(\S*)", line)
        if m:
            names.add("%s%d%s%s" % (m[1], len(m[2]), m[2], m[3]))
    return names


def test_nothing_that_no_call_reaches(exe):
    """The grouped products, the kernels for few rows and the sums; without bytes missed and with 16, 4 and 2 of them."""
    grouped = re.compile(r"product_kernel\S*ELi[1-4]EEEvNS_11ProductArgsE|experts_few_kernel|few_down_kernel|join_pairs_kernel|dots_kernel")
    mine = {n for n in compiled() if grouped.search(n)}
    assert len(mine) > 50 and all(any(k in n for n in mine) for k in ("product_kernel", "experts_few_kernel", "few_down_kernel", "join_pairs_kernel"))
    taken = set()
    for kind in TYPE:
        calls = [("experts", kind) + s + (off,) for s in gpu.EXPERTS[32 if kind == "f32" else 16] for off in ((0, 16, 4) if kind == "f32" else (0, 16, 4, 2))]
        for passes in ask(exe, calls + sample(kind, 8000, 11)):
            for status, launches in passes:
                assert status == dn.DN_OK
                taken |= {l[0] for l in launches}
    # (without dX the weights' derivatives have a launch of their own, which these calls do not make)
    missing = {n for n in mine - taken if "dots_kernel" not in n and "join_pairs_kernel" not in n}
    assert not missing, missing
