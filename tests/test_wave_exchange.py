"""The matrix products' epilogue turns a wave's sums through LDS, where lanes read what other lanes wrote.  The compiler sees one lane's
program and may move a read across a write to another address, so a wave barrier has to stand between them: after the last barrier of
the loop, in the assembly that the build's own flags give, no read of LDS follows a write, and no write a read, without one.  (No GPU.)"""
import os
import re
import subprocess

import pytest

from paper_2001_04206_amd import build

KERNELS = ["bf16, P_FWD, E_LINEAR, Small, false", "float, P_GRAD, E_STORE, Tiny, true", "f16, P_FWD, E_GATED, Small, false",
           "bf16, P_DELTA, E_DGATED, Medium, false"]


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    at = tmp_path_factory.mktemp("wave_exchange")
    src = at / "epilogues.hip"
    src.write_text('#include "dn_ffn_tile.h"\nnamespace dn {\n' +
                   "".join("template __global__ void product_kernel<%s>(const ProductArgs);\n" % k for k in KERNELS) + "}\n")
    subprocess.run([build.HIPCC, *build.FLAGS, "-I", build.CSRC, "-I", os.path.join(build.HERE, "..", "include"), "--cuda-device-only", "-S", str(src), "-o",
                    str(at / "epilogues.s")], check=True, capture_output=True)
    return (at / "epilogues.s").read_text()


def test_reads_and_writes_of_lds_are_kept_apart(assembly):
    kernels = re.findall(r"^(_Z\S*product_kernel\S*):.*?^\s*s_endpgm", assembly, re.M | re.S)
    bodies = re.findall(r"^_Z\S*product_kernel\S*:(.*?)^\.Lfunc_end", assembly, re.M | re.S)
    assert len(kernels) == len(bodies) == len(KERNELS)
    for name, body in zip(kernels, bodies):
        epilogue = body[body.rindex("s_barrier"):]
        seen = re.findall(r"(ds_write|ds_read|wave barrier)", epilogue)
        assert seen.count("ds_write") >= 8 and seen.count("ds_read") >= 8, name      # the exchange is there
        last = None
        for what in seen:
            assert not (last and what != last and what != "wave barrier"), "%s: a %s follows a %s" % (name, what, last)
            last = None if what == "wave barrier" else what
