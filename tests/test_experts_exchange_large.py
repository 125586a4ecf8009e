"""The large tiles of the experts' products turn a wave's sums through LDS as the others do (test_experts_exchange.py, which leaves them out): no
read of LDS follows a write, and no write a read, without a wave barrier between (no GPU: the assembly of the build's own flags)."""
import os
import re
import subprocess

import pytest

from paper_2001_04206_amd import build

KERNELS = ["bf16, P_FWD, E_PAIR, Large, false, G_ROWS", "bf16, P_GRAD, E_STORE, Large, false, G_TERMS_A", "f16, P_GRAD, E_STORE, Large, false, G_TERMS_B",
           "bf16, P_FWD, E_GATED, Large, false, G_TOKENS", "f16, P_DELTA, E_STORE, Large, false, G_ROWS"]


@pytest.mark.parametrize("kernel", KERNELS)
def test_reads_and_writes_of_lds_are_kept_apart(kernel, tmp_path):
    src = tmp_path / "epilogue.hip"
    src.write_text('#include "dn_ffn_tile.h"\nnamespace dn {\ntemplate __global__ void product_kernel<%s>(const ProductArgs);\n}\n' % kernel)
    subprocess.run([build.HIPCC, *build.FLAGS, "-I", build.CSRC, "-I", os.path.join(build.HERE, "..", "include"), "--cuda-device-only", "-S", str(src), "-o",
                    str(tmp_path / "epilogue.s")], check=True, capture_output=True)
    (body,) = re.findall(r"^_Z\S*product_kernel\S*:(.*?)^\.Lfunc_end", (tmp_path / "epilogue.s").read_text(), re.M | re.S)
    exchanges = 0
    for part in body.split("s_barrier"):
        seen = re.findall(r"(ds_write|ds_read|wave barrier)", part)
        if "ds_write" not in seen or "wave barrier" not in seen:
            continue
        exchanges += seen.count("ds_write")
        last = None
        for what in seen[seen.index("ds_write"):]:
            assert not (last and what != last and what != "wave barrier"), "a %s follows a %s" % (what, last)
            last = None if what == "wave barrier" else what
    assert exchanges >= 8      # the exchange is there
