"""The experts' products turn a wave's sums through LDS as the block's do (test_wave_exchange.py): between their barriers, in the assembly
that the build's own flags give, no read of LDS follows a write, and no write a read, without a wave barrier.  And waves without rows meet
the others at every barrier: as many in their short way through the loop as in the long one.  (No GPU.)"""
import os
import re
import subprocess

import pytest

from paper_2001_04206_amd import build

KERNELS = ["bf16, P_FWD, E_PAIR, Small, false, G_ROWS", "float, P_GRAD, E_STORE, Tiny, false, G_TERMS_B", "f16, P_FWD, E_GATED, Small, false, G_TOKENS",
           "bf16, P_DELTA, E_DEXPERT, Medium, false, G_TOKENS", "float, P_DELTA, E_STORE, Small, false, G_ROWS"]


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    at = tmp_path_factory.mktemp("experts_exchange")
    src = at / "epilogues.hip"
    src.write_text('#include "dn_ffn_tile.h"\nnamespace dn {\n' +
                   "".join("template __global__ void product_kernel<%s>(const ProductArgs);\n" % k for k in KERNELS) + "}\n")
    subprocess.run([build.HIPCC, *build.FLAGS, "-I", build.CSRC, "-I", os.path.join(build.HERE, "..", "include"), "--cuda-device-only", "-S", str(src), "-o",
                    str(at / "epilogues.s")], check=True, capture_output=True)
    return (at / "epilogues.s").read_text()


def test_reads_and_writes_of_lds_are_kept_apart(assembly):
    bodies = re.findall(r"^(_Z\S*product_kernel\S*):(.*?)^\.Lfunc_end", assembly, re.M | re.S)
    assert len(bodies) == len(KERNELS)
    for name, body in bodies:
        exchanges = 0
        for part in body.split("s_barrier"):
            seen = re.findall(r"(ds_write|ds_read|wave barrier)", part)
            if "ds_write" not in seen or "wave barrier" not in seen:
                continue
            exchanges += seen.count("ds_write")
            last = None
            for what in seen[seen.index("ds_write"):]:
                assert not (last and what != last and what != "wave barrier"), "%s: a %s follows a %s" % (name, what, last)
                last = None if what == "wave barrier" else what
        assert exchanges >= 8, name      # the exchange is there


def test_every_way_through_the_loop_has_the_same_barriers():
    """The two loops of the source, for every shape and number of stages: how often a wave that multiplies meets a barrier, and one that only
    loads."""
    text = open(os.path.join(build.CSRC, "dn_ffn_tile.h")).read()
    idle = text[text.index("if (IDLE && m0 + wm"):]
    idle = idle[:idle.index("return;")]
    busy = text[text.index("    Half f0, f1;"):]
    busy = busy[busy.index("prepare(t0);\n        fetch(stage0);", busy.index("return;")):busy.index("        arrived<0>();\n        terms +=")]
    assert idle.count("arrived<") == 3 and "for (; t + (S::TM == 8 ? 0 : S::NB - 1) < t1; t += S::NB)" in idle
    assert "for (; t + 2 < t1; t += 3)" in busy and "for (; t + (S::TM == 8 ? 0 : 1) < t1; t += 2)" in busy

    def multiplying(large, stages, n):
        met, t = 1, 0
        if stages == 3:
            while t + 2 < n:
                met, t = met + 3, t + 3
            met += (t < n) + (t + 1 < n)
        else:
            while t + (0 if large else 1) < n:
                met, t = met + 2, t + 2
            met += (not large) and t < n
        return met + 1

    def loading(large, stages, n):
        met, t = 1, 0
        while t + (0 if large else stages - 1) < n:
            met, t = met + stages, t + stages
        met += ((not large) and t < n) + (stages == 3 and t + 1 < n)
        return met + 1

    for large, stages in ((True, 2), (False, 2), (False, 3)):
        for n in range(200):
            assert multiplying(large, stages, n) == loading(large, stages, n), (large, stages, n)
