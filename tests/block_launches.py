"""What the residual feed-forward block's calls launch, asked of the library itself on a device that does not exist (fake_block.cpp)."""
import math
import os
import re
import subprocess

from paper_2001_04206_amd import build, dn

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
TYPE = {"f32": dn.DN_F32, "f16": dn.DN_F16, "bf16": dn.DN_BF16}
# waves down and across, blocks down and across, stages
SHAPE = {"2,4,8,4,2": "large", "2,4,4,4,3": "medium", "2,2,4,4,2": "small", "2,2,2,4,2": "tiny"}
PRODUCT = ["forward", "delta", "gradient"]
EPILOGUE = ["linear", "gated", "dgated", "store"]


def compile_program(folder):
    if not os.path.exists(dn.LIB_PATH):
        build.build()
    exe, lib = str(folder / "fake_block"), os.path.dirname(dn.LIB_PATH)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", os.path.join(ROOT, "include"), os.path.join(HERE, "fake_block.cpp"), "-o", exe, "-L" + lib,
                    "-l:libdn.so", "-Wl,--export-dynamic,--allow-shlib-undefined,--disable-new-dtags,-rpath," + lib + ",-rpath,/opt/rocm/lib"], check=True)
    return exe


def ask(exe, calls):
    """For each (kind, type, rows, n, m, bytes off): [forward, backward], each (status, [(mangled name, x, y, threads)])."""
    commands = [":".join([k, str(TYPE[t])] + [str(v) for v in rest]) for k, t, *rest in calls]
    out = subprocess.run([exe, *commands], check=True, capture_output=True, text=True, timeout=120).stdout.splitlines()
    assert len(out) == 2 * len(calls), out
    rows = []
    for line in out:
        status, *launches = line.split()
        rows.append((int(status), [(l.split("/")[0],) + tuple(int(v) for v in l.split("/")[1:]) for l in launches]))
    return [rows[i:i + 2] for i in range(0, len(rows), 2)]


def product(launch):
    """(product, epilogue, shape, whether sums come with it, parts of k) of a launch of a matrix product in tiles, or None."""
    m = re.search(r"product_kernelI\w*?Li(\d)ELi(\d)ENS_5ShapeILi(\d)ELi(\d)ELi(\d)ELi(\d)ELi(\d)EEELb([01])E", launch[0])
    return m and (PRODUCT[int(m[1])], EPILOGUE[int(m[2])], SHAPE[",".join(m.group(3, 4, 5, 6, 7))], m[8] == "1", launch[2])


def kernels(exe, calls):
    """What each call launches: tiles with their epilogue, segments and whether k is in parts; kernels for few rows; norms."""
    found = []
    for at in range(0, len(calls), 500):
        for call, passes in zip(calls[at:at + 500], ask(exe, calls[at:at + 500])):
            seen = set()
            for status, launches in passes:
                assert status == dn.DN_OK, call
                for launch in launches:
                    p = product(launch)
                    few = re.search(r"(few|token)_kernelI(.*?)Li(\d)E(.*?)EvNS", launch[0])
                    norm = re.search(r"(norm_(?:forward|backward)_kernel)I(.*?)EvNS", launch[0])
                    if p:
                        seen.add((call[1],) + p[:4] + (call[0] == "block" and p[:2] == ("delta", "store"), p[4] > 1))
                    elif few:
                        seen.add((call[1], few[1], EPILOGUE[int(few[3])], few[4]))
                    elif norm:
                        seen.add((norm[1], norm[2]))
            found.append(seen)
    return found


def sizes(rng, lo, hi):
    """A size of that range, evenly over its logarithm; four in ten a multiple of 8, the others odd."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(1, n // 8 * 8) if rng.random() < 0.4 else n | 1
