"""What the calls of a block of experts launch, asked of the library itself on a device that does not exist (fake_experts.cpp)."""
import os
import re
import subprocess

from block_launches import HERE, PRODUCT, ROOT, SHAPE, TYPE
from paper_2001_04206_amd import build, dn

EPILOGUE = ["linear", "gated", "dgated", "store", "dexpert", "pair"]
GROUP = ["none", "rows", "tokens", "terms of A", "terms of B"]


def compile_program(folder):
    if not os.path.exists(dn.LIB_PATH):
        build.build()
    exe, lib = str(folder / "fake_experts"), os.path.dirname(dn.LIB_PATH)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wno-unused-function", "-I", os.path.join(ROOT, "include"), "-I", HERE, os.path.join(HERE, "fake_experts.cpp"),
                    "-o", exe, "-L" + lib, "-l:libdn.so", "-Wl,--export-dynamic,--allow-shlib-undefined,--disable-new-dtags,-rpath," + lib + ",-rpath,/opt/rocm/lib"],
                   check=True)
    return exe


def ask(exe, calls):
    """For each (kind, type, six numbers): the two calls, each (status, [(mangled name, x, y, threads)])."""
    rows = []
    for at in range(0, len(calls), 500):
        commands = [":".join([k, str(TYPE[t])] + [str(v) for v in rest]) for k, t, *rest in calls[at:at + 500]]
        out = subprocess.run([exe, *commands], check=True, capture_output=True, text=True, timeout=120).stdout.splitlines()
        assert len(out) == 2 * len(commands), out
        for line in out:
            status, *launches = line.split()
            rows.append((int(status), [(l.split("/")[0],) + tuple(int(v) for v in l.split("/")[1:]) for l in launches]))
    return [rows[i:i + 2] for i in range(0, len(rows), 2)]


def kernel(launch):
    """What a launch is: a product's tile, its epilogue, its grouping and whether k is in parts; or the kernel's name with its parameters."""
    m = re.search(r"product_kernelI\w*?Li(\d)ELi(\d)ENS_5ShapeILi(\d)ELi(\d)ELi(\d)ELi(\d)ELi(\d)EEELb0ELi(\d)E", launch[0])
    if m:
        group = GROUP[int(m[8])]
        return (PRODUCT[int(m[1])], EPILOGUE[int(m[2])], SHAPE[",".join(m.group(3, 4, 5, 6, 7))], group, "terms" not in group and launch[2] > 1)
    m = re.search(r"\d\d([a-z_]+_kernel)(I.*?EEv|E)", launch[0])
    return (m[1], m[2], launch[1] > 1 if m[1] == "place_kernel" else None)


def kernels(exe, calls):
    found = []
    for call, passes in zip(calls, ask(exe, calls)):
        for status, _ in passes:
            assert status == dn.DN_OK, (call, status)
        found.append({kernel(l) for _, launches in passes for l in launches})
    return found
