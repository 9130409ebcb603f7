"""Build the gfx950 shared library (libvfl.so) in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libvfl.so")
SOURCES = ["chain.hip", "dw.hip", "lin.hip", "rowops.hip", "embed.hip", "rownorm.hip", "rms.hip",
           "matmul8.hip", "softloss.hip", "api.cpp", "rowops.cpp", "ops8.cpp", "schedule.cpp", "planner.cpp"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wall", "-Wno-unused-function", "-Werror=uninitialized", "-Werror=unused-variable"]


def build(verbose: bool = False) -> str:
    """Compile every source into libvfl.so (always rebuilds), a few at a time."""
    noise = "is not a recognized feature for this target"

    def hipcc(args):
        r = subprocess.run([HIPCC, *FLAGS, *args], capture_output=True, text=True)
        msgs = "\n".join(l for l in (r.stdout + r.stderr).splitlines() if noise not in l)
        if r.returncode != 0:
            raise RuntimeError("hipcc failed:\n" + msgs)
        if verbose and msgs.strip():
            print(msgs, file=sys.stderr)

    tmp = LIB + ".tmp"
    with tempfile.TemporaryDirectory() as objects, ThreadPoolExecutor(min(8, os.cpu_count() or 1)) as pool:
        objs = [os.path.join(objects, s + ".o") for s in SOURCES]
        list(pool.map(hipcc, (["-c", os.path.join(CSRC, s), "-o", o] for s, o in zip(SOURCES, objs))))
        hipcc(["-shared", *objs, "-o", tmp])
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
