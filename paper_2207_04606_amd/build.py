"""Compiles the HIP sources into paper_2207_04606_amd/libsptir.so for gfx950."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libsptir.so")
SOURCES = ["api.hip", "builder.hip", "order.hip", "spmm.hip", "spmm_slices.hip", "spmm_csr.hip", "sddmm.hip", "sddmm_slices.hip", "search.hip", "rgms.hip", "roof.hip",
           "moe_route.hip", "moe_rows.hip", "moe_product.hip", "moe_few.hip", "moe_tiles_forward.hip",
           "moe_tiles_dx.hip", "moe_tiles_dw.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # keep the compiler from forming packed-fp32 instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # float atomic adds on Y compile to the hardware instruction
    "-munsafe-fp-atomics",
    "-Wall", "-Wno-unused-function",
]


def sources():
    return [os.path.join(CSRC, s) for s in SOURCES]


def is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    headers = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".h")]
    deps = sources() + headers + [os.path.join(ROOT, "include", "sptir.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def _jobs() -> int:
    """Compilers at once (about 1.5 GB each)."""
    return max(1, min(int(os.environ.get("MAX_JOBS", 8)), os.cpu_count() or 1))


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd)


def build(verbose: bool = False) -> str:
    """Every source to an object, several at once, then the library."""
    with tempfile.TemporaryDirectory() as out, ThreadPoolExecutor(_jobs()) as pool:
        objects = [os.path.join(out, os.path.basename(s) + ".o") for s in sources()]
        includes = ["-I", os.path.join(ROOT, "include"), "-I", CSRC]
        cmds = [[HIPCC, *FLAGS, *includes, "-c", "-o", o, s] for s, o in zip(sources(), objects)]
        for done in [pool.submit(_run, cmd, verbose) for cmd in cmds]:
            done.result()
        _run([HIPCC, "--offload-arch=gfx950", "-fPIC", "-shared", "-o", LIB, *objects], verbose)
    return LIB


if __name__ == "__main__":
    build(verbose=True)
    print(LIB)
