"""Build step: compiles the HIP library for gfx950 in-tree (paper_2311_17410_amd/libtns.so)."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libtns.so")
SOURCES = ["tns_api.hip", "tns_kernels.hip", "tns_kernels_recent.hip", "tns_store.cpp", "tns_pstore.cpp", "tns_kernels_prefix.hip", "tns_kernels_team.hip", "tns_cache.hip", "tns_ingest.hip", "tns_probe.hip",
           "tns_recur.hip", "tns_pairs.hip", "tns_adamw.hip", "tns_attend.hip", "tns_attend_grad.hip", "tns_block.hip", "tns_distill.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden",
    "-Wall", "-Wextra", "-Wno-unused-parameter",
    # no packed-fp32 instructions in device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


def build(verbose: bool = False, extra: list[str] | None = None) -> str:
    """Compiles every source, as many at a time as there are processors (eight at most: each takes some GB), and links them."""
    tmp = LIB + f".tmp{os.getpid()}"
    flags = [f for f in FLAGS if f != "-shared"] + (extra or [])

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.check_call(cmd)

    with tempfile.TemporaryDirectory() as at, ThreadPoolExecutor(min(os.cpu_count() or 1, 8)) as pool:
        objects = [os.path.join(at, s + ".o") for s in SOURCES]
        list(pool.map(lambda s, o: run([HIPCC] + flags + ["-x", "hip", "-c", os.path.join(CSRC, s), "-o", o]), SOURCES, objects))
        run([HIPCC] + FLAGS + (extra or []) + objects + ["-o", tmp])
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True, extra=sys.argv[1:]))
