"""Compiles libsparsecontract.so (HIP, gfx950) in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB_PATH = os.path.join(HERE, "libsparsecontract.so")
SOURCES = ["host.cpp", "kernels.hip", "kernels_linear.hip", "kernels_order2.hip", "kernels_order4.hip", "kernels_traverse.hip", "kernels_ttmc3.hip", "kernels_slice.hip", "kernels_chain4.hip", "kernels_mttkrp.hip", "kernels_ttmc4.hip", "kernels_ttmc_all.hip", "kernels_gemm.hip", "static_scratch.hip",
           "attention.cpp", "kernels_append.hip", "kernels_prompt.hip", "kernels_prompt_window.hip", "kernels_prompt_tree.hip", "kernels_decode.hip", "kernels_tree.hip", "kernels_pages.hip"]

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    "-munsafe-fp-atomics",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function", "-Wno-unknown-attributes",
]


def build_library(verbose: bool = False) -> str:
    """Compiles every source, as many at a time as there are processors (16 at most), and links them."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.check_call(cmd)

    with tempfile.TemporaryDirectory() as objects, ThreadPoolExecutor(min(16, len(os.sched_getaffinity(0)))) as pool:
        names = [os.path.join(objects, s + ".o") for s in SOURCES]
        compiled = [pool.submit(run, [hipcc, *HIPCC_FLAGS, "-x", "hip", "-c", os.path.join(CSRC, s), "-o", o]) for s, o in zip(SOURCES, names)]
        for c in compiled:
            c.result()
        run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", *names, "-o", LIB_PATH])
    return LIB_PATH


if __name__ == "__main__":
    print(build_library(verbose=True))
