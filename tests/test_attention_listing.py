"""The listing of the built attention kernels, which are compiled from this repository's sources: what the compiler does with registers where a step takes nearly all of them."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2311_09549_amd import binding as sc

LLVM = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin")
KERNELS = ("tree_kernel", "tree_whole_kernel", "prompt_tile_kernel", "prompt_kernel", "decode_kernel")


def instructions(listing):
    """(function, label or None, instruction) line by line."""
    function, label = None, None
    for line in listing.splitlines():
        line = line.split("//")[0].strip()
        start = re.match(r"<(.+)>:$", line)
        if start:
            name = start.group(1)
            function, label = (function, name) if re.match(r"L\d+$", name) else (name, None)
        elif line and not line.startswith(";"):
            yield function, label, line


@pytest.fixture(scope="module")
def listings(tmp_path_factory):
    where = tmp_path_factory.mktemp("listing")
    library = shutil.copy(sc.LIB_PATH, where)      # what it holds for the GPU is written beside it
    run = lambda *args: subprocess.run(args, cwd=where, check=True, capture_output=True, text=True, timeout=300).stdout      # noqa: E731
    run(os.path.join(LLVM, "llvm-objdump"), "--offloading", library)
    out = []
    for name in sorted(os.listdir(where)):
        if name.endswith("gfx950") and any(k in run(os.path.join(LLVM, "llvm-readelf"), "-s", "--wide", name) for k in KERNELS):
            out.append(run(os.path.join(LLVM, "llvm-objdump"), "-d", "--no-show-raw-insn", "--no-leading-addr", "--symbolize-operands", name))
    return out


def test_m0_is_of_the_loads_to_lds_alone(listings):
    """Each load that goes straight to LDS sets m0 itself, right before it, and nothing else of its source has to do with it."""
    loads = 0
    for x in listings:
        lines = [i for _, _, i in instructions(x)]
        to_lds = [n for n, i in enumerate(lines) if "global_load_lds" in i]
        loads += len(to_lds)
        if to_lds:
            assert [n for n, i in enumerate(lines) if re.search(r"\bm0\b", i)] == [n - 2 for n in to_lds]
            assert all(re.match(r"s_mov_b32 m0, s\d+$", lines[n - 2]) and lines[n - 1] == "s_nop 0" for n in to_lds)
    assert loads > 0
