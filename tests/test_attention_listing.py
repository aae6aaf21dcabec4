"""The listing of the built attention kernels, which are compiled from this repository's sources: what the compiler does with registers where a step takes nearly all of them."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2311_09549_amd import binding as sc

LLVM = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin")
KERNELS = ("tree_kernel", "tree_whole_kernel", "prompt_tile_kernel", "prompt_kernel", "decode_kernel")

COPY = re.compile(r"v_accvgpr_(write|read|mov)_b32 [av]\d+, [av]\d+$|v_mov_b(32|64)(_e32|_e64)? v\S+, v\S+$|scratch_(load|store)_\w+ ")
LANES = re.compile(r"v_(read|write)lane_b32 ")           # scalar registers kept in lanes of a vector one, whichever lanes are on


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


def copies_before_all_lanes(listing):
    """Blocks that begin with copies of vector registers, and nothing else, before the lanes of a branch come back: such copies reach a part of the lanes only.  (A branch of which the
    whole body is a copy looks the same; these kernels have none.)"""
    found, block, copies, open_ = [], None, [], False
    for function, label, x in instructions(listing):
        if (function, label) != block:
            block, copies, open_ = (function, label), [], label is not None
        if not open_:
            continue
        if x.startswith("s_or_b64 exec, exec"):
            if copies:
                found.append((function, label, copies))
            open_ = False
        elif COPY.match(x):
            copies.append(x)
        elif re.match(r"v_|ds_|global_|buffer_|flat_|s_c?branch|s_endpgm|s_\w+_saveexec|s_\w+ exec", x) and not LANES.match(x):
            open_ = False
    return found


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


def test_no_copies_under_a_part_of_the_lanes(listings):
    functions = {function for x in listings for function, _, _ in instructions(x)}
    assert all(any(k in f for f in functions) for k in KERNELS)
    for x in listings:
        assert not copies_before_all_lanes(x)


def test_the_scan_finds_them():
    """As the compiler wrote it for two tiles of pairs of heads of 256 whose masks were made in a branch: sums of lanes without a pair were wrong."""
    text = "<tree>:\n\tv_mov_b32_e32 v1, v2\n\ts_or_b64 exec, exec, s[2:3]\n<L7>:\n%s\ts_or_b64 exec, exec, s[0:1] // 00: 0\n\tv_mfma_f32_16x16x32_bf16 a[0:3], v[0:3], v[4:7], a[0:3]\n"
    bad = "\tv_readlane_b32 s0, v252, 16\n\tv_accvgpr_write_b32 a2, v84\n\tv_readlane_b32 s0, v251, 57\n"
    assert copies_before_all_lanes(text % bad) == [("tree", "L7", ["v_accvgpr_write_b32 a2, v84"])]
    assert copies_before_all_lanes(text % "\tscratch_load_dword v3, off, s32\n")
    assert not copies_before_all_lanes(text % "\tv_readlane_b32 s0, v252, 16\n\tv_mov_b32_e32 v204, 0xffff\n")
    assert not copies_before_all_lanes(text % "\tv_add_u32_e32 v2, v3, v4\n\tv_mov_b32_e32 v204, v2\n")


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
