"""The paged attention kernels' loads into LDS are inline assembly, for which the compiler keeps no distance between an
instruction and the ones that wrote its operands: a vector instruction's scalar result (v_readfirstlane, v_readlane) may
be read by a memory instruction five wait states later, not before. Checked in the built library: every such load brings
those states itself, whatever stands before it."""
import os
import re
import shutil
import subprocess

import pytest

import paper_2607_21291_amd as P

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
WAIT_STATES = 5


def _listing(tmp_path):
    lib = os.path.join(os.path.dirname(P.__file__), "libadadsf.so")
    if not os.path.exists(OBJDUMP) or not os.path.exists(lib):
        pytest.skip("no disassembler or no built library")
    shutil.copy(lib, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True, capture_output=True)
    parts = [f for f in sorted(os.listdir(tmp_path)) if f.endswith("gfx950")]
    assert parts
    for part in parts:
        yield from subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", part], cwd=tmp_path, check=True,
                                  capture_output=True, text=True).stdout.splitlines()


def test_loads_into_lds_wait_for_their_operands(tmp_path):
    kernel, waited, loads = "", None, 0
    for line in _listing(tmp_path):
        name = re.match(r"^[0-9a-f]+ <(.+)>:", line)
        if name:
            kernel = name.group(1)
        words = line.split("//")[0].split()
        if "paged_" not in kernel or len(words) < 2:
            continue
        # wait states since the block's first instruction, s_mov_b32 m0 (itself one)
        if words[:2] == ["s_mov_b32", "m0,"]:
            waited = 1
        elif words[0] == "s_nop" and waited is not None:
            waited += int(words[1], 0) + 1
        elif words[0].startswith("buffer_load") and words[-1] == "lds":
            assert waited is not None and waited >= WAIT_STATES, f"{kernel}: {line.strip()} after {waited} wait states"
            waited, loads = None, loads + 1
        elif waited is not None:
            waited += 1
    assert loads > 0
