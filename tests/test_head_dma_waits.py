"""The head's products load LDS by inline assembly, for which the compiler keeps no distance between an instruction and
the ones that wrote its operands: a vector instruction's scalar result may be read by a memory instruction five wait
states later, not before. Checked in the built library, as for the paged attention's loads."""
import re

from test_paged_dma_waits import WAIT_STATES, _listing


def test_loads_into_lds_wait_for_their_operands(tmp_path):
    kernel, waited, moved, loads = "", None, 0, 0
    for line in _listing(tmp_path):
        name = re.match(r"^[0-9a-f]+ <(.+)>:", line)
        if name:
            kernel = name.group(1)
        words = line.split("//")[0].split()
        if "head_gemm_kernel" not in kernel or len(words) < 2:
            continue
        # wait states since the block's first instruction, a move to m0; a block may hold two loads
        if words[0] == "s_nop" and waited is not None:
            waited += int(words[1], 0) + 1
        elif words[0].startswith("buffer_load") and words[-1] == "lds":
            assert waited is not None and waited >= WAIT_STATES, f"{kernel}: {line.strip()} after {waited} wait states"
            assert moved >= 2, f"{kernel}: {line.strip()} right after its move to m0"
            waited, loads = waited + 1, loads + 1
        elif words[:2] == ["s_mov_b32", "m0,"]:
            waited, moved = 1 if waited is None else waited + 1, 0
        else:
            waited = None
        moved += 1 if words[0] != "s_nop" else int(words[1], 0) + 1
    assert loads > 0
