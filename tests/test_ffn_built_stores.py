"""The tile kernels' 16-byte stores past the caches are written out as instructions, so the compiler does not keep its distance from their
data: gfx950 wants two wait states before a register of a store of more than 8 bytes is written again (the compiler puts `s_nop 1`
behind its own).  Every such store has to bring them along, whatever follows it in the code that was built."""
import os
import re
import subprocess

import pytest
from test_built_code import OBJDUMP
from test_ffn_built_code import _objects

from paper_2406_06858_amd import build

TILES = 6               # tile shapes that each kind of product is built for, masked and not
WAIT_STATES = 2


def _check_stores(lines):
    """First streamed store among the instructions that does not bring its wait states, or None; and how many there were."""
    stores = 0
    for i, line in enumerate(lines):
        if not (line.startswith("global_store_dwordx4") and line.split()[-1] == "nt"):
            continue
        stores += 1
        states = 0
        for after in lines[i + 1:]:
            if not after.startswith("s_nop"):
                break
            states += int(after.split()[1], 0) + 1
        if states < WAIT_STATES:
            return line, stores
    return None, stores


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no disassembler")
def test_streamed_stores_bring_their_wait_states(tmp_path):
    kernels, stores = 0, 0
    for o in _objects(tmp_path):
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr", str(o)], check=True, capture_output=True, text=True).stdout
        for name, body in re.findall(r"^<(\S*tile_kernel\S*)>:\n(.*?)(?=^<_Z|\Z)", text, flags=re.S | re.M):
            lines = [line.split("//")[0].strip() for line in body.splitlines()]
            bad, n = _check_stores([line for line in lines if line and not line.endswith(":")])
            assert bad is None, f"{name}: {bad}"
            assert n > 0, name
            kernels += any(line.startswith("v_mfma") for line in lines)
            stores += n
    assert kernels == 2 * TILES * build.FFN_KINDS and stores >= 2 * kernels


@pytest.mark.parametrize("lines,bad", [
    (["global_store_dwordx4 v[0:1], v[2:5], off nt", "s_nop 0", "s_cbranch_execnz 12", "v_mov_b32_e32 v2, v9"], True),
    (["global_store_dwordx4 v[0:1], v[2:5], off nt", "v_mov_b32_e32 v2, v9"], True),
    (["global_store_dwordx4 v[0:1], v[2:5], off nt", "s_nop 1", "v_mov_b32_e32 v2, v9"], False),
    (["global_store_dwordx4 v[0:1], v[2:5], off nt", "s_nop 0", "s_nop 0", "v_mov_b32_e32 v2, v9"], False),
    (["global_store_dwordx4 v[0:1], v[2:5], off", "v_mov_b32_e32 v2, v9"], False),
])
def test_the_check_finds_what_it_looks_for(lines, bad):
    assert (_check_stores(lines)[0] is not None) == bad
