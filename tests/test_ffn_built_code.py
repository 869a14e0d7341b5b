"""The tile kernel's MFMAs and LDS reads are written out as instructions (see test_built_code): what the compiler placed between them
is checked in the code that was built, and that no register of a kernel went to scratch memory, where it would be an accumulator
stored right behind its MFMA."""
import os
import re
import subprocess

import pytest
from test_built_code import OBJDUMP, _blocks, _check_block

from paper_2406_06858_amd import build

READELF = "/opt/rocm/llvm/bin/llvm-readelf"


def _objects(tmp_path):
    lib = tmp_path / "lib.so"
    lib.symlink_to(build.FFN_LIB)
    subprocess.run([OBJDUMP, "--offloading", str(lib)], cwd=tmp_path, check=True, capture_output=True)
    return [p for p in tmp_path.iterdir() if "gfx950" in p.name]


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no disassembler")
def test_nothing_between_the_written_out_instructions(tmp_path):
    kernels = 0
    for o in _objects(tmp_path):
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr", str(o)], check=True, capture_output=True, text=True).stdout
        for name, body in re.findall(r"^<(\S*tile_kernel\S*)>:\n(.*?)(?=^<_Z|\Z)", text, flags=re.S | re.M):
            with_mfma = [b for b in _blocks(body) if any(i.startswith("v_mfma") for i in b)]
            kernels += bool(with_mfma)
            for block in with_mfma:
                assert _check_block(block) is None, name
    assert kernels >= 2 * build.FFN_KINDS


@pytest.mark.skipif(not (os.path.exists(OBJDUMP) and os.path.exists(READELF)), reason="no object tools")
def test_registers_do_not_spill(tmp_path):
    found = []
    for o in _objects(tmp_path):
        notes = subprocess.run([READELF, "--notes", str(o)], check=True, capture_output=True, text=True).stdout
        found += re.findall(r"\.name:\s+(\S+)\s+\.private_segment_fixed_size:\s+(\d+)", notes)
    assert len(found) >= 2 * build.FFN_KINDS
    assert [n for n in found if int(n[1])] == []
