"""The kernels of logits share the tile kernel's main loop, whose MFMAs, LDS reads and streamed stores are written out as instructions (see test_ffn_built_code and
test_ffn_built_stores): the same is checked in their built code."""
import os
import re
import subprocess

import pytest
from test_built_code import OBJDUMP, _blocks, _check_block
from test_ffn_built_code import _objects
from test_ffn_built_stores import TILES, _check_stores


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no disassembler")
def test_nothing_between_the_written_out_instructions(tmp_path):
    kernels, stores = 0, 0
    for o in _objects(tmp_path):
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr", str(o)], check=True, capture_output=True, text=True).stdout
        for name, body in re.findall(r"^<(\S*(?:13logits|13scaled|15streamed)_kernel\S*)>:\n(.*?)(?=^<_Z|\Z)", text, flags=re.S | re.M):
            with_mfma = [b for b in _blocks(body) if any(i.startswith("v_mfma") for i in b)]
            kernels += bool(with_mfma)
            for block in with_mfma:
                assert _check_block(block) is None, name
            lines = [line.split("//")[0].strip() for line in body.splitlines()]
            bad, n = _check_stores([line for line in lines if line and not line.endswith(":")])
            assert bad is None, f"{name}: {bad}"
            stores += n
    # statistics and dZ, masked and not, those of the four tiles of up to 128 rows with streamed weights too; dX of these four; dX and dW, masked and not
    assert kernels == 2 * 2 * (TILES + 4) + 4 + 2 * 2 * TILES and stores > 0
