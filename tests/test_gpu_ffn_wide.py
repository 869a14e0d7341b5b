"""The widest gated product of few rows: 2^28 - 8 columns over a contraction of 8, more than the kernel for few rows has threads for."""
import ctypes

import pytest
import torch

from paper_2406_06858_amd import binding as fb
from paper_2406_06858_amd import ffn

WIDE = (1 << 28) - 8
FEW = ffn.flux_ffn_tile_config_count()
PTR = 4096


def test_the_kernel_for_few_rows_refuses_it_when_named():
    p = ffn.glu_problem(1, WIDE, 8, w_is_nk=1, tile_config=FEW)
    assert ffn.lib().flux_glu(ctypes.byref(p), PTR, PTR, PTR, PTR, None, None, PTR, 1 << 40, None) == fb.FLUX_ERR_UNSUPPORTED
    assert ffn.flux_glu_workspace_bytes(ffn.FLUX_GLU_FORWARD, p) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("N", [WIDE, WIDE - 8])
def test_one_row_of_as_many_columns_as_there_can_be(N):
    """Ups of whole numbers under a gate of 64, whose SiLU is 64 to the last bit: H is 64 times the sum of a weight's row, exactly."""
    dev = "cuda:0"
    gen = torch.Generator(device=dev).manual_seed(3)
    x = torch.ones(1, 8, dtype=torch.bfloat16, device=dev)
    wg = torch.zeros(N, 8, dtype=torch.bfloat16, device=dev)
    wg[:, 5] = 64
    wu = torch.randint(-2, 3, (N, 8), generator=gen, device=dev, dtype=torch.int8).to(torch.bfloat16)
    h = torch.full((1, N), 7.0, dtype=torch.bfloat16, device=dev)
    p = ffn.glu_problem(1, N, 8, w_is_nk=1)
    n = ffn.flux_glu_workspace_bytes(ffn.FLUX_GLU_FORWARD, p)
    ffn.flux_glu(p, x, wg, wu, h, None, None, torch.zeros(n, dtype=torch.uint8, device=dev) if n else None)
    torch.cuda.synchronize()
    for c in range(0, N, 1 << 24):
        want = 64 * wu[c:c + (1 << 24)].float().sum(1)
        assert torch.equal(h[0, c:c + (1 << 24)].float(), want), c
    del wg, wu, h
    torch.cuda.empty_cache()
