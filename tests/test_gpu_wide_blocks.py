"""Blocks of rows so wide that eight (4) bits times a number's place take more than 31 bits, read back: every number."""
import pytest
import torch

from oracle import norm_loss_oracle as no
from paper_2406_06858_amd import ffn, norm

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("bits,K", [(8, (1 << 28) + 40), (4, (1 << 29) + 40)])
def test_a_wide_row(bits, K):
    blocks = (K + 31) // 32
    q = torch.empty(1, blocks * bits * 4, dtype=torch.uint8, device=DEV)
    for at, part in enumerate(q[0].split(1 << 24)):                    # (a pattern that no power of two repeats)
        part.copy_((torch.arange(len(part), device=DEV) + at * (1 << 24)) % 251)
    scales = torch.zeros(1, (blocks + 15) // 16 * 16, dtype=torch.uint8, device=DEV)
    scales[0, :blocks] = 120 + torch.arange(blocks, device=DEV) % 13
    values = torch.full((1 << bits,), float("nan"))
    levels = torch.from_numpy(no.LEVELS[bits]).float()
    values[:len(levels)], values[1 << (bits - 1):][:len(levels)] = levels, -levels
    values = values.to(DEV)
    dst = torch.full((1, K + 8), 7.0, dtype=torch.bfloat16, device=DEV)
    (norm.flux_mx8_dequantize if bits == 8 else ffn.flux_mx4_dequantize)(q, scales, dst[:, :K])
    torch.cuda.synchronize()
    assert (dst[0, K:] == 7.0).all()
    for a in range(0, K, 1 << 24):
        b = min(K, a + (1 << 24))
        code = q[0, a:b] if bits == 8 else torch.stack([q[0, a // 2:(b + 1) // 2] & 15, q[0, a // 2:(b + 1) // 2] >> 4], 1).view(-1)[:b - a]
        scale = torch.exp2(scales[0, a // 32:(b + 31) // 32].float() - 127).repeat_interleave(32)[:b - a]
        want = (values[code.long()] * scale).to(torch.bfloat16)
        assert torch.equal(dst[0, a:b].view(torch.int16)[~want.isnan()], want.view(torch.int16)[~want.isnan()]) and torch.equal(dst[0, a:b].isnan(), want.isnan()), a
