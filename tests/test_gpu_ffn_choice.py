"""What the caller's tile_config and split_k choose.  Both kernels add the same products up in another order, so that bits tell them apart:
in fp32, of random numbers."""
import pytest
import torch

from paper_2406_06858_amd import ffn

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FEW = ffn.flux_ffn_tile_config_count()


def _h(M, N, K, **choice):
    draw = lambda seed, *s: torch.randn(s, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).to(DEV)      # noqa: E731
    x, wg, wu = draw(1, M, K), draw(2, N, K), draw(3, N, K)
    p = ffn.glu_problem(M, N, K, w_is_nk=1, out_dtype="f32", **choice)
    n = ffn.flux_glu_workspace_bytes(ffn.FLUX_GLU_FORWARD, p)
    h = torch.full((M, N), float("nan"), device=DEV)
    ffn.flux_glu(p, x, wg, wu, h, None, None, torch.zeros(n, dtype=torch.uint8, device=DEV) if n else None)
    torch.cuda.synchronize()
    x, wg, wu = (t.double() for t in (x, wg, wu))
    g, u = x @ wg.t(), x @ wu.t()
    # a sum of K products is off by at most K 2^-23 of the sum of their magnitudes, a slope is at most 1.13
    eg, eu = (K * 2.0 ** -23 * (x.abs() @ w.abs().t()) for w in (wg, wu))
    a = g * torch.sigmoid(g)
    assert bool(((h - a * u).abs() <= 1.01 * (1.13 * eg * u.abs() + a.abs() * eu + 1.13 * eg * eu) + 2.0 ** -20 * (a * u).abs()).all())
    return h, n


@pytest.mark.parametrize("M,N,K", [(1, 264, 1032), (8, 520, 520), (40, 264, 1032)])
def test_no_cut_keeps_the_kernel_for_few_rows(M, N, K):
    few, n = _h(M, N, K, tile_config=FEW)
    assert n == 0
    for choice in ({}, {"split_k": 1}):
        h, n = _h(M, N, K, **choice)
        assert n == 0 and torch.equal(h, few), choice
    tiles, _ = _h(M, N, K, split_k=4)
    assert not torch.equal(tiles, few)
