"""How many digits an fp32 H of the SiLU block has.  Gates and ups are exact (one number a product), so what H is off by is the activation's
own error: exp2 and reciprocal within 1 ulp = 2 * 2^-24 each, the correction of exp2's argument, the sum 1 + exp, the product with the
gate, the product with up and the store half an ulp each: 2 + 2 + 5 = 9 times 2^-24, and one more for all that is of second order."""
import numpy as np
import pytest
import torch

from paper_2406_06858_amd import ffn

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BOUND = 10 * 2.0 ** -24


def _gates():
    """bf16 numbers of either sign from 2^-8 to 85, where exp is neither 0 nor infinite."""
    g = torch.logspace(-8, np.log2(85), 2000, base=2, dtype=torch.float64).to(torch.bfloat16)
    return torch.cat((g, -g, torch.arange(-85, 86, dtype=torch.float64).to(torch.bfloat16), torch.zeros(5, dtype=torch.bfloat16)))


@pytest.mark.parametrize("M,nk", [(1, 1), (20, 1), (60, 1), (3, 0), (70, 1), (300, 0)])
def test_silu_in_32_bits(M, nk):
    g = _gates()
    N, K = len(g), 64
    assert N % 8 == 0
    X, Wg, Wu = torch.zeros(M, K), torch.zeros(K, N), torch.zeros(K, N)
    X[:, 3], Wg[3], Wu[3] = 1, g.float(), 1.5
    x, wg, wu = (t.to(torch.bfloat16).to(DEV) for t in (X, Wg.t().contiguous() if nk else Wg, Wu.t().contiguous() if nk else Wu))
    p = ffn.glu_problem(M, N, K, w_is_nk=nk, out_dtype="f32")
    n = ffn.flux_glu_workspace_bytes(ffn.FLUX_GLU_FORWARD, p)
    ws = torch.zeros(n, dtype=torch.uint8, device=DEV) if n else None
    H = torch.full((M, N), float("nan"), device=DEV)
    ffn.flux_glu(p, x, wg, wu, H, None, None, ws)
    torch.cuda.synchronize()
    z = g.double().numpy()
    want = 1.5 * z / (1.0 + np.exp(-z))
    off = np.abs(H.cpu().double().numpy() - want) / np.maximum(np.abs(want), 1e-300)
    assert off.max() <= BOUND, f"{off.max() * 2 ** 24:.1f} * 2^-24 at {z[off.max(axis=0).argmax()]}"
