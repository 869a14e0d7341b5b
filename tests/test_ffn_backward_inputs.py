"""flux_glu_backward asks for what the gradients that are wanted read, and for nothing else: weights for dX, X for the weights' gradients.
Refusals on the CPU; on the GPU the same bits as the call with everything."""
import ctypes

import pytest
import torch

from paper_2406_06858_amd import binding as fb
from paper_2406_06858_amd import ffn

PTR = 4096            # never read: the calls are refused, or have nothing to do
NAMES = ["X", "Wg", "Wu", "G", "U", "dH", "dX", "dWg", "dWu"]


def _status(missing, odd=()):
    p = ffn.glu_problem(64, 128, 256)
    v = [0 if n in missing else PTR + 8 if n in odd else PTR for n in NAMES]
    return ffn.lib().flux_glu_backward(ctypes.byref(p), *v, PTR, 1 << 40, None)


@pytest.mark.parametrize("missing", [("X",), ("Wg",), ("Wu",), ("G",), ("U",), ("dH",), ("X", "dX"), ("Wg", "dWg", "dWu"), ("Wu", "dWg", "dWu"), ("G", "dX", "dWg", "dWu")])
def test_what_is_read_is_asked_for(missing):
    assert _status(missing) == fb.FLUX_ERR_INVALID_ARG


def test_what_is_not_read_is_not_asked_for():
    none = ("dX", "dWg", "dWu")
    for missing in ((), ("X",), ("Wg",), ("Wu",), ("X", "Wg", "Wu")):
        assert _status(none + missing) == fb.FLUX_OK, missing
    assert _status(none, odd=("X",)) == fb.FLUX_ERR_INVALID_ARG


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K,nk", [(1, 64, 72, 1), (130, 136, 264, 0), (130, 136, 264, 1)])
def test_the_same_gradients_without_the_rest(M, N, K, nk):
    draw = lambda seed, *s: torch.randn(s, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).to("cuda:0")      # noqa: E731
    x, g, u, dh = draw(1, M, K), draw(2, M, N), draw(3, M, N), draw(4, M, N)
    w = [draw(i, *((N, K) if nk else (K, N))) for i in (5, 6)]
    p = ffn.glu_problem(M, N, K, w_is_nk=nk)
    ws = torch.zeros(ffn.flux_glu_workspace_bytes(ffn.FLUX_GLU_BACKWARD, p), dtype=torch.uint8, device="cuda:0")
    new = lambda: (torch.full_like(x, 7), torch.full_like(w[0], 7), torch.full_like(w[1], 7))      # noqa: E731
    all_of_it, dx, dw = new(), new(), new()
    ffn.flux_glu_backward(p, x, *w, g, u, dh, *all_of_it, ws)
    ffn.flux_glu_backward(p, None, *w, g, u, dh, dx[0], None, None, ws)
    ffn.flux_glu_backward(p, x, None, None, g, u, dh, None, *dw[1:], ws)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(all_of_it, (dx[0], *dw[1:])))
