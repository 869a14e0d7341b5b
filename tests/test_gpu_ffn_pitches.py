"""The gated block on matrices whose rows lie so far apart that the offsets of rows past the last one pass 32 bits: the bits of rows side by side, whatever lies
between the rows."""
import pytest
import torch

from paper_2406_06858_amd import ffn

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FAR = 150_000_000


def _placed(t, ld):
    rows, cols = t.shape
    buf = torch.full(((rows - 1) * (ld or cols) + cols,), float("nan"), dtype=t.dtype, device=DEV)
    view = buf.as_strided((rows, cols), (ld or cols, 1))
    view.copy_(t)
    return view


def _workspace(op, p):
    ws = torch.empty(max(ffn.flux_glu_workspace_bytes(op, p), 16), dtype=torch.uint8, device=DEV)
    ffn.flux_ffn_init(ws)
    return ws


@pytest.mark.parametrize("M,N,K,nk,ldx,ldw,ldh", [(40, 64, 8, 0, 0, FAR, 0), (40, 8, 64, 1, 0, FAR, 0), (14, 64, 64, 0, FAR, 0, 0), (14, 64, 64, 1, FAR, 0, FAR), (3, 16, 8, 0, FAR, FAR, FAR)])
def test_rows_far_apart(M, N, K, nk, ldx, ldw, ldh):
    g = torch.Generator(device=DEV).manual_seed(1)
    draw = lambda *shape: torch.randn(shape, generator=g, device=DEV).to(torch.bfloat16)      # noqa: E731
    shape = (N, K) if nk else (K, N)
    X, Wg, Wu, dH = draw(M, K), draw(*shape), draw(*shape), draw(M, N)
    got = []
    for lx, lw, lh in ((0, 0, 0), (ldx, ldw, ldh)):
        p = ffn.glu_problem(M, N, K, w_is_nk=nk, ldx=lx, ldw=lw, ldh=lh)
        x, wg, wu, dh, h, gate, up = (_placed(t, ld) for t, ld in ((X, lx), (Wg, lw), (Wu, lw), (dH, lh), (dH, lh), (dH, lh), (dH, lh)))
        ffn.flux_glu(p, x, wg, wu, h, gate, up, _workspace(ffn.FLUX_GLU_FORWARD, p))
        dx, dwg, dwu = _placed(X, lx), _placed(Wg, lw), _placed(Wu, lw)
        ffn.flux_glu_backward(p, x, wg, wu, gate, up, dh, dx, dwg, dwu, _workspace(ffn.FLUX_GLU_BACKWARD, p))
        torch.cuda.synchronize()
        got.append([t.contiguous() for t in (h, gate, up, dx, dwg, dwu)])
        del x, wg, wu, dh, h, gate, up, dx, dwg, dwu
        torch.cuda.empty_cache()
    for a, b in zip(*got):
        assert torch.isfinite(a).all() and torch.equal(a, b)
