"""The loss's gradients on matrices with numbers behind their end that are none: nothing of them gets into a result.  (Which places a launch reads is checked without a GPU in
test_loss_launches.py.)"""
import pytest
import torch

from paper_2406_06858_amd import ffn, loss

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def workspace(op, p):
    ws = torch.full(((loss.flux_loss_workspace_bytes(op, p) + 3) // 4,), float("nan"), device=DEV)
    ffn.flux_ffn_init(ws)
    return ws


def behind(t, rows=64):
    """t's numbers in front of `rows` rows of NaN, in one buffer."""
    buf = torch.full((t.shape[0] + rows, t.shape[1]), float("nan"), dtype=t.dtype, device=DEV)
    buf[:t.shape[0]] = t
    return buf[:t.shape[0]], buf[t.shape[0]:]


@pytest.mark.parametrize("M,V,K,piece", [(256, 4095, 256, 0), (256, 4089, 256, 0), (512, 505, 256, 0), (128, 63, 128, 0), (256, 1983, 512, 640), (64, 4093, 256, 0)])
@pytest.mark.parametrize("dx", ["bf16", "f32"])
def test_what_lies_behind_the_matrices(M, V, K, piece, dx):
    """The widths of a last slab of which whole vectors of dZ, but not W's rows, fill all 64; M and K are whole tiles.  The same bits as with zeros there."""
    gen = torch.Generator(device=DEV).manual_seed(V)
    X = torch.randn(M, K, generator=gen, device=DEV).to(torch.bfloat16)
    W = (torch.randn(V, K, generator=gen, device=DEV) * 2 / K ** 0.5).to(torch.bfloat16)
    target, dloss = torch.randint(0, V, (M,), generator=gen, device=DEV), torch.randn(M, generator=gen, device=DEV)
    lse = torch.logsumexp(X.double() @ W.double().t(), 1).float()
    p = loss.loss_problem(M, V, K, piece=piece, dx_dtype=dx)
    got = []
    for fill in (0.0, float("nan")):
        x, x_end = behind(X)
        w, w_end = behind(W)
        for end in (x_end, w_end):
            end.fill_(fill)
        dX = torch.full((M, K), 7.0, dtype=(torch.bfloat16, torch.float32)[p.dx_dtype], device=DEV)
        dW = torch.full((V + 8, K), 7.0, dtype=torch.bfloat16, device=DEV)
        loss.flux_loss_backward(p, x, w, target, lse, dloss, dX, dW[:V], workspace(loss.FLUX_LOSS_BACKWARD, p))
        torch.cuda.synchronize()
        assert (dW[V:] == 7.0).all()
        got.append((dX, dW))
    assert bool(got[1][0].isfinite().all()) and bool(got[1][1].isfinite().all())
    for a, b in zip(*got):
        assert torch.equal(a, b)
    # against 64 bits: dZ's and the result's roundings, half a step of bf16 each, of the sum of magnitudes; Z's error is a hundredth of those at these widths
    z = X.double() @ W.double().t()
    dz = (torch.exp(z - lse.double()[:, None]) - torch.nn.functional.one_hot(target, V)) * dloss.double()[:, None]
    assert ((got[1][0].double() - dz @ W.double()).abs() <= 2.5 * 2.0 ** -8 * (dz.abs() @ W.double().abs())).all()
