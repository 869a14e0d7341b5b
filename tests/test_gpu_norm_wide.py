"""The norm and its gradients on the widest rows that it takes, 2^30 numbers: more columns of dW than one direction of a grid has threads for."""
import pytest
import torch

from paper_2406_06858_amd import norm

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


@pytest.mark.parametrize("M,K", [(1, 1 << 30), (2, (1 << 29) + 33)])
def test_the_widest_rows(M, K):
    """Rows of ones and minus ones: their mean square is exactly 1, and with eps = 0 so is 1 / rms.  dY is zeros but for a thousand columns."""
    gen = torch.Generator(device=DEV).manual_seed(K)
    S = torch.empty(M, K, dtype=torch.bfloat16, device=DEV)
    for part in S.view(-1).split(1 << 26):
        part.copy_(torch.randint(0, 2, part.shape, generator=gen, device=DEV) * 2 - 1)
    W = torch.empty(K, dtype=torch.bfloat16, device=DEV)
    for part in W.split(1 << 26):
        part.copy_(1 + 0.2 * torch.randn(part.shape, generator=gen, device=DEV))
    p = norm.norm_problem(M, K, eps=0.0)
    Y, rstd = torch.full((M, K), 7.0, dtype=torch.bfloat16, device=DEV), torch.empty(M, device=DEV)
    norm.flux_norm(p, S, None, W, None, Y, None, rstd)
    # (a lane's own sum of ones is a whole number below 2^24, and so are the powers of two of sums of all lanes)
    assert ((rstd - 1).abs() <= 4 * U).all()
    for a in range(0, K, 1 << 26):
        b = min(K, a + (1 << 26))
        want = S[:, a:b].float() * W[a:b].float()
        assert ((Y[:, a:b].float() - want).abs() <= want.abs() * (2.0 ** -8 + 8 * U)).all()
    at = torch.randint(0, K, (1000,), generator=gen, device=DEV).unique()
    at[0], at[-1] = 0, K - 1
    dY = torch.zeros(M, K, dtype=torch.bfloat16, device=DEV)
    dY[:, at] = torch.randn(M, len(at), generator=gen, device=DEV).to(torch.bfloat16)
    dR, dW = Y.fill_(7.0), torch.full((K,), 7.0, device=DEV)
    ws = torch.empty(norm.flux_norm_workspace_bytes(p), dtype=torch.uint8, device=DEV).fill_(255)
    norm.flux_norm_backward(p, dY, S, W, rstd, None, dR, None, dW, ws)
    torch.cuda.synchronize()
    r, dy, s, w = rstd.double()[:, None], dY[:, at].double(), S[:, at].double(), W[at].double()
    dw64 = (dy * s * r).sum(0)
    assert ((dW[at].double() - dw64).abs() <= (dy * s).abs().sum(0) * 8 * U).all()
    rest = torch.ones(K, dtype=torch.bool, device=DEV)
    rest[at] = False
    assert not dW[rest].any()
    # the mean of a thousand numbers over 2^30: next to nothing, in every column
    mean = (dy * w * s * r).sum(1, keepdim=True) / K
    off = (dy * w * s).abs().sum(1, keepdim=True) / K * 2.0 ** -8
    got, want = dR[:, at].double(), r * (dy * w - s * r * mean)
    assert ((got - want).abs() <= want.abs() * (2.0 ** -8 + 8 * U) + off).all()
    for a in range(0, K, 1 << 26):
        b = min(K, a + (1 << 26))
        want = -S[:, a:b].double() * r * r * mean
        assert (((dR[:, a:b].double() - want).abs() <= want.abs() * (2.0 ** -8 + 8 * U) + off) | ~rest[a:b]).all()
