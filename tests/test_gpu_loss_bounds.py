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


def test_rows_that_are_no_whole_lines_of_a_matrix_near_the_limit():
    """X below 2^31 elements as it is, above with its rows rounded up to whole lines.  Rows from the front, the middle and the end, against 64 bits; all others do not
    count, and their gradient is zeros."""
    M, V, K, U = 2_120_000, 16384, 1000, 2.0 ** -24
    gen = torch.Generator(device=DEV).manual_seed(1)
    X = torch.empty(M, K, dtype=torch.bfloat16, device=DEV)
    for part in X.split(1 << 18):
        part.copy_(torch.randn(part.shape, generator=gen, device=DEV))
    W = (torch.randn(V, K, generator=gen, device=DEV) * 2 / K ** 0.5).to(torch.bfloat16)
    rows = torch.cat([torch.arange(at, at + 100, device=DEV) for at in (0, 1 << 20, 2_097_100, M - 100)])          # (2_097_152: where a copy's offsets would wrap)
    target = torch.full((M,), -100, device=DEV)
    target[rows] = torch.randint(0, V, (len(rows),), generator=gen, device=DEV)
    dloss = torch.randn(M, generator=gen, device=DEV)
    p = loss.loss_problem(M, V, K)
    lse, logit, value = (torch.empty(M, device=DEV) for _ in range(3))
    ws = workspace(loss.FLUX_LOSS_FORWARD, p)
    loss.flux_loss(p, X, W, target, lse, logit, value, ws)
    torch.cuda.synchronize()
    x, w, t = X[rows].double(), W.double(), target[rows]
    z = x @ w.t()
    want = torch.logsumexp(z, 1)
    # (as in test_gpu_loss: what a logit is off by, the sums, exp's argument, the logarithm)
    z_off = (x.abs() @ w.abs().t()).amax(1) * (K / 16 + 16) * 2 * U
    off = z_off + ((torch.exp(z - want[:, None]) * (z.amax(1, keepdim=True) - z + 2)).sum(1) * 2 + V / 256 + 64 + (want.abs() + 8) * 4) * U
    z_t = z.gather(1, t[:, None])[:, 0]
    assert ((lse[rows].double() - want).abs() <= off).all()
    assert ((logit[rows].double() - z_t).abs() <= z_off).all()
    assert ((value[rows].double() - (want - z_t)).abs() <= off + z_off + (want - z_t).abs() * U).all()
    others = torch.ones(M, dtype=torch.bool, device=DEV)
    others[rows] = False
    assert not value[others].any() and bool(lse.isfinite().all())
    del ws
    dX, dW = torch.full_like(X, 7.0), torch.empty_like(W)
    loss.flux_loss_backward(p, X, W, target, lse, dloss, dX, dW, workspace(loss.FLUX_LOSS_BACKWARD, p))
    torch.cuda.synchronize()
    dz = (torch.exp(z - lse[rows].double()[:, None]) - torch.nn.functional.one_hot(t, V)) * dloss[rows].double()[:, None]
    # (dZ's and the results' roundings, 2^-8 each; zeros add nothing to a sum's error)
    assert ((dX[rows].double() - dz @ w).abs() <= 2.5 * 2.0 ** -8 * (dz.abs() @ w.abs())).all()
    assert ((dW.double() - dz.t() @ x).abs() <= 2.5 * 2.0 ** -8 * (dz.abs().t() @ x.abs())).all()
    assert not (dX.view(torch.int16) != 0)[others].any()


@pytest.mark.parametrize("M,V,dtype", [(1, 2, "f32"), (3, 3, "bf16")])
def test_the_widest_rows(M, V, dtype):
    """2^28 numbers; X is zeros but for a thousand columns, the first and the last among them, so that the logits are sums of few numbers."""
    K, U = 1 << 28, 2.0 ** -24
    gen = torch.Generator(device=DEV).manual_seed(M)
    at = torch.randint(0, K, (1000,), generator=gen, device=DEV).unique()
    at[0], at[-1] = 0, K - 1
    X = torch.zeros(M, K, dtype=torch.bfloat16, device=DEV)
    X[:, at] = torch.randn(M, len(at), generator=gen, device=DEV).to(torch.bfloat16)
    W = torch.empty(V, K, dtype=torch.bfloat16, device=DEV)
    for row in W:
        row.copy_(torch.randn(K, generator=gen, device=DEV) * 0.03)
    target, dloss = torch.arange(M, device=DEV) % V, torch.randn(M, generator=gen, device=DEV)
    p = loss.loss_problem(M, V, K, dx_dtype=dtype, dw_dtype=dtype)
    lse, logit, value = (torch.empty(M, device=DEV) for _ in range(3))
    loss.flux_loss(p, X, W, target, lse, logit, value, workspace(loss.FLUX_LOSS_FORWARD, p))
    x, w = X[:, at].double(), W[:, at].double()
    z = x @ w.t()
    z_off = (x.abs() @ w.abs().t()).amax(1) * (len(at) + 16) * 2 * U          # (each of them in a sum of its own, at worst)
    want = torch.logsumexp(z, 1)
    assert ((lse.double() - want).abs() <= z_off + 100 * U).all() and ((logit.double() - z.gather(1, target[:, None])[:, 0]).abs() <= z_off).all()
    t = (torch.bfloat16, torch.float32)[p.dx_dtype]
    dX, dW = torch.full((M, K), 7.0, dtype=t, device=DEV), torch.full((V, K), 7.0, dtype=t, device=DEV)
    loss.flux_loss_backward(p, X, W, target, lse, dloss, dX, dW, workspace(loss.FLUX_LOSS_BACKWARD, p))
    torch.cuda.synchronize()
    dz = (torch.exp(z - lse.double()[:, None]) - torch.nn.functional.one_hot(target, V)) * dloss.double()[:, None]
    # (dZ's rounding to bf16 and the result's, 2^-8 each of the sum of magnitudes; piece by piece, for memory)
    for a in range(0, K, 1 << 25):
        part = W[:, a:a + (1 << 25)].double()
        assert ((dX[:, a:a + (1 << 25)].double() - dz @ part).abs() <= 2.5 * 2.0 ** -8 * (dz.abs() @ part.abs())).all()
        part = X[:, a:a + (1 << 25)].double()
        assert ((dW[:, a:a + (1 << 25)].double() - dz.t() @ part).abs() <= 2.5 * 2.0 ** -8 * (dz.abs().t() @ part.abs())).all()
