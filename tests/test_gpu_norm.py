"""The root-mean-square norm and its backward pass on the GPU against the oracle in 64 bits.

Bounds.  A half step of a type is `torch.finfo(t).eps / 2` of a value: U = 2^-24 in fp32.  A sum of n numbers whose lanes add at most n / 16 one
after another and then meet in a tree is off by at most (n / 16 + 16) U of the sum of magnitudes, products and all; 1 / rms by half of that for the mean, and
4 U for the mean's division, eps, the root and the division.
"""
import numpy as np
import pytest
import torch

from oracle import norm_loss_oracle as no
from paper_2406_06858_amd import ffn, norm

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24


def half(dtype):
    return torch.finfo(TORCH[dtype]).eps / 2


def tree(n):
    return (n / 16 + 16) * U


def f64(t):
    return t.detach().cpu().double().numpy()


def assert_within(got, want, bound, what=""):
    g = f64(got)
    assert g.shape == want.shape, (what, g.shape, want.shape)
    bad = ~(np.abs(g - want) <= bound)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} out of bounds, first at {np.argwhere(bad)[0]}: {g[bad][0]} for {want[bad][0]}"


def padded(rows, cols, pitch, dtype, fill=7.0):
    """A view of [rows, cols] with a pitch, inside a buffer that holds `fill` everywhere else; and the buffer."""
    buf = torch.full((rows * pitch + 8,), fill, dtype=dtype, device=DEV)
    return buf[:rows * pitch].view(rows, pitch)[:, :cols], buf


def case(M, K, seed, x="bf16", s="bf16", w="bf16", pad=(0, 0, 0)):
    gen = torch.Generator().manual_seed(seed)
    draw = lambda *shape: torch.randn(shape, generator=gen)                                                 # noqa: E731
    X, _ = padded(M, K, K + pad[0], TORCH[x])
    R, _ = padded(M, K, K + pad[1], TORCH[s])
    X.copy_(draw(M, K))
    R.copy_(draw(M, K) * torch.exp(draw(1, K)))
    return X, R, (1 + 0.2 * draw(K)).to(TORCH[w]).to(DEV)


def run_forward(X, R, W, out, eps, pad=(0, 0, 0), in_place=False, rstd=True):
    M, K = X.shape
    p = norm.norm_problem(M, K, x_dtype=X.dtype, s_dtype=R.dtype if R is not None else X.dtype, w_dtype=W.dtype, out=out, eps=eps,
                          ldx=K + pad[0], lds=K + pad[1], ldy=K + pad[2])
    S = None if R is None else R if in_place else padded(M, K, K + pad[1], R.dtype)[0]
    scales = None
    if out in ("mx4", "mx8"):
        row = (ffn.flux_mx4_row_bytes if out == "mx4" else norm.flux_mx8_row_bytes)(K)
        Y = torch.full((M + 1, row), 0xAA, dtype=torch.uint8, device=DEV)
        scales = torch.full((M + 1, ffn.flux_mx4_scale_row_bytes(K)), 0xAA, dtype=torch.uint8, device=DEV)
        whole = Y
    else:
        Y, whole = padded(M, K, K + pad[2], TORCH[out])
    r = torch.full((M + 1,), 7.0, device=DEV) if rstd else None
    norm.flux_norm(p, X, R, W, S, Y, scales, r)
    torch.cuda.synchronize()
    return S, Y, scales, r, whole


SHAPES = [(1, 1), (1, 7), (3, 8), (2, 64), (5, 127), (9, 128), (33, 129), (4, 500), (7, 512), (3, 1000), (17, 1024), (2, 1031), (5, 2048), (3, 2880), (2, 4096),
          (3, 5111), (66, 8192), (2, 8200), (2, 12288), (2, 12284), (3, 12299), (2, 16384), (2, 16391), (2, 32761), (2, 32768), (1, 33000), (2, 70001)]


@pytest.mark.parametrize("M,K", SHAPES)
@pytest.mark.parametrize("x,s,w,out", [("bf16", "bf16", "bf16", "bf16"), ("bf16", "f32", "f32", "f32"), ("f32", "bf16", "bf16", "bf16"), ("f32", "f32", "f32", "bf16"),
                                       ("bf16", None, "bf16", "f32"), ("f32", None, "bf16", "f32"), ("bf16", "bf16", "f32", "f32")])
def test_forward(M, K, x, s, w, out):
    pad = (3, 5, 1) if K % 2 else (0, 8, 24)
    X, R, W = case(M, K, M * 100003 + K, x, s or "bf16", w, pad)
    eps = 1e-5
    before = None if s is None else f64(R)
    S, Y, _, r, whole = run_forward(X, R if s else None, W, out, eps, pad)
    if s:
        want = f64(X) + before
        assert_within(S, want, np.abs(want) * (U + half(s)) + 2.0 ** -133, "S")
        assert (f64(R) == before).all()
    y, rstd = no.norm(f64(S if s else X), f64(W), eps)
    off = tree(K) / 2 + 4 * U
    assert_within(r[:M], rstd, rstd * off, "rstd")
    assert_within(Y, y, np.abs(y) * (off + 2 * U + half(out)), "Y")
    assert r[M] == 7.0 and (whole.view(-1)[M * (K + pad[2]):] == 7.0).all()
    if M > 1 and pad[2]:
        assert (whole[:M * (K + pad[2])].view(M, -1)[:, K:] == 7.0).all()


@pytest.mark.parametrize("M,K", [(1, 1), (3, 31), (2, 33), (5, 500), (3, 512), (2, 513), (4, 2047), (3, 5111), (64, 8192), (2, 12288), (1, 33001)])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("s", ["bf16", "f32"])
def test_blocks(M, K, bits, s):
    X, R, W = case(M, K, 7 * M + K, s=s)
    S, q, scales, r, _ = run_forward(X, R, W, f"mx{bits}", 1e-5)
    y, _ = no.norm(f64(S), f64(W), 1e-5)
    off = tree(K) / 2 + 6 * U                             # of every number before it is coded
    kb = -(-K // 32)
    q, scales = q.cpu().numpy(), scales.cpu().numpy()
    assert (q[M] == 0xAA).all() and (scales[M] == 0xAA).all() and not scales[:M, kb:].any()
    q, byte = q[:M], scales[:M, :kb]
    lo, hi = no.blocks(y * (1 - off), bits)[1], no.blocks(y * (1 + off), bits)[1]
    assert ((byte == lo) | (byte == hi)).all()
    codes = (q.reshape(M, kb, 32) if bits == 8 else np.stack([q & 15, q >> 4], axis=-1).reshape(M, kb, 32))
    got = no.block_values(codes, byte, bits)
    assert not got[:, K:].any()
    # nobody is further from a number than the nearest level is, but for what the number itself may be off by
    unit = 2.0 ** (byte.astype(np.float64) - 127).repeat(32, axis=1)[:, :K]
    levels = no.LEVELS[bits]
    held = np.minimum(np.abs(y) / unit, levels[-1])
    near = np.minimum(np.abs(held - levels[np.clip(np.searchsorted(levels, held), 0, len(levels) - 1)]),
                      np.abs(held - levels[np.clip(np.searchsorted(levels, held) - 1, 0, len(levels) - 1)]))
    assert (np.abs(np.abs(got[:, :K]) / unit - held) <= near + 2 * off * held).all()
    assert ((got[:, :K] == 0) | (np.sign(got[:, :K]) == np.sign(y))).all()


def special_numbers():
    """Every bf16 number, ties and their neighbours in fp32 around them, in blocks of one exponent and mixed."""
    every = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).float()
    ties = []
    for levels in (no.E2M1, no.E4M3):
        mid = torch.from_numpy((levels[1:] + levels[:-1]) / 2).float()
        bits = mid.view(torch.int32)
        t = torch.cat([mid, (bits + 1).view(torch.float32), (bits - 1).view(torch.float32)])
        for top in (float(levels[-1]), float(levels[-1]) * 1.14):
            # a block of 31 of them under the one number that sets the scale
            t = torch.cat([t, t.new_zeros(-len(t) % 31)])
            b = torch.cat([t.view(-1, 31), t.new_full((len(t) // 31, 1), top)], 1).reshape(-1)
            ties += [b, -b, b * 2.0 ** 20, b * 2.0 ** -120, b * 2.0 ** -126, b * 2.0 ** 110]
            t = torch.cat([mid, (bits + 1).view(torch.float32), (bits - 1).view(torch.float32)])
    tiny = torch.arange(1, 4097, dtype=torch.int32).view(torch.float32)
    return torch.cat([every] + ties + [tiny, tiny * 2.0 ** 10])


@pytest.mark.parametrize("bits", [4, 8])
def test_coding_bit_for_bit(bits):
    """A row of ones has a mean square of exactly 1: with eps = 0 Y is W."""
    w = special_numbers()
    K = len(w)
    X, W = torch.ones(2, K, dtype=torch.bfloat16, device=DEV), w.to(DEV)
    _, q, scales, r, _ = run_forward(X, None, W, f"mx{bits}", 0.0)
    assert (r[:2] == 1).all()
    codes, byte = no.blocks(w.double().numpy()[None], bits)
    want_q, want_s = no.packed(codes, byte, bits)
    for row in range(2):
        assert (scales[row].cpu().numpy() == want_s[0]).all()
        assert (q[row].cpu().numpy() == want_q[0]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K", [32 * 256, 32 * 256 - 11, 5])
def test_8_bit_blocks_read_back(dtype, K):
    """Every code under every byte."""
    kb = -(-K // 32)
    rng = np.random.default_rng(K)
    codes = np.stack([np.arange(kb * 32, dtype=np.int64).reshape(kb, 32) % 256, rng.integers(0, 256, (kb, 32))]).astype(np.uint8)
    byte = np.stack([np.arange(kb) % 256, rng.integers(0, 256, kb)]).astype(np.uint8)
    q, s = no.packed(codes, byte, 8)
    dst, whole = padded(2, K, K + 3, TORCH[dtype])
    norm.flux_mx8_dequantize(torch.from_numpy(q).to(DEV), torch.from_numpy(s).to(DEV), dst)
    want = torch.from_numpy(no.block_values(codes, byte, 8)[:, :K]).to(TORCH[dtype])       # (64 bits to either type in one rounding: 4 significant bits)
    got = dst.cpu()
    assert (got.isnan() == want.isnan()).all() and (got[~want.isnan()] == want[~want.isnan()]).all()
    assert (whole[:2 * (K + 3)].view(2, -1)[:, K:] == 7.0).all()


def test_8_bit_blocks_read_back_refuse_views():
    q, s = (torch.zeros(4, n, dtype=torch.uint8, device=DEV) for n in (64, 16))
    dst = torch.zeros(4, 64, dtype=torch.bfloat16, device=DEV)
    for bad in ((q[:, ::2], s, dst), (q[:2], s, dst), (q, s[:2], dst), (q, s, dst.t()), (q, s, dst[:1].expand(4, 64)), (q.cpu(), s, dst)):
        with pytest.raises(ValueError):
            norm.flux_mx8_dequantize(*bad)


@pytest.mark.parametrize("s", ["bf16", "f32"])
@pytest.mark.parametrize("M,K", [(3, 128), (2, 8192), (5, 5111), (2, 40000)])
def test_in_place(M, K, s):
    X, R, W = case(M, K, 11, s=s)
    R2 = R.clone()
    S, Y, _, r, _ = run_forward(X, R, W, "f32", 1e-6)
    S2, Y2, _, r2, _ = run_forward(X, R2, W, "f32", 1e-6, in_place=True)
    assert S2.data_ptr() == R2.data_ptr()
    assert torch.equal(S, S2) and torch.equal(Y, Y2) and torch.equal(r, r2)


def test_rows_of_zeros_and_of_what_is_not_finite():
    M, K = 6, 1000
    X, R, W = case(M, K, 3)
    X[1], R[1] = 0, 0
    X[2, 500], X[4, 3] = float("nan"), float("inf")
    for out in ("f32", "mx4", "mx8"):
        S, Y, scales, r, _ = run_forward(X, R, W, out, 1e-5)
        assert abs(float(r[1]) - 1e-5 ** -0.5) < 1e-3 and bool(r[2].isnan()) and float(r[4]) == 0
        good = [0, 3, 5]
        alone = run_forward(X[good].contiguous(), R[good].contiguous(), W, out, 1e-5)
        assert torch.equal(S[good], alone[0]) and torch.equal(Y[good], alone[1][:3]) and torch.equal(r[good], alone[3][:3])
        if out == "f32":
            assert not Y[1].any() and bool(Y[2].isnan().all()) and bool(Y[4, 3].isnan()) and not Y[4, 4:].any()
        else:
            assert (scales[2, :32] == 255).all() and not scales[1].any() and scales[4, 0] == 255 and not scales[4, 1:].any()
            assert out != "mx4" or not Y[2].any()
    # (33 numbers: two blocks, fourteen bytes of padding, which are zeros in a row of NaN as well)
    X, R, W = case(3, 33, 4)
    X[1, 2] = float("nan")
    for out in ("mx4", "mx8"):
        scales = run_forward(X, R, W, out, 1e-5)[2]
        assert (scales[1, :2] == 255).all() and not scales[:3, 2:].any()


def test_a_column_that_dwarfs_the_others():
    X, R, W = case(2, 8192, 5, s="f32")
    R[:, 77] = 1e15
    S, Y, _, r, _ = run_forward(X, R, W, "f32", 1e-5)
    y, rstd = no.norm(f64(S), f64(W), 1e-5)
    off = tree(8192) / 2 + 4 * U
    assert_within(r[:2], rstd, rstd * off)
    assert_within(Y, y, np.abs(y) * (off + 3 * U))


# ---- backward -----------------------------------------------------------------------------------------------------
def run_backward(p, dY, S, W, rstd, dS, want=("dR", "dX", "dW"), pad=(0, 0, 0), in_place=False, dW=None):
    M, K = S.shape
    ws = torch.zeros(max(norm.flux_norm_workspace_bytes(p), 1), dtype=torch.uint8, device=DEV)
    dR = (dS if in_place else padded(M, K, K + pad[1], S.dtype)[0]) if "dR" in want else None
    dX = padded(M, K, K + pad[0], (torch.bfloat16, torch.float32)[p.x_dtype])[0] if "dX" in want else None
    if dW is None and "dW" in want:
        dW = torch.full((K,), 7.0, dtype=(torch.bfloat16, torch.float32)[p.dw_dtype], device=DEV)
    norm.flux_norm_backward(p, dY, S, W, rstd, dS, dR, dX, dW, ws if "dW" in want else None)
    torch.cuda.synchronize()
    return dR, dX, dW


def backward_bounds(dy, s, w, r, ds):
    """Want and bound of dR and dW but for their last rounding."""
    dr, dw = no.norm_backward(dy, s, w, r, ds)
    M, K = s.shape
    h, g = np.abs(s * r[:, None]), np.abs(dy * w)
    mean = (g * h).mean(axis=1, keepdims=True)
    return dr, (np.abs(r)[:, None] * (g + h * mean) + np.abs(ds)) * 8 * U + np.abs(r)[:, None] * h * mean * tree(K), dw, np.abs(dy * h).sum(axis=0) * (M + 80) * U


@pytest.mark.parametrize("M,K", SHAPES + [(300, 64), (700, 1024), (1030, 129)])
@pytest.mark.parametrize("x,s,w,y,dw", [("bf16", "bf16", "bf16", "bf16", "f32"), ("bf16", "f32", "f32", "bf16", "bf16"), ("f32", "bf16", "bf16", "f32", "f32"),
                                        ("f32", "f32", "f32", "f32", "f32")])
def test_backward(M, K, x, s, w, y, dw):
    pad = (3, 5, 1) if K % 2 else (0, 8, 24)
    _, S, W = case(M, K, M * 7 + K, x, s, w, pad)
    dY, dS = padded(M, K, K + pad[2], TORCH[y])[0], padded(M, K, K + pad[1], TORCH[s])[0]
    gen = torch.Generator().manual_seed(K)
    dY.copy_(torch.randn(M, K, generator=gen))
    dS.copy_(torch.randn(M, K, generator=gen))
    rstd = torch.from_numpy(no.norm(f64(S), f64(W), 1e-5)[1]).float().to(DEV)
    p = norm.norm_problem(M, K, x_dtype=x, s_dtype=s, w_dtype=w, out=y, dw_dtype=dw, ldx=K + pad[0], lds=K + pad[1], ldy=K + pad[2])
    args = f64(dY), f64(S), f64(W), f64(rstd), f64(dS)
    dr, dr_off, dw64, dw_off = backward_bounds(*args)
    dR, dX, dW = run_backward(p, dY, S, W, rstd, dS, pad=pad)
    assert_within(dR, dr, dr_off + (np.abs(dr) + dr_off) * half(s), "dR")
    assert_within(dX, dr, dr_off + (np.abs(dr) + dr_off) * half(x), "dX")
    assert_within(dW, dw64, dw_off + (np.abs(dw64) + dw_off) * half(dw), "dW")
    # each by itself, dR in dS's place, and once more: the same bits
    assert torch.equal(run_backward(p, dY, S, W, rstd, dS, ("dR",), pad)[0], dR)
    assert torch.equal(run_backward(p, dY, S, W, rstd, dS, ("dX",), pad)[1], dX)
    assert torch.equal(run_backward(p, dY, S, W, rstd, dS, ("dW",), pad)[2], dW)
    assert torch.equal(run_backward(p, dY, S, W, rstd, dS, ("dR", "dW"), pad, in_place=True)[0], dR)


@pytest.mark.parametrize("dw", ["bf16", "f32"])
@pytest.mark.parametrize("M,K", [(1, 40), (40, 2048), (130, 5111)])
def test_backward_without_a_stream_and_added_up(M, K, dw):
    _, S, W = case(M, K, 21, s="f32")
    dY = torch.randn(M, K, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).to(DEV)
    rstd = torch.from_numpy(no.norm(f64(S), f64(W), 1e-5)[1]).float().to(DEV)
    zero = np.zeros((M, K))
    dr, dr_off, dw64, dw_off = backward_bounds(f64(dY), f64(S), f64(W), f64(rstd), zero)
    p = norm.norm_problem(M, K, s_dtype="f32", dw_dtype=dw, dw_accumulate=1)
    held = torch.randn(K, generator=torch.Generator().manual_seed(9)).to(TORCH[dw]).to(DEV)
    want = dw64 + f64(held)
    dR, _, dW = run_backward(p, dY, S, W, rstd, None, ("dR", "dW"), dW=held)
    assert_within(dR, dr, dr_off + np.abs(dr) * half("f32") * 2)
    assert_within(dW, want, dw_off + (np.abs(want) + dw_off) * (half(dw) + U))


@pytest.mark.parametrize("M,K,ld", [(15, 1029, 150_000_001), (3, 40000, 1_073_000_000)])
def test_pitches_whose_offsets_pass_32_bits(M, K, ld):
    """The bits of rows side by side."""
    X, S, W = case(M, K, 5, s="f32")
    dY = torch.randn(M, K, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).to(DEV)
    got = []
    for pitch in (K, ld):
        views = []
        for t in (X, S, dY, S, X, X, S):                                          # X, R, dY; S, Y, dX, dR
            buf = torch.full(((M - 1) * pitch + K,), float("nan"), dtype=t.dtype, device=DEV)
            views.append(buf.as_strided((M, K), (pitch, 1)))
            views[-1].copy_(t)
        p = norm.norm_problem(M, K, s_dtype="f32", ldx=pitch, lds=pitch, ldy=pitch)
        rstd, dW = torch.empty(M, device=DEV), torch.empty(K, device=DEV)
        norm.flux_norm(p, views[0], views[1], W, views[3], views[4], None, rstd)
        ws = torch.zeros(norm.flux_norm_workspace_bytes(p), dtype=torch.uint8, device=DEV)
        norm.flux_norm_backward(p, views[2], views[3], W, rstd, None, views[6], views[5], dW, ws)
        torch.cuda.synchronize()
        got.append([rstd, dW] + [v.contiguous() for v in views[3:]])
        del views, buf
        torch.cuda.empty_cache()
    for a, b in zip(*got):
        assert torch.isfinite(a).all() and torch.equal(a, b)


@pytest.mark.parametrize("K", [1, 3])
def test_more_rows_than_a_grid_is_wide(K):
    M = (1 << 27) + 33 if K == 1 else (1 << 24) + 5
    X = torch.randn(1 << 16, K, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).to(torch.bfloat16).repeat(-(-M // (1 << 16)), 1)[:M]
    W = torch.full((K,), 2.0, device=DEV)
    p = norm.norm_problem(M, K, w_dtype="f32")
    Y, r = torch.zeros_like(X), torch.zeros(M, device=DEV)
    norm.flux_norm(p, X, None, W, None, Y, None, r)
    n = 1 << 16
    assert torch.equal(Y[-(M % n or n):], Y[:M % n or n]) and torch.equal(Y[n:2 * n], Y[:n]) and torch.equal(r[M - M % n:], r[:M % n])
    y, rstd = no.norm(f64(X[:1000]), f64(W), 1e-5)
    assert_within(r[:1000], rstd, rstd * (tree(K) + 4 * U))
    assert_within(Y[:1000], y, np.abs(y) * (tree(K) + 6 * U + half("bf16")))
    # the gradient: of the last rows as of the first
    dX = torch.zeros_like(X)
    norm.flux_norm_backward(p, Y, X, W, r, None, None, dX)
    assert torch.equal(dX[M - M % n:], dX[:M % n]) and torch.equal(dX[n:2 * n], dX[:n])


def test_nothing_asked_for():
    p = norm.norm_problem(4, 64)
    t = torch.zeros(4, 64, dtype=torch.bfloat16, device=DEV)
    norm.flux_norm_backward(p, t, t, t[0], torch.ones(4, device=DEV))


def test_backward_is_the_forward_pass_slope():
    """Against differences of the forward pass itself, in fp32: a step of 2^-7 along d changes Y . dY by the gradient times the step, off by the rounding of
    both ends (2^-24 of every term of the sums) over the step, and by the third derivative, which a central difference leaves to the step's square."""
    M, K = 3, 64
    gen = torch.Generator().manual_seed(5)
    S, W, dY, d = (torch.randn(*shape, generator=gen).to(DEV) for shape in ((M, K), (K,), (M, K), (M, K)))
    p = norm.norm_problem(M, K, x_dtype="f32", s_dtype="f32", w_dtype="f32", out="f32")
    _, _, _, r, _ = run_forward(S, None, W, "f32", 1e-5)
    dR, _, dW = run_backward(p, dY, S, W, r[:M].contiguous(), None, ("dR", "dW"))
    h = 2.0 ** -7
    ends = [run_forward(S + e * d, None, W, "f32", 1e-5)[1] for e in (h, -h)]
    slope = ((f64(ends[0]) - f64(ends[1])) * f64(dY)).sum() / (2 * h)
    scale = (np.abs(f64(ends[0])) * np.abs(f64(dY))).sum()
    assert abs(slope - (f64(dR) * f64(d)).sum()) <= scale * (32 * U / h + 8 * h * h)
    along = (f64(W) * 0 + f64(d)[0])
    want = ((f64(S) * f64(r[:M])[:, None] * along) * f64(dY)).sum()
    assert abs((f64(dW) * along).sum() - want) <= (np.abs(f64(S) * f64(r[:M])[:, None] * along * f64(dY))).sum() * 100 * U


# ---- streams, graphs, devices -----------------------------------------------------------------------------------------
def test_captured_and_replayed():
    M, K = 70, 8192
    X, R, W = case(M, K, 31, s="f32")
    dY = torch.randn(M, K, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(DEV)
    p = norm.norm_problem(M, K, s_dtype="f32")
    S, Y, r = torch.empty_like(R), torch.empty_like(X), torch.empty(M, device=DEV)
    dR, dW = torch.empty_like(R), torch.empty(K, device=DEV)
    ws = torch.zeros(norm.flux_norm_workspace_bytes(p), dtype=torch.uint8, device=DEV)

    def step():
        norm.flux_norm(p, X, R, W, S, Y, None, r)
        norm.flux_norm_backward(p, dY, S, W, r, R, dR, None, dW, ws)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    for i in range(4):
        X.copy_(torch.randn(M, K, generator=torch.Generator().manual_seed(40 + i)))
        step()
        want = [t.clone() for t in (S, Y, r, dR, dW)]
        for t in (S, Y, r, dR, dW):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, (S, Y, r, dR, dW)):
            assert torch.equal(a, b), i


def test_streams_of_their_own():
    M, K = 64, 8192
    X, R, W = case(M, K, 51)
    want = run_forward(X, R, W, "bf16", 1e-5)
    p = norm.norm_problem(M, K)
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = []
    torch.cuda.synchronize()
    for s in streams:
        S, Y = torch.empty_like(R), torch.empty_like(X)
        norm.flux_norm(p, X, R, W, S, Y, stream=s)
        outs.append((S, Y))
    torch.cuda.synchronize()
    for S, Y in outs:
        assert torch.equal(S, want[0]) and torch.equal(Y, want[1])


def test_tensors_of_another_type_or_device_are_refused():
    X, R, W = case(4, 64, 1)
    p = norm.norm_problem(4, 64)
    Y, S = torch.empty_like(X), torch.empty_like(R)
    for args in ((X.float(), R, W, S, Y), (X.cpu(), R, W, S, Y), (X, R.float(), W, S, Y), (X, R, W.float(), S, Y), (X, R, W, S.cpu(), Y), (X, R, W, S, Y.float())):
        with pytest.raises(ValueError):
            norm.flux_norm(p, *args)
    with pytest.raises(ValueError):
        norm.flux_norm_backward(p, X, R, W, torch.ones(4, device=DEV), dW=torch.empty(64, device=DEV), workspace=torch.zeros(1 << 20, dtype=torch.uint8))


@pytest.mark.parametrize("bits", [4, 8])
def test_what_the_4_bit_cast_makes_of_the_norm(bits):
    """In 4 bits the two launches norm in fp32, cast and the one launch norm in blocks give the same bits where no number lies next to a border: rows of
    ones give W itself."""
    K = 8192
    W = torch.randn(K, generator=torch.Generator().manual_seed(3)).to(DEV)
    X = torch.ones(3, K, dtype=torch.bfloat16, device=DEV)
    _, q, scales, _, _ = run_forward(X, None, W, f"mx{bits}", 0.0)
    if bits == 4:
        q2, s2 = torch.empty(3, K // 2, dtype=torch.uint8, device=DEV), torch.empty(3, K // 32, dtype=torch.uint8, device=DEV)
        ffn.flux_mx4_quantize(W.expand(3, K).contiguous(), q2, s2)
        assert torch.equal(q[:3], q2) and torch.equal(scales[:3], s2)
    else:
        back = torch.empty(3, K, device=DEV)
        norm.flux_mx8_dequantize(q[:3], scales[:3], back)
        codes, byte = no.blocks(f64(W)[None], 8)
        assert (f64(back) == no.block_values(codes, byte, 8)).all()
