"""The gated feed-forward block on the GPU against its definition in 64 bits.

Bounds, elementwise.  A product of bf16 numbers is exact in fp32 and a sum of K of them is off by at most K 2^-23 of the sum of
their magnitudes (twice the unit roundoff, for whatever the matrix cores drop); exp2, reciprocal and the few operations of an
activation by 2^-19 of it; one rounding to bf16 by 2^-8, to fp32 by 2^-24.  The activations' slopes are at most 1.13."""
import numpy as np
import pytest
import torch

from oracle import ffn_oracle as oo
from paper_2406_06858_amd import ffn

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
ROUND = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
SLOPE = 1.13


def _np(t):
    return t.detach().cpu().double().numpy()


def _draw(seed, *shape, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(torch.bfloat16)


def _pitched(t, pitch, fill):
    """`t` on the GPU in rows of `pitch` elements, `fill` between them."""
    store = torch.full((t.shape[0], pitch), fill, dtype=t.dtype, device=DEV)
    store[:, :t.shape[1]] = t.to(DEV)
    return store


def _workspace(op, p):
    n = ffn.flux_glu_workspace_bytes(op, p)
    if n == 0:
        return None
    ws = torch.full((n,), 255, dtype=torch.uint8, device=DEV)
    ffn.flux_ffn_init(ws)
    return ws


def _forward(M, N, K, act, nk, out="bf16", save=True, pad=0, seed=1, X=None, Wg=None, Wu=None, scale=None,
             tile_config=0, split_k=0):
    scale = K ** -0.5 if scale is None else scale
    X = _draw(seed, M, K) if X is None else X
    Wg = _draw(seed + 1, K, N, scale=2 * scale) if Wg is None else Wg
    Wu = _draw(seed + 2, K, N, scale=scale) if Wu is None else Wu
    w_cols = K if nk else N
    p = ffn.glu_problem(M, N, K, act=act, w_is_nk=nk, out_dtype=out, ldx=K + pad if pad else 0, ldw=w_cols + 2 * pad if pad else 0,
                        ldh=N + 3 * pad if pad else 0, tile_config=tile_config, split_k=split_k)
    nan = float("nan")
    w = [_pitched(t.t().contiguous() if nk else t, w_cols + 2 * pad, nan) for t in (Wg, Wu)]
    x = _pitched(X, K + pad, nan)
    H = torch.full((M, N + 3 * pad), 7.0, dtype=TORCH[out], device=DEV)
    G, U = (torch.full((M, N + 3 * pad), 7.0, dtype=torch.bfloat16, device=DEV) if save else None for _ in range(2))
    ffn.flux_glu(p, x, *w, H, G, U, _workspace(ffn.FLUX_GLU_FORWARD, p))
    torch.cuda.synchronize()
    for t in (H, G, U):
        assert t is None or pad == 0 or bool((t[:, N:] == 7.0).all()), "written between the rows"
    return (X, Wg, Wu), tuple(None if t is None else t[:, :N] for t in (H, G, U))


def _check_forward(ins, outs, act, out="bf16"):
    x, wg, wu = (_np(t) for t in ins)
    K = x.shape[1]
    h, g, u = oo.glu(act, x, wg, wu)
    eg, eu = (K * 2.0 ** -23 * (np.abs(x) @ np.abs(w)) for w in (wg, wu))
    a = oo.act(act, g)
    bound = (ROUND[out] + 2.0 ** -19) * np.abs(h) + 1.01 * (SLOPE * eg * np.abs(u) + np.abs(a) * eu + SLOPE * eg * eu) + 1e-30
    err = np.abs(_np(outs[0]) - h)
    assert (err <= bound).all(), f"H off by {np.max(err / bound):.3g} of its bound"
    for name, got, want, e in (("G", outs[1], g, eg), ("U", outs[2], u, eu)):
        if got is not None:
            assert (np.abs(_np(got) - want) <= 2.0 ** -8 * np.abs(want) + 1.01 * e).all(), name


FORWARD = [
    # one row, few rows, rows around every height that a block of rows ends at
    (1, 64, 64), (1, 8, 8), (1, 136, 2056), (2, 520, 40), (7, 264, 1024), (15, 72, 200), (16, 128, 512), (17, 96, 1032), (31, 200, 328), (33, 128, 640),
    (48, 384, 264), (63, 64, 4096), (64, 512, 1024), (65, 136, 520), (100, 328, 776), (127, 64, 2048), (128, 256, 512), (129, 256, 264),
    # tiles: divided, ragged in every direction, K shorter than a slab, long K over few tiles
    (256, 256, 256), (256, 512, 1024), (300, 520, 392), (255, 248, 8), (257, 8, 64), (200, 264, 4104), (512, 128, 8192), (1000, 136, 72), (640, 1032, 520),
]


@pytest.mark.parametrize("nk", [0, 1])
@pytest.mark.parametrize("M,N,K", FORWARD)
def test_forward(M, N, K, nk):
    act = ("silu", "gelu", "gelu_tanh")[(M + N + K) // 8 % 3]
    _check_forward(*_forward(M, N, K, act, nk, save=M % 2 == 0), act)


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("M,N,K", [(5, 72, 264), (40, 72, 264), (300, 264, 264)])
@pytest.mark.parametrize("nk", [0, 1])
def test_forward_in_32_bits(M, N, K, act, nk):
    _check_forward(*_forward(M, N, K, act, nk, out="f32", seed=11), act, "f32")


@pytest.mark.parametrize("M,N,K,nk", [(1, 72, 264, 1), (3, 72, 264, 0), (64, 72, 520, 1), (70, 264, 136, 0), (300, 264, 136, 1), (256, 256, 128, 0)])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_forward_pitches(M, N, K, nk, out):
    _check_forward(*_forward(M, N, K, "silu", nk, out=out, pad=8, seed=21), "silu", out)


@pytest.mark.parametrize("M,N,K,nk", [(1, 128, 512, 1), (16, 64, 2048, 0), (60, 136, 512, 1), (256, 264, 512, 0), (520, 512, 200, 1)])
def test_forward_whole_numbers_are_exact(M, N, K, nk):
    """Every partial sum of integers below 2^24 is exact, so G and U are the one rounding of the exact product."""
    gen = torch.Generator().manual_seed(5)
    X, Wg, Wu = ((torch.randint(-8, 9, s, generator=gen)).to(torch.bfloat16) for s in ((M, K), (K, N), (K, N)))
    (_, _, _), (H, G, U) = _forward(M, N, K, "silu", nk, X=X, Wg=Wg, Wu=Wu)
    for got, w in ((G, Wg), (U, Wu)):
        assert torch.equal(got.cpu(), (X.double() @ w.double()).to(torch.bfloat16))


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("M,nk", [(4, 1), (4, 0), (300, 1)])
def test_forward_far_out(act, M, nk):
    """Gates of up to 10^30 in magnitude: 0 or g, and never NaN."""
    K = N = 64
    X = torch.zeros(M, K, dtype=torch.bfloat16)
    X[:, 0] = 1
    Wg, Wu = torch.zeros(K, N, dtype=torch.bfloat16), torch.zeros(K, N, dtype=torch.bfloat16)
    Wg[0] = torch.tensor([s * 10.0 ** e for e in range(-1, 31) for s in (1, -1)]).to(torch.bfloat16)
    Wu[0] = 1
    (_, _, _), (H, G, U) = _forward(M, N, K, act, nk, X=X, Wg=Wg, Wu=Wu)
    g = _np(Wg)[0]
    with np.errstate(over="ignore"):
        want = np.where(g < -30, 0, np.where(g > 30, g, oo.act(act, np.clip(g, -30, 30))))
    assert (np.abs(_np(H) - want[None]) <= 2.0 ** -8 * np.abs(want) + 1e-6).all()


@pytest.mark.parametrize("M,nk", [(3, 1), (40, 0), (300, 1), (300, 0)])
def test_forward_keeps_rows_apart(M, nk):
    """A row of zeros gives zeros, a row with NaN or infinity spoils itself alone."""
    N, K = 136, 264
    X = _draw(31, M, K)
    X[0] = 0
    X[M - 1, 5] = float("nan")
    X[M // 2, K - 1] = float("inf")
    Wg, Wu = _draw(32, K, N, scale=0.1), _draw(33, K, N, scale=0.1)
    _, (H, G, U) = _forward(M, N, K, "silu", nk, X=X, Wg=Wg, Wu=Wu)
    keep = [i for i in range(M) if i not in (M - 1, M // 2)]
    assert not H[0].any() and bool(torch.isnan(H[M - 1]).all()) and not bool(torch.isfinite(G[M // 2]).any())
    _check_forward((X[keep], Wg, Wu), (H[keep], G[keep], U[keep]), "silu")


TILES = list(range(1, ffn.flux_ffn_tile_config_count()))        # (the last one is for few rows)


@pytest.mark.parametrize("nk", [0, 1])
@pytest.mark.parametrize("split", [1, 3])
@pytest.mark.parametrize("cfg", TILES)
def test_forward_of_every_tile(cfg, split, nk):
    """Shapes that no tile divides and one that all do; K shorter than the ring of slabs and longer, cut and whole."""
    for M, N, K in ((300, 200, 1480), (512, 256, 1024), (70, 72, 72)):
        _check_forward(*_forward(M, N, K, "silu", nk, tile_config=cfg, split_k=split), "silu")


# ---- backward -----------------------------------------------------------------------------------------------------
def _backward(M, N, K, act, nk, out="bf16", dw="bf16", accumulate=0, pad=0, seed=3, X=None, Wg=None, Wu=None, G=None, U=None, dH=None,
              want_x=True, want_w=True, tile_config=0, split_k=0):
    X = _draw(seed, M, K) if X is None else X
    Wg, Wu = _draw(seed + 1, K, N, scale=K ** -0.5) if Wg is None else Wg, _draw(seed + 2, K, N, scale=K ** -0.5) if Wu is None else Wu
    G, U = _draw(seed + 3, M, N, scale=2.0) if G is None else G, _draw(seed + 4, M, N) if U is None else U
    dH = _draw(seed + 5, M, N) if dH is None else dH
    w_cols = K if nk else N
    p = ffn.glu_problem(M, N, K, act=act, w_is_nk=nk, out_dtype=out, dw_dtype=dw, dw_accumulate=accumulate, ldx=K + pad if pad else 0,
                        ldw=w_cols + 2 * pad if pad else 0, ldh=N + 3 * pad if pad else 0, tile_config=tile_config, split_k=split_k)
    nan = float("nan")
    w = [_pitched(t.t().contiguous() if nk else t, w_cols + 2 * pad, nan) for t in (Wg, Wu)]
    x = _pitched(X, K + pad, nan)
    g, u, dh = (_pitched(t, N + 3 * pad, nan) for t in (G, U, dH))
    dX = torch.full((M, K + pad), 7.0, dtype=TORCH[out], device=DEV) if want_x else None
    dW = [torch.full((w[0].shape[0], w_cols + 2 * pad), 7.0, dtype=TORCH[dw], device=DEV) if want_w else None for _ in range(2)]
    ffn.flux_glu_backward(p, x, *w, g, u, dh, dX, *dW, _workspace(ffn.FLUX_GLU_BACKWARD, p))
    torch.cuda.synchronize()
    for t, cols in ((dX, K), (dW[0], w_cols), (dW[1], w_cols)):
        assert t is None or pad == 0 or bool((t[:, cols:] == 7.0).all()), "written between the rows"
    outs = [None if dX is None else dX[:, :K]] + [None if t is None else (t[:, :w_cols].t() if nk else t[:, :w_cols]) for t in dW]
    return (X, Wg, Wu, G, U, dH), outs


def _check_backward(ins, outs, act, out="bf16", dw="bf16", start=0.0):
    x, wg, wu, g, u, dh = (_np(t) for t in ins)
    dx, dwg, dwu, dg, du = oo.glu_backward(act, x, wg, wu, g, u, dh)
    # dG, dU: fp32, then one rounding to bf16
    edg = 2.0 ** -8 * np.abs(dg) + 2.0 ** -18 * np.abs(dh * u) * (1 + np.abs(g))
    edu = 2.0 ** -8 * np.abs(du) + 2.0 ** -18 * np.abs(dh) * (1 + np.abs(g))
    N, M = g.shape[1], g.shape[0]
    want = {"dX": (dx, 1.01 * (edg @ np.abs(wg).T + edu @ np.abs(wu).T) + 2 * N * 2.0 ** -23 * (np.abs(dg) @ np.abs(wg).T + np.abs(du) @ np.abs(wu).T), out),
            "dWg": (dwg + start, 1.01 * np.abs(x).T @ edg + (M + 1) * 2.0 ** -23 * (np.abs(x).T @ np.abs(dg) + abs(start)), dw),
            "dWu": (dwu + start, 1.01 * np.abs(x).T @ edu + (M + 1) * 2.0 ** -23 * (np.abs(x).T @ np.abs(du) + abs(start)), dw)}
    for (name, (ref, e, dtype)), got in zip(want.items(), outs):
        if got is None:
            continue
        err = np.abs(_np(got) - ref)
        bound = ROUND[dtype] * (np.abs(ref) + e) + e + 1e-30
        assert (err <= bound).all(), f"{name} off by {np.max(err / bound):.3g} of its bound"
        if ref.size >= 4096 and not start and min(M, N) >= 64:
            # two independent roundings, each 2^-8 / sqrt 3 of the result in the mean at most
            assert np.linalg.norm(err) <= 2.0 ** -8 * np.linalg.norm(ref), name


BACKWARD = [
    (1, 8, 8), (1, 136, 264), (2, 64, 512), (9, 72, 40), (16, 128, 128), (33, 200, 72), (64, 64, 64), (65, 264, 136), (128, 256, 256), (200, 136, 520),
    (256, 256, 256), (264, 512, 264), (300, 264, 392), (512, 72, 1032), (1000, 136, 72), (72, 1000, 136), (136, 72, 1000), (2048, 64, 64), (512, 256, 512),
]


@pytest.mark.parametrize("nk", [0, 1])
@pytest.mark.parametrize("M,N,K", BACKWARD)
def test_backward(M, N, K, nk):
    act = ("silu", "gelu", "gelu_tanh")[(M + N + K) // 8 % 3]
    _check_backward(*_backward(M, N, K, act, nk), act)


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("nk", [0, 1])
@pytest.mark.parametrize("M,N,K", [(10, 72, 136), (300, 264, 264)])
def test_backward_in_32_bits_and_accumulated(M, N, K, act, nk):
    _check_backward(*_backward(M, N, K, act, nk, out="f32", dw="f32", accumulate=1, seed=41), act, "f32", "f32", start=7.0)
    _check_backward(*_backward(M, N, K, act, nk, accumulate=1, seed=42), act, start=7.0)


@pytest.mark.parametrize("M,N,K,nk", [(1, 72, 264, 1), (65, 72, 136, 0), (300, 264, 136, 1), (256, 256, 128, 0)])
def test_backward_pitches(M, N, K, nk):
    _check_backward(*_backward(M, N, K, "gelu_tanh", nk, pad=8, seed=51), "gelu_tanh")
    _check_backward(*_backward(M, N, K, "silu", nk, out="f32", dw="f32", pad=16, seed=52), "silu", "f32", "f32")


@pytest.mark.parametrize("nk", [0, 1])
@pytest.mark.parametrize("split", [1, 3])
@pytest.mark.parametrize("cfg", TILES)
def test_backward_of_every_tile(cfg, split, nk):
    for M, N, K in ((300, 712, 264), (256, 512, 256), (70, 72, 72)):
        _check_backward(*_backward(M, N, K, "silu", nk, tile_config=cfg, split_k=split), "silu")


@pytest.mark.parametrize("want_x,want_w", [(True, False), (False, True), (False, False)])
def test_backward_of_some(want_x, want_w):
    ins, outs = _backward(130, 136, 264, "silu", 1, want_x=want_x, want_w=want_w)
    assert (outs[0] is not None) == want_x and (outs[1] is not None) == want_w
    _check_backward(ins, outs, "silu")


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_backward_far_out(act):
    """Gates of up to 10^30: slopes 0 and 1, gradients of them, and never NaN."""
    M, N, K = 2, 64, 64
    g = torch.tensor([s * 10.0 ** e for e in range(-1, 31) for s in (1, -1)]).to(torch.bfloat16)
    one = torch.ones(M, N, dtype=torch.bfloat16)
    eye = torch.eye(N, dtype=torch.bfloat16)
    _, (dX, dWg, dWu) = _backward(M, N, K, act, 1, X=torch.ones(M, K, dtype=torch.bfloat16), Wg=eye, Wu=torch.zeros_like(eye), G=g.expand(M, N).contiguous(), U=one, dH=one)
    x = _np(g)
    want = np.where(x < -30, 0, np.where(x > 30, 1, oo.slope(act, np.clip(x, -30, 30))))
    assert (np.abs(_np(dX) - want[None]) <= 2.0 ** -7 * np.abs(want) + 1e-5).all()
    up = np.where(x < -30, 0, np.where(x > 30, x, oo.act(act, np.clip(x, -30, 30))))
    assert (np.abs(_np(dWu) - 2 * up[None]) <= 2.0 ** -6 * np.abs(up) + 1e-5).all()


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("M,N,K,nk", [(8, 64, 64, 1), (96, 128, 72, 0)])
def test_backward_against_differences(act, M, N, K, nk):
    """d/dt of sum(dH * H(X + t D)) and of the weights', by central differences in 64 bits.  X, Wg and Wu are whole multiples of 1/4 small
    enough for G and U to be bf16 numbers, so the gradients are those of the very function that is differenced."""
    gen = torch.Generator().manual_seed(9)
    X = torch.zeros(M, K)
    X[torch.arange(M).repeat_interleave(4), torch.randint(0, K, (4 * M,), generator=gen)] = torch.randint(-2, 3, (4 * M,), generator=gen).float()
    Wg, Wu = (torch.randint(-4, 5, (K, N), generator=gen).float() / 4 for _ in range(2))
    G, U = X @ Wg, X @ Wu
    assert torch.equal(G.to(torch.bfloat16).float(), G) and torch.equal(U.to(torch.bfloat16).float(), U)
    dH = _draw(61, M, N)
    bf = [t.to(torch.bfloat16) for t in (X, Wg, Wu, G, U)]
    ins, outs = _backward(M, N, K, act, nk, X=bf[0], Wg=bf[1], Wu=bf[2], G=bf[3], U=bf[4], dH=dH)
    rng = np.random.default_rng(4)
    base = [_np(t) for t in ins[:3]]
    for i, got in enumerate(outs):
        D = rng.normal(size=base[i].shape)
        h = 1e-5
        def at(t):
            v = list(base)
            v[i] = v[i] + t * D
            return (oo.glu(act, *v)[0] * _np(ins[5])).sum()
        diff, grad = (at(h) - at(-h)) / (2 * h), (_np(got) * D).sum()
        # the gradient's own error is at most 2^-8 of it in the norm (see _check_backward); D is independent of it
        assert abs(diff - grad) <= 4 * 2.0 ** -8 * np.linalg.norm(_np(got)) + 1e-6, (i, diff, grad)


# ---- streams, graphs, repeated calls ------------------------------------------------------------------------------
@pytest.mark.parametrize("M,N,K", [(1, 1024, 2048), (40, 512, 2048), (200, 256, 2048), (300, 512, 512)])
@pytest.mark.parametrize("nk", [0, 1])
def test_same_bits_again_on_another_stream_and_in_a_graph(M, N, K, nk):
    X, G, U, dH = (_draw(70 + i, M, n).to(DEV) for i, n in enumerate((K, N, N, N)))
    Wg, Wu = (_draw(80 + i, *((N, K) if nk else (K, N)), scale=K ** -0.5).to(DEV) for i in range(2))
    p = ffn.glu_problem(M, N, K, w_is_nk=nk)
    wf, wb = _workspace(ffn.FLUX_GLU_FORWARD, p), _workspace(ffn.FLUX_GLU_BACKWARD, p)
    outs = [torch.empty(s, dtype=torch.bfloat16, device=DEV) for s in ((M, N), (M, N), (M, N), X.shape, Wg.shape, Wu.shape)]

    def both(stream=None):
        ffn.flux_glu(p, X, Wg, Wu, *outs[:3], wf, stream)
        ffn.flux_glu_backward(p, X, Wg, Wu, G, U, dH, *outs[3:], wb, stream)

    both()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(torch.cuda.current_stream())
    for _ in range(3):
        for t in outs:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
        both()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
