"""Calls whose tiles are cut along the contraction, side by side on several streams.  The parts of a tile wait for each other, and
beside other grids some of them are not given a compute unit for long: the calls have to end, with the same bits, and leave their
workspaces as they found them."""
import pytest
import torch

from paper_2406_06858_amd import ffn

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _draw(seed, *shape, scale=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(torch.bfloat16)


def _workspace(n):
    ws = torch.empty(max(n, 16), dtype=torch.uint8, device=DEV)
    ffn.flux_ffn_init(ws)
    return ws


def _glu(seed, M, N, K, nk, **choice):
    """A forward call and its outputs, to be made again and again."""
    X, Wg, Wu = _draw(seed, M, K), *(_draw(seed + i, *((N, K) if nk else (K, N)), scale=K ** -0.5) for i in (1, 2))
    p = ffn.glu_problem(M, N, K, w_is_nk=nk, **choice)
    ws = _workspace(ffn.flux_glu_workspace_bytes(ffn.FLUX_GLU_FORWARD, p))
    H = torch.empty(M, N, dtype=torch.bfloat16, device=DEV)
    return lambda w, stream=None: ffn.flux_glu(p, X, Wg, Wu, H, None, None, w, stream), [H], ws


def _backward(seed, M, N, K, nk, **choice):
    X, Wg, Wu = _draw(seed, M, K), *(_draw(seed + i, *((N, K) if nk else (K, N)), scale=K ** -0.5) for i in (1, 2))
    G, U, dH = (_draw(seed + i, M, N) for i in (3, 4, 5))
    p = ffn.glu_problem(M, N, K, w_is_nk=nk, **choice)
    ws = _workspace(ffn.flux_glu_workspace_bytes(ffn.FLUX_GLU_BACKWARD, p))
    outs = [torch.empty_like(t) for t in (X, Wg, Wu)]
    return lambda w, stream=None: ffn.flux_glu_backward(p, X, Wg, Wu, G, U, dH, *outs, w, stream), outs, ws


def _mx4(seed, M, N, K, **choice):
    g = torch.Generator(device=DEV).manual_seed(seed)
    mats = []
    for rows in (M, N):
        mats.append(torch.randint(0, 256, (rows, ffn.flux_mx4_row_bytes(K)), generator=g, device=DEV, dtype=torch.uint8))
        s = torch.zeros(rows, ffn.flux_mx4_scale_row_bytes(K), dtype=torch.uint8, device=DEV)
        s[:, :(K + 31) // 32] = torch.randint(100, 140, (rows, (K + 31) // 32), generator=g, device=DEV, dtype=torch.uint8)
        mats.append(s)
    p = ffn.mx4_problem(M, N, K, out_dtype="f32", **choice)
    ws = _workspace(ffn.flux_mx4_workspace_bytes(ffn.FLUX_MX4_GEMM, p))
    C = torch.empty(M, N, dtype=torch.float32, device=DEV)
    return lambda w, stream=None: ffn.flux_mx4_gemm(p, *mats, C, w, stream), [C], ws


def test_cut_tiles_of_several_streams_at_once():
    calls = [_glu(1, 200, 1792, 4096, 0), _glu(11, 200, 1792, 4096, 0, tile_config=1, split_k=16), _backward(21, 520, 712, 1032, 1, split_k=7),
             _mx4(31, 200, 1032, 8192, tile_config=1, split_k=16), _glu(41, 2048, 1792, 2048, 1, split_k=1)]
    streams = [torch.cuda.Stream() for _ in calls]
    want = []
    for call, outs, ws in calls:
        call(ws)
        torch.cuda.synchronize()
        want.append([t.clone() for t in outs])
    for _ in range(4):
        for _, outs, _ in calls:
            for t in outs:
                t.fill_(float("nan"))
        torch.cuda.synchronize()
        for _ in range(12):
            for (call, _, ws), s in zip(calls, streams):
                call(ws, s)
        torch.cuda.synchronize()
        for i, (_, outs, ws) in enumerate(calls):
            assert all(torch.equal(a, b) for a, b in zip(outs, want[i])), i
            assert not bool(ws[:512 * 64].any()), "the words of the cut tiles are zero between calls"


def test_a_workspace_serves_all_operators_in_turn():
    """One workspace, problems of every kind one after the other: as with workspaces of their own."""
    calls = [_glu(1, 200, 520, 4096, 1, split_k=8), _backward(21, 300, 264, 520, 0), _mx4(31, 70, 264, 4096, split_k=4), _glu(5, 300, 264, 520, 0)]
    want = []
    for call, outs, ws in calls:
        call(ws)
        torch.cuda.synchronize()
        want.append([t.clone() for t in outs])
    most = max(ws.numel() for _, _, ws in calls)
    shared = torch.full((most,), 255, dtype=torch.uint8, device=DEV)
    ffn.flux_ffn_init(shared)
    for _ in range(2):
        for i, (call, outs, _) in enumerate(calls):
            for t in outs:
                t.fill_(float("nan"))
            call(shared)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs, want[i])), i
