"""The gated MLP of examples/gated_mlp.py, trained and served, against plain numpy in 64 bits: the operators of both
libraries one after the other on one stream.  Bounds are of the whole chain, in the norm: every bf16 rounding on the way adds at most
2^-8 / sqrt 3 of what it rounds; four of them lie between X and Y or a gradient, and one between dY and dX's operands more."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

import gated_mlp as gm  # noqa: E402
from oracle import ffn_oracle as oo  # noqa: E402

pytestmark = pytest.mark.gpu
ROUND = 2.0 ** -8 / np.sqrt(3)


def _np(t):
    return t.detach().cpu().double().numpy()


def _draw(seed, *shape, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(torch.bfloat16).to("cuda:0")


def _off(got, want):
    return np.linalg.norm(_np(got) - want) / np.linalg.norm(want)


@pytest.mark.parametrize("M,D,N,R,rank,act", [(16, 256, 128, 2, 1, "silu"), (256, 512, 320, 4, 0, "gelu_tanh"), (520, 328, 264, 8, 5, "gelu")])
def test_training_step(M, D, N, R, rank, act):
    X, Wg, Wu, Wd = _draw(1, M, D), _draw(2, N, D, std=D ** -0.5), _draw(3, N, D, std=D ** -0.5), _draw(4, N, D, std=N ** -0.5)
    peers = [None if r == rank else _draw(10 + r, M, D) for r in range(R)]
    chunks = [_draw(30 + r, M // R, D) for r in range(R)]
    mlp = gm.GatedMlp(M, D, N, R, rank, act)
    for _ in range(2):                                     # (the second step finds the workspaces as the first left them)
        Y = mlp.forward(X, Wg, Wu, Wd, peers)
        grads = mlp.backward(X, Wg, Wu, Wd, chunks)
    torch.cuda.synchronize()
    h, g, u = oo.glu(act, _np(X), _np(Wg).T, _np(Wu).T)
    y = h @ _np(Wd) + sum(_np(p) for p in peers if p is not None)
    assert _off(torch.cat(Y), y) <= 3 * ROUND
    dy = np.concatenate([_np(c) for c in chunks])
    # the kept G and U are rounded: the gradients are those at the rounded point
    want = oo.glu_backward(act, _np(X), _np(Wg).T, _np(Wu).T, _np(mlp.G), _np(mlp.U), dy @ _np(Wd).T)[:3]
    assert _off(mlp.G, g) <= ROUND and _off(mlp.U, u) <= ROUND
    for got, ref in zip(grads, (want[0], want[1].T, want[2].T)):
        assert _off(got, ref) <= 4 * ROUND


@pytest.mark.parametrize("M,D,N", [(1, 256, 128), (33, 512, 320), (300, 1024, 264)])
def test_serving_step(M, D, N):
    X, Wg, Wu, Wd = _draw(5, M, D), _draw(6, N, D, std=D ** -0.5), _draw(7, N, D, std=D ** -0.5), _draw(8, N, D, std=N ** -0.5)
    serve = gm.GatedMlp4Bit(M, Wg, Wu, Wd)
    serve(X)
    Y = serve(X).clone()
    torch.cuda.synchronize()
    x, wg, wu, wd = (_np(m.read(k)) for m, k in ((serve.X, D), (serve.Wg, D), (serve.Wu, D), (serve.Wd, N)))
    assert np.array_equal(x, oo.mx4_values(*oo.mx4_quantize(_np(X)))[:, :D])
    h = oo.glu("silu", x, wg.T, wu.T)[0]
    assert _off(serve.H, h) <= ROUND
    # what the block made of H in 4 bits is a whole rounding of it, so the rest is checked from there on
    h4 = _np(serve.H4.read(N))
    assert np.array_equal(h4, oo.mx4_values(*oo.mx4_quantize(_np(serve.H)))[:, :N])
    assert np.abs(_np(Y) - h4 @ wd.T).max() <= (N + 1) * 2.0 ** -23 * (np.abs(h4) @ np.abs(wd).T).max()
