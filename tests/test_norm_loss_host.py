"""CPU-only checks of the norm's and the loss's entry points and of their oracle: exports, struct layout, refusals before anything is enqueued,
the oracle's gradients against differences, its 8-bit rounding against values worked out by hand."""
import ctypes
import os
import re

import numpy as np
import pytest

from oracle import ffn_oracle as oo
from oracle import norm_loss_oracle as no
from paper_2406_06858_amd import binding as fb
from paper_2406_06858_amd import ffn, loss, norm

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PTR = 4096            # never read: the calls below are refused before anything is enqueued


@pytest.mark.parametrize("header,module", [("flux_norm.h", norm), ("flux_loss.h", loss)])
def test_library_exports_what_the_headers_declare(header, module):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header)).read(), flags=re.S)
    declared = set(re.findall(r"\b(flux_[a-z0-9_]+)\s*\(", text))
    assert declared == set(module.EXPORTS)
    assert all(hasattr(module.lib(), name) for name in declared)


def test_struct_layouts():
    assert ctypes.sizeof(norm.flux_norm_t) == 64 and norm.flux_norm_t.eps.offset == 32 and norm.flux_norm_t.ldx.offset == 40
    assert ctypes.sizeof(loss.flux_loss_t) == 80 and loss.flux_loss_t.v0.offset == 16 and loss.flux_loss_t.ldx.offset == 48


# ---- norm ---------------------------------------------------------------------------------------------------------
def _norm(p, **ptrs):
    v = dict(X=PTR, R=PTR, W=PTR, S=PTR, Y=PTR, scales=0, rstd=PTR, **{})
    v.update(ptrs)
    return norm.lib().flux_norm(None if p is None else ctypes.byref(p), *[v[n] for n in ("X", "R", "W", "S", "Y", "scales", "rstd")], None)


def _norm_bwd(p, ws=(PTR, 1 << 40), **ptrs):
    names = ["dY", "S", "W", "rstd", "dS", "dR", "dX", "dW"]
    v = {n: PTR for n in names}
    v.update(ptrs)
    return norm.lib().flux_norm_backward(None if p is None else ctypes.byref(p), *[v[n] for n in names], *ws, None)


@pytest.mark.parametrize("bad,status", [
    (dict(M=0), fb.FLUX_ERR_SHAPE), (dict(M=-3), fb.FLUX_ERR_SHAPE), (dict(K=0), fb.FLUX_ERR_SHAPE), (dict(K=(1 << 30) + 1), fb.FLUX_ERR_SHAPE),
    (dict(ldx=255), fb.FLUX_ERR_SHAPE), (dict(lds=1), fb.FLUX_ERR_SHAPE), (dict(ldy=200), fb.FLUX_ERR_SHAPE), (dict(ldx=-256), fb.FLUX_ERR_INVALID_ARG),
    (dict(lds=1 << 62), fb.FLUX_ERR_SHAPE), (dict(ldy=1 << 26), fb.FLUX_ERR_SHAPE), (dict(M=1 << 24), fb.FLUX_ERR_SHAPE),
    (dict(x_dtype=2), fb.FLUX_ERR_INVALID_ARG), (dict(s_dtype=-1), fb.FLUX_ERR_INVALID_ARG), (dict(w_dtype=7), fb.FLUX_ERR_INVALID_ARG),
    (dict(dw_dtype=2), fb.FLUX_ERR_INVALID_ARG), (dict(out=4), fb.FLUX_ERR_INVALID_ARG), (dict(out=-1), fb.FLUX_ERR_INVALID_ARG),
    (dict(dw_accumulate=2), fb.FLUX_ERR_INVALID_ARG), (dict(reserved=1), fb.FLUX_ERR_INVALID_ARG), (dict(eps=-1e-6), fb.FLUX_ERR_INVALID_ARG),
    (dict(eps=float("nan")), fb.FLUX_ERR_INVALID_ARG), (dict(eps=float("inf")), fb.FLUX_ERR_INVALID_ARG),
])
def test_norm_refuses_problems(bad, status):
    p = norm.norm_problem(64, 256)
    for k, v in bad.items():
        setattr(p, k, v)
    assert _norm(p) == status and _norm_bwd(p) == status
    assert norm.flux_norm_workspace_bytes(p) == 0


def test_norm_refuses_pointers():
    p = norm.norm_problem(64, 256)
    for ptrs in (dict(X=0), dict(W=0), dict(Y=0), dict(R=0), dict(S=0), dict(X=PTR + 1), dict(S=PTR + 1), dict(Y=PTR + 1), dict(scales=PTR), dict(rstd=PTR + 2)):
        assert _norm(p, **ptrs) == fb.FLUX_ERR_INVALID_ARG, ptrs
    for out in ("mx4", "mx8"):
        p = norm.norm_problem(64, 256, out=out)
        for ptrs in (dict(), dict(scales=PTR + 8), dict(scales=PTR, Y=PTR + 8)):
            assert _norm(p, **ptrs) == fb.FLUX_ERR_INVALID_ARG, ptrs
        assert _norm_bwd(p) == fb.FLUX_ERR_UNSUPPORTED and norm.flux_norm_workspace_bytes(p) == 0
    p = norm.norm_problem(64, 256, s_dtype="f32", out="f32", x_dtype="f32", w_dtype="f32")
    for ptrs in (dict(X=PTR + 2), dict(R=PTR + 2), dict(W=PTR + 2), dict(Y=PTR + 2)):
        assert _norm(p, **ptrs) == fb.FLUX_ERR_INVALID_ARG, ptrs
    for ptrs in (dict(dY=0), dict(S=0), dict(W=0), dict(rstd=0), dict(dY=PTR + 2), dict(dS=PTR + 2), dict(dR=PTR + 2), dict(dX=PTR + 2), dict(dW=PTR + 2)):
        assert _norm_bwd(p, **ptrs) == fb.FLUX_ERR_INVALID_ARG, ptrs
    assert _norm(None) == fb.FLUX_ERR_INVALID_ARG and _norm_bwd(None) == fb.FLUX_ERR_INVALID_ARG


def test_norm_backward_wants_its_workspace_for_dw():
    p = norm.norm_problem(64, 256)
    need = norm.flux_norm_workspace_bytes(p)
    assert need > 0
    for ws in ((0, 0), (PTR, need - 1), (PTR + 8, need)):
        assert _norm_bwd(p, ws=ws) == fb.FLUX_ERR_WORKSPACE


@pytest.mark.parametrize("args,status", [
    ((0, 64, 0, PTR, 0, PTR, PTR), fb.FLUX_ERR_SHAPE), ((4, 0, 0, PTR, 0, PTR, PTR), fb.FLUX_ERR_SHAPE), ((4, 64, 0, PTR, 63, PTR, PTR), fb.FLUX_ERR_SHAPE),
    ((4, 64, 2, PTR, 0, PTR, PTR), fb.FLUX_ERR_INVALID_ARG), ((4, 64, 0, 0, 0, PTR, PTR), fb.FLUX_ERR_INVALID_ARG),
    ((4, 64, 0, PTR, 0, PTR + 8, PTR), fb.FLUX_ERR_INVALID_ARG), ((4, 64, 0, PTR, 0, PTR, PTR + 4), fb.FLUX_ERR_INVALID_ARG),
    ((4, 64, 1, PTR + 2, 0, PTR, PTR), fb.FLUX_ERR_INVALID_ARG), ((5, 64, 0, PTR, 1 << 62, PTR, PTR), fb.FLUX_ERR_SHAPE),
])
def test_reading_8_bit_blocks_refuses(args, status):
    rows, K, dtype, wide, ld, q, scales = args
    assert norm.lib().flux_mx8_dequantize(rows, K, q, scales, dtype, wide, ld, None) == status


def test_mx8_row_sizes():
    for K, q in ((1, 32), (32, 32), (33, 64), (512, 512), (513, 544)):
        assert norm.flux_mx8_row_bytes(K) == q
    assert norm.flux_mx8_row_bytes(0) == 0


# ---- loss ---------------------------------------------------------------------------------------------------------
def _loss(p, ws=(PTR, 1 << 50), **ptrs):
    names = ["X", "W", "target", "lse", "logit", "loss"]
    v = {n: PTR for n in names}
    v.update(ptrs)
    return loss.lib().flux_loss(None if p is None else ctypes.byref(p), *[v[n] for n in names], *ws, None)


def _loss_bwd(p, ws=(PTR, 1 << 50), **ptrs):
    names = ["X", "W", "target", "lse", "dloss", "dX", "dW"]
    v = {n: PTR for n in names}
    v.update(ptrs)
    return loss.lib().flux_loss_backward(None if p is None else ctypes.byref(p), *[v[n] for n in names], *ws, None)


@pytest.mark.parametrize("bad,status", [
    (dict(M=0), fb.FLUX_ERR_SHAPE), (dict(V=0), fb.FLUX_ERR_SHAPE), (dict(K=0), fb.FLUX_ERR_SHAPE), (dict(K=100), fb.FLUX_ERR_SHAPE), (dict(V=-5), fb.FLUX_ERR_SHAPE),
    (dict(ldx=248), fb.FLUX_ERR_SHAPE), (dict(ldw=260), fb.FLUX_ERR_SHAPE), (dict(ldx=-256), fb.FLUX_ERR_INVALID_ARG), (dict(ldw=1 << 62), fb.FLUX_ERR_SHAPE),
    (dict(M=1 << 24), fb.FLUX_ERR_SHAPE), (dict(V=1 << 24), fb.FLUX_ERR_SHAPE), (dict(target_dtype=2), fb.FLUX_ERR_INVALID_ARG),
    (dict(v0=-1), fb.FLUX_ERR_INVALID_ARG), (dict(vocab=-1), fb.FLUX_ERR_INVALID_ARG), (dict(vocab=999), fb.FLUX_ERR_SHAPE), (dict(v0=1, vocab=1000), fb.FLUX_ERR_SHAPE),
    (dict(M=1 << 20, V=(1 << 16) + 1, K=8), fb.FLUX_ERR_SHAPE), (dict(M=(1 << 27) + 1, V=8, K=8), fb.FLUX_ERR_SHAPE),
    (dict(v0=(1 << 62) + 1), fb.FLUX_ERR_SHAPE), (dict(vocab=(1 << 62) + 1), fb.FLUX_ERR_SHAPE),
    (dict(dloss_one=2), fb.FLUX_ERR_INVALID_ARG), (dict(dx_dtype=2), fb.FLUX_ERR_INVALID_ARG), (dict(dw_dtype=-1), fb.FLUX_ERR_INVALID_ARG),
    (dict(dw_accumulate=2), fb.FLUX_ERR_INVALID_ARG), (dict(piece=-64), fb.FLUX_ERR_INVALID_ARG), (dict(piece=100), fb.FLUX_ERR_SHAPE),
    (dict(tile_config=99), fb.FLUX_ERR_INVALID_ARG), (dict(split_k=65), fb.FLUX_ERR_INVALID_ARG), (dict(reserved=1), fb.FLUX_ERR_INVALID_ARG),
    (dict(tile_config=ffn.flux_ffn_tile_config_count()), fb.FLUX_ERR_UNSUPPORTED),
])
def test_loss_refuses_problems(bad, status):
    p = loss.loss_problem(256, 1000, 256)
    for k, v in bad.items():
        setattr(p, k, v)
    assert _loss(p) == status and _loss_bwd(p) == status
    assert loss.flux_loss_workspace_bytes(0, p) == 0 and loss.flux_loss_workspace_bytes(1, p) == 0


def test_loss_refuses_pointers_and_workspaces():
    p = loss.loss_problem(256, 1000, 256)
    for ptrs in (dict(X=0), dict(W=0), dict(target=0), dict(lse=0), dict(logit=0), dict(X=PTR + 8), dict(W=PTR + 2), dict(target=PTR + 4), dict(lse=PTR + 2), dict(loss=PTR + 1)):
        assert _loss(p, **ptrs) == fb.FLUX_ERR_INVALID_ARG, ptrs
    for ptrs in (dict(X=0), dict(W=0), dict(target=0), dict(lse=0), dict(dloss=0), dict(dX=PTR + 8), dict(dW=PTR + 4), dict(dloss=PTR + 2)):
        assert _loss_bwd(p, **ptrs) == fb.FLUX_ERR_INVALID_ARG, ptrs
    p.target_dtype = loss.FLUX_TARGET_I32
    assert _loss(p, target=PTR + 2) == fb.FLUX_ERR_INVALID_ARG
    for op, call in ((loss.FLUX_LOSS_FORWARD, _loss), (loss.FLUX_LOSS_BACKWARD, _loss_bwd)):
        need = loss.flux_loss_workspace_bytes(op, p)
        assert need > 0
        for ws in ((0, 0), (PTR, need - 1), (PTR + 8, need)):
            assert call(p, ws=ws) == fb.FLUX_ERR_WORKSPACE
        assert call(None) == fb.FLUX_ERR_INVALID_ARG
    assert loss.flux_loss_workspace_bytes(2, p) == 0


def test_a_piece_that_no_matrix_may_be_as_large_as():
    p = loss.loss_problem(1 << 17, 1 << 15, 64, piece=1 << 15)
    assert loss.flux_loss_workspace_bytes(loss.FLUX_LOSS_BACKWARD, p) == 0 and _loss_bwd(p) == fb.FLUX_ERR_SHAPE
    assert loss.flux_loss_workspace_bytes(loss.FLUX_LOSS_FORWARD, p) > 0


def test_the_backward_pass_holds_a_piece_and_not_the_logits():
    M, V, K = 8192, 32000, 8192
    for piece in (0, 64, 1024, 8192):
        p = loss.loss_problem(M, V, K, piece=piece)
        assert loss.flux_loss_workspace_bytes(loss.FLUX_LOSS_BACKWARD, p) < (2 * M * piece or 256 << 20) + 4 * M * K + (100 << 20)


def test_many_rows_get_small_pieces():
    p = loss.loss_problem(1 << 22, 1 << 14, 64)
    need = loss.flux_loss_workspace_bytes(loss.FLUX_LOSS_BACKWARD, p)
    assert 0 < need < 2 << 32
    p = loss.loss_problem(1 << 25, 1 << 11, 8)                        # (even 64 columns are too many)
    assert loss.flux_loss_workspace_bytes(loss.FLUX_LOSS_BACKWARD, p) == 0 and _loss_bwd(p) == fb.FLUX_ERR_SHAPE


def _join(p, R, lses=(PTR, PTR), logits=(PTR, PTR), target=PTR, out=(PTR, PTR, PTR)):
    lists = [None if v is None else (ctypes.c_void_p * len(v))(*v) for v in (lses, logits)]
    return loss.lib().flux_loss_join(None if p is None else ctypes.byref(p), R, *lists, target, *out, None)


def test_join_refuses():
    p = loss.loss_problem(256, 1000, 256)
    many = (PTR,) * 17
    for args in (dict(p=None), dict(R=0), dict(R=17, lses=many, logits=many), dict(lses=None), dict(logits=None), dict(target=0), dict(target=PTR + 4),
                 dict(lses=(PTR, 0)), dict(logits=(0, PTR)), dict(lses=(PTR, PTR + 1)), dict(out=(PTR + 1, 0, 0)), dict(out=(0, 0, PTR + 2))):
        assert _join(**{"p": p, "R": 2, **args}) == fb.FLUX_ERR_INVALID_ARG, args
    p.M = 0
    assert _join(p, 2) == fb.FLUX_ERR_SHAPE


# ---- the oracle ---------------------------------------------------------------------------------------------------
def test_oracle_norm_gradients_against_differences():
    rng = np.random.default_rng(1)
    s, w, dy, ds = rng.normal(size=(4, 9)), rng.normal(size=9), rng.normal(size=(4, 9)), rng.normal(size=(4, 9))
    f = lambda s_, w_: (no.norm(s_, w_, 1e-3)[0] * dy).sum() + (s_ * ds).sum()        # noqa: E731
    dr, dw = no.norm_backward(dy, s, w, no.norm(s, w, 1e-3)[1], ds)
    h = 1e-6
    for grad, at in ((dr, 0), (dw, 1)):
        d = rng.normal(size=grad.shape)
        ins = [[s, w], [s, w]]
        ins[0][at], ins[1][at] = ins[0][at] + h * d, ins[1][at] - h * d
        assert np.isclose((f(*ins[0]) - f(*ins[1])) / (2 * h), (grad * d).sum(), rtol=1e-7, atol=1e-8)


def test_oracle_loss_gradients_against_differences():
    rng = np.random.default_rng(2)
    x, w, dloss = rng.normal(size=(5, 4)), rng.normal(size=(7, 4)), rng.normal(size=5)
    target = np.array([0, 6, -100, 3, 7])
    f = lambda x_, w_: (no.loss(x_, w_, target, 0, 7)[2] * dloss).sum()               # noqa: E731
    lse = no.loss(x, w, target, 0, 7)[0]
    grads = no.loss_backward(x, w, target, 0, 7, lse, dloss)
    h = 1e-6
    for at in (0, 1):
        d = rng.normal(size=grads[at].shape)
        ins = [[x, w], [x, w]]
        ins[0][at], ins[1][at] = ins[0][at] + h * d, ins[1][at] - h * d
        assert np.isclose((f(*ins[0]) - f(*ins[1])) / (2 * h), (grads[at] * d).sum(), rtol=1e-7, atol=1e-8)
    assert not grads[0][[2, 4]].any()


def test_oracle_shards_are_the_whole():
    rng = np.random.default_rng(3)
    x, w = rng.normal(size=(6, 4)), rng.normal(size=(12, 4))
    target = np.array([0, 3, 4, 11, -1, 12])
    whole = no.loss(x, w, target, 0, 12)
    parts = [no.loss(x, w[v:v + 4], target, v, 12) for v in (0, 4, 8)]
    assert np.allclose(np.log(sum(np.exp(p[0]) for p in parts)), whole[0])
    assert np.allclose(sum(p[1] for p in parts), whole[1])
    assert (whole[2][4:] == 0).all()


def test_oracle_rounding_by_hand():
    x = np.zeros((1, 32))
    x[0, :10] = [448, 449, 479, -500, 17, 19, 2.0 ** -10, 3 * 2.0 ** -10, -0.0, 2.0 ** -9]
    codes, scales = no.blocks(x, 8)                      # the largest is 500: floor(log2) = 8, scale 1; 17 and 19 tie to 16 and 20
    assert scales[0, 0] == 127
    assert list(no.block_values(codes, scales, 8)[0, :10]) == [448, 448, 448, -448, 16, 20, 0, 2 * 2.0 ** -9, 0, 2.0 ** -9]
    for top, byte in ((1.0, 119), (0.999, 118), (2.0 ** -119, 0), (2.0 ** -118, 1), (2.0 ** -149, 0), (2.0 ** 127, 246), (np.inf, 255), (np.nan, 255), (0.0, 0)):
        x[:] = 0
        x[0, 3] = top
        assert no.blocks(x, 8)[1][0, 0] == byte, top
    x = np.random.default_rng(4).normal(size=(3, 70)) * 2.0 ** np.random.default_rng(5).integers(-20, 20, (3, 70))
    assert all((a == b).all() for a, b in zip(no.blocks(x, 4), oo.mx4_quantize(x)))
    assert no.E4M3[1] == 2.0 ** -9 and no.E4M3[126] == 448 and no.E4M3[56] == 1
