"""CPU-only: what the loss launches reads nothing past the end of its matrices.  The launches are noted by tests/launch_recorder.py, and the places that a grid of
tiles reads are worked out from the arguments, in whole numbers of any size."""
import random

import pytest
from launch_recorder import WORKSPACE, record

from paper_2406_06858_amd import binding as fb
from paper_2406_06858_amd import loss

ALONG, DX, DW = 2, 3, 4                        # kinds of tile kernels: both operands along the contraction; the second across; both across
BACKWARD = range(7)                            # X, W, target, lse, dloss, dX, dW


def _reads(t):
    """Bytes of A and of B up to the end of the last row that a kernel without masks reads."""
    rows, cols, depth = t["tiles_m"] * t["bm"], t["tiles_n"] * t["bn"], t["slabs"] * 64
    across = lambda n, pitch: (depth - 1) * pitch + n * 2              # noqa: E731
    along = lambda n, pitch: (n - 1) * pitch + depth * 2               # noqa: E731
    return (across if t["kind"] == DW else along)(rows, t["pitch_a"]), (along if t["kind"] == ALONG else across)(cols, t["pitch_b"])


def _check(call, problem):
    assert call["status"] == 0, problem
    assert all(g * b < 1 << 32 for t in call["launches"] for g, b in zip(t["grid"], t["block"])), problem
    tiles = [t for t in call["launches"] if "kind" in t]
    for t in tiles:
        if not t["masked"]:
            a, b = _reads(t)
            assert a <= t["bytes_a"] and b <= t["bytes_b"], (problem, t["name"], a - t["bytes_a"], b - t["bytes_b"])
    return tiles


@pytest.mark.parametrize("M,K", [(256, 256), (8192, 1024), (128, 4096)])
def test_gradients_read_no_row_past_the_weights(tmp_path, M, K):
    """Every width of the last slab of a vocabulary; M and K are multiples of all tiles.  (dX runs over V rows of weights, and dZ is in whole vectors of 8.)"""
    problems = [dict(M=M, V=V, K=K, **kw) for V in list(range(4033, 4097)) + [30522, 50303, 57, 63] for kw in ({}, {"piece": 1024})]
    calls = record(tmp_path, [("flux_loss_backward", p, BACKWARD) for p in problems])
    masks = set()
    for call, p in zip(calls, problems):
        dx = [t for t in _check(call, p) if t["kind"] == DX]
        assert dx
        masks.update(t["masked"] for t in dx)
    assert masks == {0, 1}


def _whole_vectors(n):
    return (n + 7) // 8 * 8


def _extents(t):
    """Bytes that A and B span, as the buffers' records have to say it (whole numbers of any size)."""
    across = lambda n, pitch: (t["depth"] - 1) * pitch + n * 2         # noqa: E731
    along = lambda n, pitch, row: (n - 1) * pitch + row * 2            # noqa: E731
    rows, cols, depth = t["rows"], t["cols"], t["depth"]
    if t["kind"] == DW:
        return across(_whole_vectors(rows), t["pitch_a"]), across(cols, t["pitch_b"])
    row = depth if t["kind"] == ALONG else _whole_vectors(depth)
    return along(rows, t["pitch_a"], row), along(cols, t["pitch_b"], depth) if t["kind"] == ALONG else across(cols, t["pitch_b"])


# X below 2^31 elements as it is, and not with its rows rounded up to whole lines; on either side of the border; with a pitch of its own; far from it
WIDE = [dict(M=420000, V=50257, K=5112), dict(M=2120000, V=32000, K=1000), dict(M=419430, V=50257, K=5112), dict(M=419431, V=50257, K=5112),
        dict(M=420000, V=50257, K=5040, ldx=5112), dict(M=8192, V=50257, K=5112)]


@pytest.mark.parametrize("function,pointers", [("flux_loss", range(6)), ("flux_loss_backward", BACKWARD)])
def test_buffers_span_what_their_32_bits_say(tmp_path, function, pointers):
    calls = record(tmp_path, [(function, p, pointers) for p in WIDE])
    for call, p in zip(calls, WIDE):
        tiles = _check(call, p)
        assert tiles
        for t in tiles:
            assert (t["bytes_a"], t["bytes_b"]) == _extents(t) and max(_extents(t)) < 1 << 32, (p, t["name"], t["bytes_a"], t["bytes_b"], _extents(t))


def test_a_copy_is_made_where_its_offsets_fit():
    """The forward pass's workspace has room for X in whole lines, or has not.  (Everything else in it is smaller.)"""
    fit = [(p["M"] - 1) * ((p["K"] + 63) // 64 * 64) + p["K"] < 1 << 31 for p in WIDE]
    assert fit == [False, False, True, False, True, True]
    for p, fits in zip(WIDE, fit):
        need = loss.flux_loss_workspace_bytes(loss.FLUX_LOSS_FORWARD, loss.loss_problem(**p))
        assert (need >= 2 * p["M"] * ((p["K"] + 63) // 64 * 64)) == fits, p


def test_results_have_their_places_in_32_bits(tmp_path):
    """A result's place in its row is counted in bytes, a tile's past the last column too.  Wider rows are refused."""
    problems = [dict(M=M, V=V, K=K, dx_dtype=dtype, dw_dtype=dtype) for K in (1 << 28, (1 << 28) + 8, 1 << 29, (1 << 29) + 4096, 3 << 28, 1 << 30, (1 << 31) - 8)
                for M, V in ((1, 1), (3, 7), (2, 2)) if max(M, V) * K < 1 << 31 for dtype in ("bf16", "f32")]
    calls = record(tmp_path, [("flux_loss_backward", p, BACKWARD) for p in problems])
    for call, p in zip(calls, problems):
        if p["K"] > 1 << 28:
            assert call["status"] == fb.FLUX_ERR_SHAPE and not call["launches"], p
            assert loss.flux_loss_workspace_bytes(loss.FLUX_LOSS_BACKWARD, loss.loss_problem(**p)) == 0
            continue
        for t in _check(call, p):
            assert t["tiles_n"] * t["bn"] * 4 < 1 << 31, (p, t["name"])


def _some_problem(rng):
    """Sizes over their logarithm, in turn whole tiles, multiples of 8 and 64 and odd; pitches, pieces, tiles and cuts of the caller's own."""
    size = lambda most, step: max(step, int(most ** rng.random()) // step * step)      # noqa: E731
    while True:
        step = rng.choice([1, 1, 8, 64, 256])
        p = dict(M=size(rng.choice([128, 20000, 1 << 22]), step), V=size(rng.choice([5000, 60000, 1 << 20]), step), K=size(rng.choice([2048, 16384]), rng.choice([8, 8, 64, 256])))
        if rng.random() < 0.2:
            p["ldx"], p["ldw"] = p["K"] + 8 * rng.randrange(0, 20), p["K"] + 8 * rng.randrange(0, 20)
        if rng.random() < 0.3:
            p["piece"] = 64 * rng.randrange(1, 200)
        if rng.random() < 0.3:
            p["tile_config"], p["split_k"] = rng.randrange(0, 7), rng.randrange(0, 9)
        p.update(dx_dtype=rng.choice(["bf16", "f32"]), dw_dtype=rng.choice(["bf16", "f32"]), dloss_one=rng.randrange(2))
        if loss.flux_loss_workspace_bytes(loss.FLUX_LOSS_BACKWARD, loss.loss_problem(**p)) > 0:
            return p


@pytest.mark.parametrize("function,pointers,op", [("flux_loss", range(6), loss.FLUX_LOSS_FORWARD), ("flux_loss_backward", BACKWARD, loss.FLUX_LOSS_BACKWARD)])
def test_any_problem_stays_in_its_buffers(tmp_path, function, pointers, op):
    rng = random.Random(function)
    problems = [_some_problem(rng) for _ in range(600)]
    calls = record(tmp_path, [(function, p, pointers) for p in problems])
    kinds = set()
    for call, p in zip(calls, problems):
        end = WORKSPACE + loss.flux_loss_workspace_bytes(op, loss.loss_problem(**p))
        for t in call["launches"]:
            if "terms" in t:
                assert t["xt"] - t["zt"] == t["rows"] * t["terms"] * 2 and t["xt"] + t["cols"] * t["terms"] * 2 <= end and t["grid"][1] * t["rows_each"] >= t["rows"], p
                kinds.add("outer")
        for t in _check(call, p):
            bytes_a, bytes_b = _extents(t)
            assert (t["bytes_a"], t["bytes_b"]) == (bytes_a, bytes_b), (p, t["name"])
            held = [(t["a"][0], bytes_a), (t["b"][0], bytes_b)]
            if t["kind"] != ALONG:
                held.append((t["out"][0], ((t["rows"] - 1) * t["ld"] + t["cols"]) * (4 if t["out_f32"] else 2)))
            if t["kind"] == DX and t["addend"]:
                held.append((t["addend"], ((t["rows"] - 1) * t["ld"] + t["cols"]) * 4))
            if t["cut_tiles"]:
                held.append((t["partial"], t["cut_tiles"] * t["parts"] * t["bm"] * t["bn"] * 4))
                assert t["counters"] == WORKSPACE and t["cut_tiles"] <= 512 and (t["parts"] - 1) * t["part_slabs"] < t["slabs"] <= t["parts"] * t["part_slabs"], p
            lx, lw = p.get("ldx", p["K"]), p.get("ldw", p["K"])
            x, w = (p["M"] - 1) * lx + p["K"], (p["V"] - 1) * lw + p["K"]
            ends = {0: x * 2, 1: w * 2, 5: x * (2, 4)[p["dx_dtype"] == "f32"], 6: w * (2, 4)[p["dw_dtype"] == "f32"], (WORKSPACE >> 40) - 1: end - WORKSPACE}
            for at, size in held:
                assert at % (1 << 40) + size <= ends[(at >> 40) - 1], (p, t["name"], at, size)
            assert t["full_tiles"] + t["cut_tiles"] == t["tiles_m"] * t["tiles_n"] and t["grid"][0] == t["full_tiles"] + t["cut_tiles"] * t["parts"], p
            kinds.add((t["kind"], t["masked"], bool(t["cut_tiles"])))
    assert {(ALONG, m, c) for m in (0, 1) for c in (False, True)} <= kinds
    if op == loss.FLUX_LOSS_BACKWARD:
        assert {(k, 1, c) for k in (DX, DW) for c in (False, True)} | {(DX, 0, False), (DW, 0, False), "outer"} <= kinds


def test_grids_of_gradients_at_their_limits(tmp_path):
    problems = [dict(M=1, V=(1 << 28) - 1, K=8), dict(M=64, V=(1 << 28) - 1, K=8), dict(M=100, V=(1 << 28) - 64, K=8), dict(M=(1 << 25) - 1, V=64, K=56), dict(M=(1 << 25) - 1, V=2047, K=8, piece=64),
                dict(M=1, V=7, K=1 << 28), dict(M=7, V=7, K=1 << 28), dict(M=129, V=1, K=(1 << 24) - (1 << 18)), dict(M=3, V=(1 << 21) + 1, K=1016)]
    problems = [dict(p, dx_dtype=dtype, dw_dtype=dtype) for p in problems for dtype in ("bf16", "f32")]
    for call, p in zip(record(tmp_path, [("flux_loss_backward", p, BACKWARD) for p in problems]), problems):
        assert _check(call, p)


def test_grids_are_below_2_32_threads(tmp_path):
    """The most tiles that the limits on M, V and K allow, both sides rounded up."""
    problems = [dict(M=133956083, V=513, K=8), dict(M=1 << 27, V=512, K=8), dict(M=(1 << 27) - 64 + 1, V=449, K=8), dict(M=1, V=(1 << 28) - 8, K=8), dict(M=257, V=(1 << 27) - 1, K=8),
                dict(M=(1 << 25) - 1, V=2047, K=8), dict(M=512, V=1 << 27, K=8)]
    problems = [dict(p, tile_config=config) for p in problems for config in range(7)]
    tiles = 0
    for call, p in zip(record(tmp_path, [("flux_loss", p, range(6)) for p in problems]), problems):
        assert call["status"] == 0 and all(g * b < 1 << 32 for t in call["launches"] for g, b in zip(t["grid"], t["block"])), p
        tiles = max([tiles] + [t["grid"][0] for t in call["launches"] if "kind" in t])
    assert 1 << 23 < tiles < 1 << 24
