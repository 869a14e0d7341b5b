"""CPU-only: what the loss launches reads nothing past the end of its matrices.  The launches are noted by tests/launch_recorder.py, and the places that a grid of
tiles reads are worked out from the arguments, in whole numbers of any size."""
import pytest
from launch_recorder import record

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
