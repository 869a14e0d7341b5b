"""CPU-only: the norm's grids at the limits of its problems, noted by tests/launch_recorder.py.  A launch takes fewer than 2^32 threads along a direction."""
import pytest
from launch_recorder import record

SIZES = [(1, 1 << 30), (1, (1 << 30) - 1), (1, 1 << 29), (3, (1 << 29) + 1), (1, (1 << 29) - 32), (2, (1 << 28) + 8), ((1 << 31) - 1, 1), ((1 << 27) + 5, 15), ((1 << 24) - 1, 128),
         ((1 << 21), 1023), ((1 << 18) - 1, 8192), (1 << 17, 12288), ((1 << 17) - 1, 16384), (1 << 16, 32767), (60000, 33000)]


@pytest.mark.parametrize("function,pointers,outs", [("flux_norm", (0, 1, 2, 3, 4, 6), ("bf16", "f32")), ("flux_norm", range(7), ("mx4", "mx8")),
                                                    ("flux_norm_backward", range(8), ("bf16", "f32"))])
def test_grids_are_below_2_32_threads(tmp_path, function, pointers, outs):
    problems = [dict(M=M, K=K, s_dtype=s, out=out) for M, K in SIZES for s in ("bf16", "f32") for out in outs]
    for call, p in zip(record(tmp_path, [(function, p, pointers) for p in problems]), problems):
        assert call["status"] == 0 and call["launches"], p
        for t in call["launches"]:
            assert all(g * b < 1 << 32 for g, b in zip(t["grid"], t["block"])), (p, t)
