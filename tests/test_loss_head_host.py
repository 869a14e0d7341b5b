"""CPU-only: examples/loss_head.py refuses what it cannot share out, before it makes a buffer."""
import os
import sys

import pytest

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import loss_head  # noqa: E402


@pytest.mark.parametrize("M,R", [(10, 4), (3, 4), (129, 2), (0, 2)])
def test_tokens_that_the_ranks_cannot_share(M, R):
    with pytest.raises(ValueError, match="tokens"):
        loss_head.LossHead(M, 64, 16, R)
