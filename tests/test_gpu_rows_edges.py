"""Decode over rows where scores are NaN."""
import numpy as np
import pytest
import torch

from paper_2510_20787_b200 import lte
from tests.test_gpu_decode_accum import Run

pytestmark = pytest.mark.gpu

NANS = [0x7fc00000, -0x400000, 0x7f800001, -1]                 # quiet, negative, signalling, all bits set


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["accum", "four accum"])
@pytest.mark.parametrize("nan", NANS)
def test_scores_that_are_nan_rank_above_every_number(nan, kind, dtype):
    W, R, n = 16, 12, 100

    def after(leaving, pool):
        """Positions in the pool, in slot order, after a step in which the token n - W has the score `leaving` (an int: its bits)."""
        r = Run(kind, dtype, 1, 2, 1, 64, W, R, n, R)
        blocks = r.cache[256:].view(2, -1)
        score = blocks[:, r.lay.at["score"][0]:r.lay.at["score"][1]].view(torch.int32)
        bits = lambda x: x if isinstance(x, int) else int(np.float32(x).view(np.int32))  # noqa: E731
        score[:, n % W] = bits(leaving)
        for m, x in enumerate(pool):
            score[:, W + m] = bits(x)
        before = r.lay.part(r.cache, "pos", torch.int32).cpu().numpy()
        r.call(*r.tokens())
        pos = r.lay.part(r.cache, "pos", torch.int32).cpu().numpy()
        assert np.array_equal(pos[0] != before[0], pos[1] != before[1])
        gone = np.flatnonzero(pos[0] != before[0])
        assert (pos[:, gone] == n - W).all() and len(gone) <= 1
        return gone.tolist()
    numbers = [float(x) for x in range(5, 5 + R)]
    assert after(nan, numbers) == [0]                          # above the highest number too: the lowest goes
    assert after(nan, [float("inf")] * 3 + numbers[3:]) == [3]
    assert after(7.5, [nan] * 2 + numbers[2:]) == [2]          # the lowest number goes, not a NaN
    assert after(float("inf"), [nan] * R) == []                # nothing that is a number gets past NaN
    assert after(nan, [nan] * R) == []                         # no more than the entry has: stays out
    assert after(nan, [nan] * (R - 1) + [float("inf")]) == [R - 1]
