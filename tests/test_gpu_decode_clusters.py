"""Decode over rows in clusters of an odd number of blocks, at the most heads that take them (on 148 SMs: 7, 5 and 3 blocks a head)."""
import pytest

from paper_2510_20787_b200 import lte
from tests.test_gpu_decode_accum import KINDS, Run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("B,H,G,d,W,R,n,cnt", [(1, 18, 3, 128, 300, 700, 2000, 700), (1, 23, 5, 128, 200, 500, 900, 480), (2, 21, 9, 128, 130, 300, 700, 300),
                                               (1, 23, 2, 64, 300, 300, 900, 300), (2, 21, 4, 64, 2000, 500, 9000, 500)])
def test_odd_clusters(kind, B, H, G, d, W, R, n, cnt):
    r = Run(kind, "bf16", B, H, G, d, W, R, n, cnt, sink=1)
    for decay in (0.9, 0.0):
        r.step(decay=decay, which=[0, 1, H - 1, B * H - 1])
    assert lte.lte_device_status() == 0
