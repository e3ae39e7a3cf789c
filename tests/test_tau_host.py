"""Calls that have no threshold take any tau (nothing is launched: each call is refused for another reason, which stands behind the shape's checks)."""
import ctypes

import pytest

from paper_2510_20787_b200 import lte

FAKE = 4096


@pytest.mark.parametrize("tau", [1.0, 2.0, float("inf"), float("nan")])
def test_calls_without_a_threshold_ignore_tau(tau):
    L, a = lte.lib(), ctypes.addressof
    s = lte.shape(2, 3, 64, 64, 16, 8, lte.BF16, tau=tau)
    assert lte.lte_cache4_bytes(s) == lte.lte_cache4_bytes(lte.shape(2, 3, 64, 64, 16, 8, lte.BF16)) > 0
    long = lte.shape(1, 2, 64, 64, 768, 32001, lte.BF16, tau=tau)
    conv = lte.LteConv(1, 7, 1, 256, 0)
    six = [FAKE] * 6 + [None]
    assert L.lte_attn_decode_accum(a(long), 1.0, *six) == -2 == L.lte_attn_decode4_accum(a(long), 1.0, *six)
    assert L.lte_cache_init_accum(a(long), *six) == -2
    assert L.lte_cache4_pack(a(long), FAKE, 2 * FAKE, None) == -2 == L.lte_cache4_unpack(a(long), FAKE, 2 * FAKE, None)
    assert L.lte_attn_decode4(a(s), a(conv), *six) == -1       # the learned rule has one
    far = lte.shape(1, 1, 2 ** 24 + 64, 32, 16, 8, lte.BF16, tau=tau)
    assert L.lte_select_rule(a(far), lte.RULE_ACCUM_ATTN, FAKE, FAKE, FAKE, None, None, 0, None) == -2
    assert L.lte_select_rule(a(far), lte.RULE_LEARNED, FAKE, FAKE, FAKE, None, None, 0, None) == -1
