"""Host-side checks of the calls on caches that evict by accumulated attention or hold 4 bits (nothing is launched), and the reference
of their GPU tests against small cases worked by hand."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2510_20787_b200 import lte
from tests import rows_ref as ref

FAKE = 4096                                                    # never dereferenced: validation fails first


def test_refusals():
    L, a = lte.lib(), ctypes.addressof
    s = lte.shape(1, 2, 64, 64, 16, 8, lte.BF16)
    conv = lte.LteConv(1, 7, 1, 256, 0)
    args = {"accum": [a(s), 1.0] + [FAKE] * 6 + [None], "four": [a(s), a(conv)] + [FAKE] * 6 + [None], "four accum": [a(s), 1.0] + [FAKE] * 6 + [None]}
    calls = {"accum": L.lte_attn_decode_accum, "four": L.lte_attn_decode4, "four accum": L.lte_attn_decode4_accum}

    def call(kind, at=None, to=None):
        x = list(args[kind])
        if at is not None:
            x[at] = to
        return calls[kind](*x)
    for kind in calls:
        assert call(kind, 0, None) == -1
        for i in range(2, 8):
            assert call(kind, i, None) == -1                   # no cache, q1, k1, v1, o1, lse1
        for i in range(2, 6):
            assert call(kind, i, FAKE + 8) == -1               # off a 16-byte boundary
        assert call(kind, 6, FAKE + 1) == -1 and call(kind, 7, FAKE + 2) == -1
        for bad in (lte.shape(0, 2, 0, 64, 16, 8, lte.BF16), lte.shape(1, 2, 0, 64, 0, 8, lte.BF16), lte.shape(1, 2, 0, 64, 16, -1, lte.BF16),
                    lte.shape(1, 2, 0, 64, 16, 8, 7), lte.shape(1, 2, 0, 64, 16, 8, lte.BF16, group=-1), lte.shape(1, 2, 0, 64, 16, 8, lte.BF16, sink=-1)):
            assert call(kind, 0, a(bad)) == -1
        for bad in (lte.shape(1, 2, 0, 48, 16, 8, lte.BF16), lte.shape(1, 2, 0, 64, 768, 32001, lte.BF16), lte.shape(1, 2, 0, 64, 2 ** 31 - 1, 2 ** 31 - 1, lte.BF16),
                    lte.shape(2 ** 15, 2 ** 15, 0, 64, 16, 8, lte.BF16)):
            assert call(kind, 0, a(bad)) == -2
    for kind in ("accum", "four accum"):
        for decay in (-0.01, 1.01, float("nan"), float("inf")):
            assert call(kind, 1, decay) == -1
    assert call("four", 1, None) == -1
    for bad, status in ((lte.LteConv(1, 6, 1, 256, 0), -1), (lte.LteConv(1, 17, 1, 256, 0), -1), (lte.LteConv(1, 7, 1, 0, 0), -1), (lte.LteConv(1, 7, 1, 258, 0), -1), (lte.LteConv(1, 7, 1, 256, 258), -1),
                        (lte.LteConv(3, 3, 2, 256, 0), -2)):
        assert call("four", 1, a(bad)) == status
    narrow = lte.shape(1, 2, 0, 64, 5, 8, lte.BF16)
    assert call("four", 0, a(narrow)) == -1                    # a window shorter than the receptive field
    # set-up and conversion
    init = [a(s)] + [FAKE] * 6 + [None]
    for i in range(0, 7):
        x = list(init)
        x[i] = None
        assert L.lte_cache_init_accum(*x) == -1
    x = list(init); x[6] = FAKE + 4
    assert L.lte_cache_init_accum(*x) == -1
    x = list(init); x[1] = FAKE + 1
    assert L.lte_cache_init_accum(*x) == -1
    long, odd = lte.shape(1, 2, 64, 64, 768, 32001, lte.BF16), lte.shape(1, 2, 0, 48, 16, 8, lte.BF16)
    x = list(init); x[0] = a(long)
    assert L.lte_cache_init_accum(*x) == -2
    for f in (L.lte_cache4_pack, L.lte_cache4_unpack):
        assert f(None, FAKE, 2 * FAKE, None) == f(a(s), None, FAKE, None) == f(a(s), FAKE, None, None) == -1
        assert f(a(s), FAKE, FAKE, None) == f(a(s), FAKE + 8, 2 * FAKE, None) == f(a(s), FAKE, 2 * FAKE + 8, None) == -1
        assert f(a(odd), FAKE, 2 * FAKE, None) == -2
        first = lte.lte_cache_bytes(s) if f is L.lte_cache4_pack else lte.lte_cache4_bytes(s)
        assert f(a(s), FAKE, FAKE + first - 16, None) == -1    # overlapping


@pytest.mark.parametrize("d,W,R", [(32, 16, 8), (64, 768, 512), (128, 77, 41), (32, 5, 0), (32, 1, 2)])
def test_sizes(d, W, R):
    rows = W + R
    per = sum((x + 15) // 16 * 16 for x in (rows * d // 2, rows * d // 2, rows * d // 8, rows * d // 8, rows * 4, R * 4)) + 16
    s = lte.shape(3, 2, 0, d, W, R, lte.BF16)
    assert lte.lte_cache4_bytes(s) == 256 + 6 * ((per + 255) // 256 * 256)
    assert lte.lte_cache4_bytes(s) == 256 + 6 * ref.Layout(s, True).stride and lte.lte_cache_bytes(s) == 256 + 6 * ref.Layout(s, False).stride
    assert lte.lte_cache4_bytes(lte.shape(3, 2, 0, 40, W, R, lte.BF16)) == 0 == lte.lte_cache4_bytes(lte.shape(3, 2, 0, d, 1, 32768, lte.BF16))


def test_the_rule_by_hand():
    x = np.zeros(32, np.float32)
    x[:6] = [-1.0, 14.0, 0.0, 0.49, 0.5, 1.5]                  # zero -1, step 1: codes 0, 15, 1, 1 (1.49), 2 (1.5, to even), 2 (2.5, to even)
    val, step, zero = ref.four(x)
    assert step[0] == 1 and zero[0] == -1
    assert val[:7].tolist() == [-1, 14, 0, 0, 1, 1, 0]
    assert np.isnan(ref.four(np.full(32, np.inf, np.float32))[0]).all()
    assert (ref.four(np.full(32, 7.0, np.float32))[0] == 7).all()


def test_the_reference_step_by_hand():
    """A window of 2, a pool of 1, keys of zero (equal weights): scores, the replaced entry and the output by hand."""
    s = lte.shape(1, 1, 0, 32, 2, 1, lte.F32)
    lay = ref.Layout(s, False)
    before = {"k": np.zeros((1, 3, 32)), "v": np.zeros((1, 3, 32)), "score": np.array([[5.0, 3.0, 4.0]]), "pos": np.array([[1]]), "count": np.array([[6, 1, 0, 0]])}
    before["v"][0, :, 0] = [1, 2, 4]                           # ring: positions 4, 5; pool: position 1
    one = torch.zeros((1, 1, 32))
    v1 = torch.zeros((1, 1, 32)); v1[..., 0] = 9
    st, o, lse, _ = ref.step(s, lay, before, one, one, v1, True, decay=0.5)
    # position 4 (score 5) leaves slot 0 and beats the pool's 4: attended are 4, 5 and the new token, a third each
    assert np.allclose(o[0, 0, 0], (1 + 2 + 9) / 3) and np.allclose(lse, np.log(3))
    assert np.allclose(st["score"], [[1 / 3, 1.5 + 1 / 3, 2.5 + 1 / 3]]) and st["pos"][0, 0] == 4 and st["count"][0].tolist() == [7, 1, 0, 0]
    assert st["v"][0, :, 0].tolist() == [9, 2, 1]
    before["score"][0, 2] = 5.0                                # no more than the entry has: stays out, and is not attended
    st, o, lse, _ = ref.step(s, lay, before, one, one, v1, True, decay=0.5)
    assert np.allclose(o[0, 0, 0], (2 + 4 + 9) / 3) and st["pos"][0, 0] == 1
    assert np.allclose(st["score"], [[1 / 3, 1.5 + 1 / 3, 2.5 + 1 / 3]])
