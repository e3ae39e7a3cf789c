"""Caches whose offsets pass 32 bits: 4 bits, conversions, fp32 steps."""
import pytest
import torch

from paper_2510_20787_b200 import lte
from tests.test_gpu_decode_accum import Run

pytestmark = pytest.mark.gpu


def _big(small, heads):
    """A cache of `heads` empty heads whose last two are those of `small`."""
    block = small.lay.stride
    cache = torch.zeros(256 + heads * block, dtype=torch.uint8, device="cuda")
    cache[-2 * block:] = small.cache[256:]
    return cache


def _near(a, b, e):
    return bool(((a.double() - b.double()).abs() <= e * b.double().abs().max()).all())


def test_4_bits_past_4_gigabytes():
    d, W, R, heads = 128, 2768, 30000, 900
    one = Run("accum", "bf16", 1, 2, 1, d, W, R, 90000, R)
    s = lte.shape(1, heads, 0, d, W, R, lte.BF16)
    ordinary = _big(one, heads)
    small = Run("four accum", "bf16", 1, 2, 1, d, W, R, 90000, R)
    cache4 = lte.lte_cache4_pack(s, ordinary)
    assert cache4.numel() > 2 ** 32
    block, plain = small.lay.stride, one.lay.stride
    assert torch.equal(cache4[-2 * block:], small.cache[256:])
    ordinary.fill_(255)
    lte.lte_cache4_unpack(s, cache4, cache=ordinary)
    assert torch.equal(ordinary[-2 * plain:], lte.lte_cache4_unpack(small.s, small.cache)[256:])
    del ordinary
    q, k, v = small.tokens()
    big = [torch.zeros((1, heads, d), dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    for x, y in zip(big, (q, k, v)):
        x[:, -2:] = y
    o, lse = lte.lte_attn_decode4_accum(s, cache4, *big)
    o2, l2 = small.call(q, k, v)
    # (other numbers of warps share a head: fp32 sums in another order, weights' products with steps rounded at another scale)
    assert _near(o[:, -2:], o2, 2.0 ** -7) and _near(lse[:, -2:], l2, 1e-6)
    got, want = cache4[-2 * block:].view(2, block), small.cache[256:].view(2, block)
    a, b = small.lay.at["score"]
    assert _near(got[:, a:b].view(torch.float32), want[:, a:b].view(torch.float32), 1e-6)
    assert torch.equal(got[:, :a], want[:, :a]) and torch.equal(got[:, b:], want[:, b:])
    assert bool((cache4[256:-2 * block].view(heads - 2, block)[:, small.lay.at["count"][0]:][:, :4].view(torch.int32) == 1).all())


@pytest.mark.parametrize("kind,d,heads", [("accum", 128, 140), ("four accum", 128, 900), ("four learned", 64, 1700)])
def test_fp32_steps_past_4_gigabytes(kind, d, heads):
    W, R = 2768, 30000
    small = Run(kind, "f32", 1, 2, 1, d, W, R, 90000, R)
    s = lte.shape(1, heads, 0, d, W, R, lte.F32)
    cache = _big(small, heads)
    assert cache.numel() > 2 ** 32
    q, k, v = small.tokens()
    big = [torch.zeros((1, heads, d), device="cuda") for _ in range(3)]
    for x, y in zip(big, (q, k, v)):
        x[:, -2:] = y
    if kind == "four learned":
        w, bias = torch.zeros((heads,) + small.w.shape[1:], device="cuda"), torch.zeros(heads, device="cuda")
        w[-2:], bias[-2:] = small.w, small.bias
        o, lse = lte.lte_attn_decode4(s, lte.conv(w, bias), cache, *big)
    else:
        o, lse = (lte.lte_attn_decode_accum if kind == "accum" else lte.lte_attn_decode4_accum)(s, cache, *big)
    o2, l2 = small.call(q, k, v)
    assert _near(o[:, -2:], o2, 1e-5) and _near(lse[:, -2:], l2, 1e-6)
    block = small.lay.stride
    got, want = cache[-2 * block:].view(2, block), small.cache[256:].view(2, block)
    a, b = small.lay.at["score"]
    x, y = got[:, a:b].view(torch.float32), want[:, a:b].view(torch.float32)
    same = torch.isfinite(y)
    assert torch.equal(torch.isfinite(x), same) and _near(x[same], y[same], 1e-6)
    assert torch.equal(got[:, :a], want[:, :a]) and torch.equal(got[:, b:], want[:, b:])
