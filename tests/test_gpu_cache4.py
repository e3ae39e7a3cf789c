"""GPU parity of the decode cache in 4 bits: packing and unpacking against the rule, and the calls in the order of a conversation."""
import numpy as np
import pytest
import torch

from paper_2510_20787_b200 import lte
from tests import rows_ref as ref

pytestmark = pytest.mark.gpu

SHAPES = [("bf16", 2, 2, 64, 100, 99), ("bf16", 1, 3, 64, 128, 128), ("bf16", 1, 2, 128, 77, 41), ("bf16", 1, 2, 32, 5, 0), ("f32", 2, 1, 64, 63, 65),
          ("f32", 1, 2, 32, 1, 1), ("f32", 1, 1, 128, 130, 7), ("bf16", 3, 2, 64, 768, 512)]


def caches(dtype, B, H, d, W, R, fill=None, seed=0):
    s = lte.shape(B, H, 0, d, W, R, lte.BF16 if dtype == "bf16" else lte.F32)
    lay = ref.Layout(s, False)
    g = torch.Generator(device="cuda").manual_seed(seed)
    cache = torch.zeros(lte.lte_cache_bytes(s), dtype=torch.uint8, device="cuda")
    blocks = cache[256:].view(B * H, -1)
    for name in ("k", "v"):
        a, b = lay.at[name]
        part = blocks[:, a:b].view(torch.bfloat16 if dtype == "bf16" else torch.float32)
        x = torch.randn(part.shape, generator=g, device="cuda")
        x = x if fill is None else fill(x)
        if lay.swizzled:
            x.view(B * H, 256, -1)[:, W + R:] = 0
        part.copy_(x)
    for name, t in (("score", torch.float32), ("pos", torch.int32), ("count", torch.int32)):
        a, b = lay.at[name]
        part = blocks[:, a:b].view(t)
        part.copy_(torch.randint(0, 1000, part.shape, generator=g, device="cuda"))
    return s, lay, cache


def check(s, lay, cache):
    before = lay.state(cache)
    keep = cache.clone()
    cache4 = lte.lte_cache4_pack(s, cache)
    assert torch.equal(cache, keep)
    lay4 = ref.Layout(s, True)
    assert cache4.numel() == 256 + s.B * s.H * lay4.stride == lte.lte_cache4_bytes(s)
    held = lay4.state(cache4)
    back = torch.full_like(cache, 255)
    lte.lte_cache4_unpack(s, cache4, cache=back)
    after = lay.state(back)
    for name in ("k", "v"):
        want = ref.four(before[name])[0]
        assert np.array_equal(held[name], want, equal_nan=True)
        t = torch.from_numpy(want)
        want = (t.to(torch.float32).to(torch.bfloat16) if s.dtype == lte.BF16 else t.to(torch.float32)).double().numpy()
        assert np.array_equal(after[name], want, equal_nan=True)
    for name in ("score", "pos", "count"):
        assert np.array_equal(held[name], before[name]) and np.array_equal(after[name], before[name])
    if lay.swizzled:                                           # the rows behind the last one stay zero
        for name in ("k", "v"):
            a, b = lay.at[name]
            assert not back[256:].view(-1, lay.stride)[:, a:b].view(-1, 256, 128)[:, s.W + s.R:].any()
    return cache4


@pytest.mark.parametrize("dtype,B,H,d,W,R", SHAPES)
def test_pack_and_unpack(dtype, B, H, d, W, R):
    check(*caches(dtype, B, H, d, W, R))


def _halves(x):                                                # many values half-way between two codes: step is 1/8 exactly, halves of it occur
    y = torch.randint(0, 31, x.shape, device=x.device).float() / 16
    y.view(-1, 32)[:, 0], y.view(-1, 32)[:, 1] = 0, 1.875
    return y


FILLS = {
    "ties": _halves,
    "offset": lambda x: 100 + x,
    "constant": lambda x: torch.full_like(x, -3.3),
    "zeros": torch.zeros_like,
    "tiny": lambda x: x * 1e-38,
    "subnormal": lambda x: x * 1e-40,
    "huge": lambda x: x * 1e37,
    "too wide": lambda x: x.sign() * 3.0e38,
    "not finite": lambda x: torch.where(x > 2.2, float("inf"), torch.where(x < -2.2, float("nan"), x)),
    "one infinite": lambda x: torch.where(torch.arange(x.numel(), device=x.device).view(x.shape) % 509 == 0, -float("inf"), x),
}


@pytest.mark.parametrize("fill", list(FILLS))
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_hard_values(dtype, fill):
    check(*caches(dtype, 1, 2, 64, 40, 24, FILLS[fill]))
    check(*caches(dtype, 1, 1, 128, 40, 24, FILLS[fill]))


def test_a_conversation():
    """Prompt, cache, into 4 bits, steps, back, the next turn's prompt as a chunk: the calls take each other's state, and the 4-bit steps
    stay near the same steps in bf16 (keys and values off by half a step of 4 bits at most)."""
    B, H, G, d, W, R, K, T, N, M = 2, 4, 2, 64, 96, 64, 7, 400, 40, 70
    g = torch.Generator(device="cuda").manual_seed(3)
    n = lambda *shape: torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    s = lte.shape(B, H, T, d, W, R, lte.BF16, group=G)
    c = lte.conv(torch.randn((H, K, 2 * d), generator=g, device="cuda") * 0.05)
    q, k, v = n(B, H * G, T, d), n(B, H, T, d), n(B, H, T, d)
    z = lte.lte_scores(s, c, k, v)
    idx, cnt = lte.lte_select(s, z)
    lte.lte_attn_prefill(s, q, k, v, idx, cnt)
    cache = lte.lte_cache_init(s, c, k, v, z, idx, cnt)
    cache4 = lte.lte_cache4_pack(s, cache)
    w = c._keep[0].double().cpu().numpy()
    off = []
    for _ in range(N):
        q1, k1, v1 = n(B, H * G, d), n(B, H, d), n(B, H, d)
        o, _ = lte.lte_attn_decode(s, c, cache, q1, k1, v1)
        o4, _ = ref.check_step(s, ref.Layout(s, True), cache4, q1, k1, v1, lambda: lte.lte_attn_decode4(s, c, cache4, q1, k1, v1), False, w=w)
        off.append(float((o4.float() - o.float()).norm() / o.float().norm()))
    # A channel is off by step / 2 at most, a step of a group of 32 normal values being about 4.1 / 15: 0.08 in the mean square, in
    # values and (through logits off by |q| 0.08 = 0.08 in the mean square) in weights.  The retained lists may part where logits are close.
    assert np.median(off) < 0.25
    back = lte.lte_cache4_unpack(s, cache4)
    s2 = lte.shape(B, H, M, d, W, R, lte.BF16, group=G)
    o, lse = lte.lte_attn_prefill_chunk(s2, c, back, T + N, n(B, H * G, M, d), n(B, H, M, d), n(B, H, M, d))
    assert bool(torch.isfinite(o.float()).all()) and bool(torch.isfinite(lse).all())
    assert lte.lte_device_status() == 0
    count = ref.Layout(s, False).part(back, "count", torch.int32)
    assert bool((count[:, 0] == T + N + M).all())


def test_accumulated_attention_from_prompt_to_4_bits():
    B, H, G, d, W, R, T = 2, 2, 4, 128, 64, 48, 300
    g = torch.Generator(device="cuda").manual_seed(4)
    n = lambda *shape: torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    s = lte.shape(B, H, T, d, W, R, lte.BF16, group=G, sink=2)
    q, k, v = n(B, H * G, T, d), n(B, H, T, d), n(B, H, T, d)
    idx, cnt = lte.lte_select_rule(s, lte.RULE_UNIFORM, device=q.device)
    _, lse = lte.lte_attn_prefill(s, q, k, v, idx, cnt)
    a = lte.lte_attn_colsum(s, q, k, lse, idx, cnt)
    idx, cnt = lte.lte_select_rule(s, lte.RULE_ACCUM_ATTN, a)
    cache = lte.lte_cache_init_accum(s, k, v, a, idx, cnt)
    st = ref.Layout(s, False).state(cache)
    for h in range(B * H):
        assert np.array_equal(st["pos"][h], idx.view(B * H, R)[h].cpu().numpy())
        assert np.array_equal(st["score"][h, W:], a.view(B * H, T)[h].double().cpu().numpy()[st["pos"][h]])
        assert np.array_equal(st["score"][h, np.arange(T - W, T) % W], a.view(B * H, T)[h, T - W:].double().cpu().numpy())
    cache4 = lte.lte_cache4_pack(s, cache)
    for _ in range(12):
        q1, k1, v1 = n(B, H * G, d), n(B, H, d), n(B, H, d)
        ref.check_step(s, ref.Layout(s, False), cache, q1, k1, v1, lambda: lte.lte_attn_decode_accum(s, cache, q1, k1, v1, decay=0.97), True, 0.97)
        ref.check_step(s, ref.Layout(s, True), cache4, q1, k1, v1, lambda: lte.lte_attn_decode4_accum(s, cache4, q1, k1, v1, decay=0.97), True, 0.97)
    assert lte.lte_device_status() == 0
