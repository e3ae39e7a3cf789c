"""Caches say what they hold: a call that cannot read one says so and, but for lte_attn_decode, leaves it alone."""
import pytest
import torch

from paper_2510_20787_b200 import lte
from tests import rows_ref as ref

pytestmark = pytest.mark.gpu

TYPES = {"bf16": (lte.BF16, torch.bfloat16), "f32": (lte.F32, torch.float32)}


class World:
    def __init__(self, dtype, d, W, R, G=1, H=3, T=200):
        self.g = torch.Generator(device="cuda").manual_seed(7)
        self.dt, B = TYPES[dtype][1], 2
        self.T, self.G, self.H, self.d = T, G, H, d
        self.s = s = lte.shape(B, H, T, d, W, R, TYPES[dtype][0], group=G)
        self.w = self.n(H, 5, 2 * d, plain=True) * 0.05
        self.c = lte.conv(self.w)
        q, k, v = self.n(B, H * G, T, d), self.n(B, H, T, d), self.n(B, H, T, d)
        z = lte.lte_scores(s, self.c, k, v)
        idx, cnt = lte.lte_select(s, z)
        self.learned = lte.lte_cache_init(s, self.c, k, v, z, idx, cnt)
        _, lse = lte.lte_attn_prefill(s, q, k, v, idx, cnt)
        a = lte.lte_attn_colsum(s, q, k, lse, idx, cnt)
        self.accum = lte.lte_cache_init_accum(s, k, v, a, *lte.lte_select_rule(s, lte.RULE_ACCUM_ATTN, a))
        self.learned4, self.accum4 = lte.lte_cache4_pack(s, self.learned), lte.lte_cache4_pack(s, self.accum)

    def n(self, *size, plain=False):
        x = torch.randn(size, generator=self.g, device="cuda")
        return x if plain else x.to(self.dt)

    def token(self):
        return self.n(2, self.H * self.G, self.d), self.n(2, self.H, self.d), self.n(2, self.H, self.d)


SHAPES = [("bf16", 64, 40, 60, 1), ("bf16", 64, 300, 60, 1), ("bf16", 64, 40, 60, 4), ("bf16", 128, 700, 900, 2), ("bf16", 32, 20, 30, 1),
          ("f32", 64, 40, 60, 1), ("f32", 32, 300, 1000, 1), ("f32", 128, 100, 60, 3), ("f32", 64, 700, 900, 2)]


@pytest.mark.parametrize("dtype,d,W,R,G", SHAPES)
def test_what_cannot_be_read_is_reported(dtype, d, W, R, G):
    w = World(dtype, d, W, R, G)
    s, c, M = w.s, w.c, 9
    assert lte.lte_device_status() == 0
    s2 = lte.shape(2, w.H, M, d, W, R, s.dtype, group=G)
    chunk = (w.n(2, w.H * G, M, d), w.n(2, w.H, M, d), w.n(2, w.H, M, d))
    o, lse = torch.full((2, w.H * G, d), 3.0, dtype=w.dt, device="cuda"), torch.full((2, w.H * G), 3.0, device="cuda")
    back = lte.lte_cache4_unpack(s, w.accum4)
    big = torch.cat([w.accum4, w.accum4.new_zeros(lte.lte_cache_bytes(s))])       # a buffer long enough for any cache
    left_alone = [
        (w.accum, lambda x: lte.lte_attn_prefill_chunk(s2, c, x, w.T, *chunk)),
        (w.accum, lambda x: lte.lte_attn_prefill_chunk(s2, c, x, w.T, *chunk, streaming=True)),
        (back, lambda x: lte.lte_attn_prefill_chunk(s2, c, x, w.T, *chunk)),
        (w.accum4, lambda x: lte.lte_attn_decode4(s, c, x, *w.token(), o1=o, lse1=lse)),
        (w.accum, lambda x: lte.lte_attn_decode4(s, c, x, *w.token(), o1=o, lse1=lse)),
        (w.accum, lambda x: lte.lte_attn_decode4_accum(s, x, *w.token(), o1=o, lse1=lse)),
        (big, lambda x: lte.lte_attn_decode_accum(s, x, *w.token(), o1=o, lse1=lse)),
        (w.accum, lambda x: lte.lte_cache4_unpack(s, x, cache=torch.empty_like(back))),
    ]
    if d != 128 and W >= 20:
        stack = lte.conv_stack([w.n(w.H, d, 3, 2 * d, plain=True), w.n(w.H, d // 2, 3, d, plain=True), w.n(w.H, d // 4, 3, d // 2, plain=True)], w.n(w.H, d // 4, plain=True))
        left_alone.append((w.accum, lambda x: lte.lte_cache_score(s, stack, x)))
    for i, (cache, call) in enumerate(left_alone):
        x = cache.clone()
        call(x)
        assert lte.lte_device_status() == -6, i
        assert torch.equal(x, cache), i
    assert bool((o == 3).all()) and bool((lse == 3).all())
    lte.lte_attn_decode(s, c, w.accum.clone(), *w.token())     # says so too, but writes (fp32 steps of one query head do not look)
    assert lte.lte_device_status() == (0 if dtype == "f32" and G == 1 else -6)


@pytest.mark.parametrize("dtype,d,W,R,G", SHAPES)
def test_what_can_be_read_is_not(dtype, d, W, R, G):
    w = World(dtype, d, W, R, G)
    s, c, M = w.s, w.c, 9
    s2 = lte.shape(2, w.H, M, d, W, R, s.dtype, group=G)
    assert not bool(w.learned[:256].any())
    for _ in range(2):
        lte.lte_attn_decode(s, c, w.learned, *w.token())
        lte.lte_attn_decode_accum(s, w.accum, *w.token())
        lte.lte_attn_decode4(s, c, w.learned4, *w.token())
        lte.lte_attn_decode4_accum(s, w.accum4, *w.token())
    again = lte.lte_cache4_pack(s, lte.lte_cache4_unpack(s, w.accum4))
    lte.lte_attn_decode4_accum(s, again, *w.token())
    lte.lte_attn_decode_accum(s, lte.lte_cache4_unpack(s, again), *w.token())
    back = lte.lte_cache4_unpack(s, w.learned4)
    assert not bool(back[:256].any())
    lte.lte_attn_prefill_chunk(s2, c, back, w.T + 2, w.n(2, w.H * G, M, d), w.n(2, w.H, M, d), w.n(2, w.H, M, d))
    plain, four = w.accum.clone(), w.accum4.clone()            # caches whose header says nothing
    for fill in (0, 255):
        plain[:256], four[:256] = fill, fill
        lte.lte_attn_decode_accum(s, plain, *w.token())
        lte.lte_attn_decode4_accum(s, four, *w.token())
        lte.lte_attn_decode4(s, c, four, *w.token())
        lte.lte_cache4_unpack(s, four)
    assert lte.lte_device_status() == 0
    assert ref.Layout(s, True).part(four, "count", torch.int32)[:, 0].eq(w.T + 6).all()
