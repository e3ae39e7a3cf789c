"""GPU parity of the decode step under eviction by accumulated attention (lte_attn_decode_accum), and of both rules over caches in 4 bits
(lte_attn_decode4, lte_attn_decode4_accum): every step against the same step in 64 bits from the same bytes."""
import numpy as np
import pytest
import torch

from paper_2510_20787_b200 import lte
from tests import rows_ref as ref

pytestmark = pytest.mark.gpu

TYPES = {"bf16": (torch.bfloat16, lte.BF16), "f32": (torch.float32, lte.F32)}


class Run:
    """A cache in a given state, and steps on it."""

    def __init__(self, kind, dtype, B, H, G, d, W, R, n, cnt, sink=0, K=7, seed=0, scale=0.0, spread=1.5):
        self.kind, self.dt = kind, TYPES[dtype][0]
        self.s = s = lte.shape(B, H, 0, d, W, R, TYPES[dtype][1], sink=sink, group=G, softmax_scale=scale)
        self.g = g = torch.Generator(device="cuda").manual_seed(1000 * W + 10 * R + seed)
        self.K = K
        heads, rows = B * H, W + R
        self.plain = ref.Layout(s, False)
        self.cache = self.empty(s)
        learned = kind == "four learned"
        blocks = self.cache[256:].view(heads, -1)
        used = torch.cat([torch.arange(W, device="cuda") < n, torch.arange(R, device="cuda") < cnt])
        def put(name, x):
            a, b = self.plain.at[name]
            blocks[:, a:b] = x.contiguous().view(torch.uint8).view(heads, -1)
        alloc = (self.plain.at["k"][1] - self.plain.at["k"][0]) // (d * self.plain.esz)
        for name in ("k", "v"):
            x = torch.zeros((heads, alloc, d), dtype=self.dt, device="cuda")
            x[:, :rows] = torch.where(used[:, None], self.normal(heads, rows, d), 0)
            if self.plain.swizzled:
                y = torch.empty_like(x).view(heads, alloc, 8, 8)
                for r in range(8):
                    for c in range(8):
                        y[:, r::8, c ^ r] = x.view(heads, alloc, 8, 8)[:, r::8, c]
                x = y
            put(name, x)
        sc = torch.randn((heads, rows), generator=g, device="cuda") * spread
        sc = torch.where(used, sc if learned else sc.exp(), -float("inf"))
        if learned:
            for t in range(max(0, n - K // 2), n):
                sc[:, t % W] = -float("inf")
        put("score", sc)
        each = max(1, max(0, n - W) // max(1, cnt))
        pos = torch.arange(R, device="cuda") * each + (torch.rand((heads, R), generator=g, device="cuda") * each).long()
        pos[:, :sink] = torch.arange(min(sink, R), device="cuda")
        put("pos", torch.where(torch.arange(R, device="cuda") < cnt, pos, 0).int())
        put("count", torch.tensor([n, cnt, 0, 0], dtype=torch.int32, device="cuda").expand(heads, 4))
        self.lay = self.plain
        if kind != "accum":
            self.cache, self.lay = lte.lte_cache4_pack(s, self.cache), ref.Layout(s, True)
        self.w = torch.randn((H, K, 2 * d), generator=g, device="cuda") * 0.05 if learned else None
        self.bias = torch.randn((H,), generator=g, device="cuda") * 0.1 if learned else None
        self.conv = lte.conv(self.w, self.bias) if learned else None

    @staticmethod
    def empty(s):
        return torch.zeros(lte.lte_cache_bytes(s), dtype=torch.uint8, device="cuda")

    def normal(self, *size, scale=1.0):
        return (torch.randn(size, generator=self.g, device="cuda") * scale).to(self.dt)

    def tokens(self, q_scale=1.5):
        s, G = self.s, max(1, self.s.group)
        return self.normal(s.B, s.H * G, s.d, scale=q_scale), self.normal(s.B, s.H, s.d), self.normal(s.B, s.H, s.d)

    def call(self, q, k, v, decay=1.0, **kw):
        if self.kind == "accum":
            return lte.lte_attn_decode_accum(self.s, self.cache, q, k, v, decay=decay, **kw)
        if self.kind == "four accum":
            return lte.lte_attn_decode4_accum(self.s, self.cache, q, k, v, decay=decay, **kw)
        return lte.lte_attn_decode4(self.s, self.conv, self.cache, q, k, v, **kw)

    def step(self, decay=1.0, tokens=None, which=None):
        q, k, v = tokens or self.tokens()
        f = lambda t: None if t is None else t.double().cpu().numpy()  # noqa: E731
        return ref.check_step(self.s, self.lay, self.cache, q, k, v, lambda: self.call(q, k, v, decay), self.kind != "four learned", decay, f(self.w), f(self.bias), which)


KINDS = ["accum", "four accum", "four learned"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype,B,H,G,d,W,R,n,cnt,sink,K", [
    ("f32", 1, 2, 1, 32, 16, 8, 0, 0, 0, 5),           # from the empty cache on
    ("f32", 2, 2, 3, 64, 20, 12, 25, 5, 2, 7),         # the pool fills up
    ("f32", 1, 3, 5, 128, 37, 19, 300, 19, 1, 13),     # two passes of query heads, the pool is full
    ("f32", 1, 1, 2, 64, 700, 333, 5000, 333, 0, 7),   # rows shared by a cluster
    ("bf16", 1, 2, 1, 32, 13, 6, 0, 0, 0, 13),
    ("bf16", 2, 2, 1, 64, 100, 99, 120, 20, 1, 5),     # swizzled rows
    ("bf16", 2, 3, 8, 64, 128, 128, 900, 128, 0, 7),   # swizzled, a full pass of query heads
    ("bf16", 3, 5, 3, 128, 301, 77, 1000, 77, 1, 3),
    ("bf16", 1, 2, 9, 128, 250, 70, 400, 70, 3, 7),    # two passes of query heads
    ("bf16", 1, 2, 12, 32, 64, 300, 364, 300, 0, 7),
    ("bf16", 1, 2, 4, 64, 768, 512, 1500, 512, 4, 7),  # a cluster
    ("bf16", 40, 16, 1, 64, 33, 31, 70, 31, 0, 7),     # many heads
    ("bf16", 1, 2, 2, 128, 13, 1, 40, 1, 0, 7),        # one entry
    ("bf16", 2, 2, 1, 64, 257, 0, 255, 0, 0, 7),       # no pool, the ring fills up
    ("bf16", 1, 1, 1, 128, 1000, 2000, 9000, 2000, 0, 7),
])
def test_steps(kind, dtype, B, H, G, d, W, R, n, cnt, sink, K):
    r = Run(kind, dtype, B, H, G, d, W, R, n, cnt, sink, K)
    for i in range(6):
        r.step(decay=(1.0, 0.9, 0.0)[i % 3])
    assert lte.lte_device_status() == 0


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("B,H,G,d,W,R,n,cnt", [
    (1, 8, 3, 128, 700, 1300, 4000, 1300),             # (on 148 SMs: clusters of 10; their shares of the outputs are of unequal sizes
    (1, 12, 1, 64, 512, 700, 3000, 690),               # of 9
    (2, 8, 5, 128, 300, 600, 900, 600),                # of 6
    (2, 13, 7, 128, 100, 500, 700, 500),               # of 5
    (4, 9, 9, 128, 130, 300, 700, 300),                # of 3, two passes of query heads
    (4, 10, 3, 64, 100, 250, 99, 0),                   # of 3, the ring not full
    (11, 6, 17, 64, 128, 128, 500, 128),               # of 2, swizzled rows, three passes of query heads
    (37, 4, 2, 128, 100, 29, 1000, 29),                # one block a head
    (37, 4, 1, 64, 100, 70, 3, 0),                     # the same, hardly a row
    (1, 4, 8, 128, 2048, 4000, 30000, 4000),           # of 16
])
def test_blocks_of_eight_warps_one_an_sm(kind, B, H, G, d, W, R, n, cnt):
    r = Run(kind, "bf16", B, H, G, d, W, R, n, cnt, sink=1)
    for decay in (0.9, 1.0, 0.0):
        r.step(decay=decay, which=[0, 1, H - 1, B * H // 2, B * H - 1])
    assert lte.lte_device_status() == 0


@pytest.mark.parametrize("B,H,G,d,W,R,n,cnt", [
    (1, 8, 8, 128, 1000, 28000, 90000, 28000),         # logits do not fit beside the stages of eight warps: the keys once more
    (1, 5, 11, 128, 2000, 30768, 90000, 30768),
])
def test_scores_of_long_4_bit_rows(B, H, G, d, W, R, n, cnt):
    r = Run("four accum", "bf16", B, H, G, d, W, R, n, cnt, sink=1)
    for decay in (0.9, 0.0):
        r.step(decay=decay, which=[0, H - 1])


@pytest.mark.parametrize("kind", ["accum", "four accum"])
@pytest.mark.parametrize("B,H,G,d,W,R,n,cnt", [
    (80, 16, 17, 32, 150, 150, 900, 150),              # a warp a head, three passes of query heads
    (100, 16, 9, 64, 100, 156, 700, 156),              # the same, swizzled rows
    (100, 16, 8, 64, 120, 137, 1000, 90),              # the pool not full
    (32, 16, 12, 64, 900, 1100, 890, 0),               # several warps a head, the ring not full
    (32, 16, 12, 64, 600, 1400, 5000, 1400),
    (20, 15, 17, 128, 500, 1000, 9000, 1000),
    (2, 37, 9, 32, 1000, 5000, 30000, 5000),           # a cluster a head
])
def test_scores_of_heads_whose_logits_do_not_fit(kind, B, H, G, d, W, R, n, cnt):
    """So many rows, query heads and heads at once that the logits of an SM's heads do not fit its shared memory: the weights come from the
    keys, read once more."""
    r = Run(kind, "bf16", B, H, G, d, W, R, n, cnt, sink=1)
    for decay in (0.9, 0.0):
        r.step(decay=decay, which=[0, 1, H - 1, B * H // 2, B * H - 1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["accum", "four accum"])
def test_smallest_window(kind, dtype):
    r = Run(kind, dtype, 1, 2, 1, 64, 1, 3, 0, 0)
    for _ in range(8):
        r.step()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", KINDS)
def test_most_rows(kind, dtype):
    r = Run(kind, dtype, 1, 1, 5, 64, 2768, 30000, 100000, 30000)
    r.step()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["accum", "four accum"])
def test_equal_scores_let_the_youngest_go(kind, dtype):
    r = Run(kind, dtype, 1, 2, 1, 64, 16, 12, 100, 12, spread=0.0)     # every score is 1
    blocks = r.cache[256:].view(2, -1)
    a, b = r.lay.at["score"]
    blocks[:, a:b].view(torch.float32)[:, :16] = 1.5                   # the tokens in the window have more
    pos = r.lay.part(r.cache, "pos", torch.int32).cpu().numpy()
    r.step(decay=0.0)
    after = r.lay.part(r.cache, "pos", torch.int32).cpu().numpy()
    for h in range(2):
        assert set(pos[h]) - set(after[h]) == {pos[h].max()} and 84 in after[h]
    r = Run(kind, dtype, 1, 2, 1, 64, 16, 12, 100, 12, spread=0.0)     # a token with no more than the lowest stays out
    pos = r.lay.part(r.cache, "pos", torch.int32).cpu()
    r.step()
    assert torch.equal(r.lay.part(r.cache, "pos", torch.int32).cpu(), pos)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", KINDS)
def test_a_pool_of_sink_tokens_takes_nothing_else(kind, dtype):
    r = Run(kind, dtype, 1, 2, 1, 64, 20, 4, 50, 4, sink=4)
    for _ in range(3):
        r.step()
    assert torch.equal(r.lay.part(r.cache, "pos", torch.int32).cpu(), torch.arange(4, dtype=torch.int32).expand(2, 4))


@pytest.mark.parametrize("dtype,d,W,R,n,cnt", [("bf16", 64, 48, 40, 30, 0), ("bf16", 128, 50, 300, 100, 21), ("f32", 32, 30, 20, 44, 9), ("bf16", 32, 33, 90, 60, 20)])
@pytest.mark.parametrize("kind", KINDS)
def test_rows_that_hold_nothing_are_not_read(kind, dtype, d, W, R, n, cnt):
    """NaN in every row that is not in use, scores and positions included: o, lse and the state come out the same."""
    a, b = Run(kind, dtype, 2, 2, 2, d, W, R, n, cnt), Run(kind, dtype, 2, 2, 2, d, W, R, n, cnt)
    blocks, lay, rows = b.cache[256:].view(4, -1), b.lay, W + R
    free = torch.cat([torch.arange(W) >= n, torch.arange(R) >= cnt]).cuda()
    for name in [x for x in ("k", "v", "kpar", "vpar", "score") if x in lay.at]:
        i, j = lay.at[name]
        alloc = 256 if lay.swizzled and name in "kv" else rows
        part = blocks[:, i:j].view(4, alloc, -1)
        part[:, :rows][:, free] = 255                          # (all bits set: NaN in bf16 and fp32)
        part[:, rows:] = 255
    for _ in range(3):
        t = a.tokens()
        (o1, l1), (o2, l2) = a.call(*t), b.call(*t)
        assert torch.equal(o1, o2) and torch.equal(l1, l2)
    sa, sb = a.lay.state(a.cache), b.lay.state(b.cache)
    for h in range(4):
        used = np.concatenate([np.arange(W) < n + 3, np.arange(R) < sa["count"][h, 1]])
        for name in ("k", "v", "score"):
            assert np.array_equal(sa[name][h][used], sb[name][h][used], equal_nan=True)
    assert np.array_equal(sa["count"], sb["count"])


@pytest.mark.parametrize("dtype,d,W,R,G", [("bf16", 64, 48, 40, 1), ("bf16", 64, 300, 40, 4), ("bf16", 128, 50, 300, 2), ("f32", 32, 30, 20, 1), ("bf16", 32, 33, 90, 3)])
@pytest.mark.parametrize("kind", ["accum", "four accum"])
def test_infinite_values_go_with_their_row(kind, dtype, d, W, R, G):
    """An infinite value in the row that leaves, and in the entry that is replaced: the step in which they go does not see them."""
    for leaves in (True, False):
        r = Run(kind, dtype, 1, 2, G, d, W, R, W + 3 * R, R)
        blocks, lay, n = r.cache[256:].view(2, -1), r.lay, W + 3 * R
        score = blocks[:, lay.at["score"][0]:lay.at["score"][1]].view(torch.float32)
        score[:, n % W] = 1e-9 if leaves else 1e9              # stays out, or replaces the lowest entry
        score[:, W + 7] = 1e-6
        row = n % W if leaves else W + 7
        part, width = ("vpar", 4 * d // 32) if lay.four else ("v", d * lay.esz)
        v = blocks[:, lay.at[part][0]:lay.at[part][1]].view(2, -1, width)[:, row]
        v.view(torch.bfloat16 if lay.four or lay.esz == 2 else torch.float32)[:] = float("inf")
        q, k1, v1 = r.tokens()
        o, lse = r.call(q, k1, v1)
        assert bool(torch.isfinite(o).all()) and bool(torch.isfinite(lse).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size", [30.0, 1e6, 1e18])
def test_large_logits(kind, dtype, size):
    r = Run(kind, dtype, 1, 2, 3, 64, 70, 60, 400, 60)
    q, k, v = r.tokens(q_scale=size)
    r.step(tokens=(q, k, v), decay=0.5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", KINDS)
def test_a_captured_step_replays(kind, dtype):
    """Steps in a CUDA graph leave what the same steps leave when called, on a stream other than the tensors' own."""
    a, b = (Run(kind, dtype, 2, 4, 2, 64, 60, 50, 500, 50) for _ in range(2))
    tokens = [a.tokens() for _ in range(6)]
    q, k, v = (t.clone() for t in tokens[0])
    o, lse = torch.empty_like(q), torch.empty(q.shape[:2], dtype=torch.float32, device="cuda")
    keep = b.cache.clone()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        b.call(q, k, v, 0.9, o1=o, lse1=lse)
        b.cache.copy_(keep)
        st.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            b.call(q, k, v, 0.9, o1=o, lse1=lse)
    torch.cuda.synchronize()
    for t in tokens:
        for to, x in zip((q, k, v), t):
            to.copy_(x)
        g.replay()
        o2, l2 = a.call(*t, 0.9)
        torch.cuda.synchronize()
        assert torch.equal(o, o2) and torch.equal(lse, l2)
    assert torch.equal(a.cache, b.cache)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", KINDS)
def test_two_streams_at_once(kind, dtype):
    runs = [Run(kind, dtype, 4, 4, 2, 64, 100, 200, 700, 200, seed=i) for i in range(2)]
    want = [Run(kind, dtype, 4, 4, 2, 64, 100, 200, 700, 200, seed=i) for i in range(2)]
    tokens = [[r.tokens() for _ in range(20)] for r in runs]
    streams = [torch.cuda.Stream() for _ in runs]
    torch.cuda.synchronize()
    for i in range(20):
        for r, st, t in zip(runs, streams, tokens):
            with torch.cuda.stream(st):
                r.call(*t[i])
    torch.cuda.synchronize()
    for r, w, t in zip(runs, want, tokens):
        for x in t:
            w.call(*x)
        torch.cuda.synchronize()
        assert torch.equal(r.cache, w.cache)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 32)])
def test_scorer_weights_off_a_16_byte_boundary(dtype, d):
    a, b = (Run("four learned", dtype, 2, 3, 2, d, 40, 30, 300, 30, K=9) for _ in range(2))
    b.conv = lte.conv(torch.cat([b.w.new_zeros(1), b.w.flatten()])[1:].view(b.w.shape), b.bias)
    for _ in range(3):
        t = a.tokens()
        for x, y in zip(a.call(*t), b.call(*t)):
            assert torch.equal(x, y)
    assert torch.equal(a.cache, b.cache)


def test_caches_past_4_gigabytes():
    """The last heads of a cache whose offsets pass 32 bits."""
    B, H, d, W, R = 9, 32, 128, 2768, 30000
    s = lte.shape(B, H, 0, d, W, R, lte.BF16)
    cache = torch.zeros(lte.lte_cache_bytes(s), dtype=torch.uint8, device="cuda")
    assert cache.numel() > 2 ** 32
    small = Run("accum", "bf16", 1, 2, 1, d, W, R, 90000, R)
    block = small.lay.stride
    cache[-2 * block:] = small.cache[256:]
    q, k, v = small.tokens()
    big = [torch.zeros((B, H, d), dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    for x, y in zip(big, (q, k, v)):
        x[-1, -2:] = y
    o, lse = lte.lte_attn_decode_accum(s, cache, *big)
    o2, l2 = small.call(q, k, v)
    near = lambda a, b, e: bool(((a.double() - b.double()).abs() <= e * b.double().abs().max()).all())  # noqa: E731
    assert near(o[-1, -2:], o2[0], 2.0 ** -7) and near(lse[-1, -2:], l2[0], 1e-6)
    a, b = small.lay.at["score"]
    got, want = (x[-2 * block:].view(2, block)[:, a:b].view(torch.float32) for x in (cache, small.cache))
    assert near(got, want, 1e-6)
    assert torch.equal(cache[-2 * block:].view(2, block)[:, b:], small.cache[-2 * block:].view(2, block)[:, b:])


def test_the_prompt_s_sums_go_on():
    """Prompt, its accumulated attention, decode steps: with room for every token the scores are the accumulated attention of the whole
    sequence, in fp32."""
    B, H, G, d, W, T, N = 1, 2, 3, 64, 12, 60, 15
    R = T + N
    g = torch.Generator(device="cuda").manual_seed(5)
    n = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    q, k, v = n(B, H * G, T + N, d), n(B, H, T + N, d), n(B, H, T + N, d)

    def prompt(t):
        s = lte.shape(B, H, t, d, W, R, lte.F32, group=G)
        qp, kp, vp = (x[:, :, :t].contiguous() for x in (q, k, v))
        idx, cnt = lte.lte_select_rule(s, lte.RULE_ACCUM_ATTN, torch.ones((B, H, t), device="cuda"))   # every token out of the window
        o, lse = lte.lte_attn_prefill(s, qp, kp, vp, idx, cnt)
        return s, kp, vp, o, lse, idx, cnt, lte.lte_attn_colsum(s, qp, kp, lse, idx, cnt)
    s, kp, vp, _, _, idx, cnt, a = prompt(T)
    cache = lte.lte_cache_init_accum(s, kp, vp, a, idx, cnt)
    steps = [lte.lte_attn_decode_accum(s, cache, q[:, :, t].contiguous(), k[:, :, t].contiguous(), v[:, :, t].contiguous()) for t in range(T, T + N)]
    _, _, _, o, lse, _, _, a2 = prompt(T + N)
    st = ref.Layout(s, False).state(cache)
    for h in range(H):
        total = np.empty(T + N)
        total[st["pos"][h, :T + N - W]] = st["score"][h, W:T + N]
        for t in range(T + N - W, T + N):
            total[t] = st["score"][h, t % W]
        np.testing.assert_allclose(total, a2[0, h].double().cpu().numpy(), rtol=2e-5)   # sums of up to 225 weights, each within 1e-6 and 2^-24 a sum
    for i, (o1, l1) in enumerate(steps):
        torch.testing.assert_close(o1, o[:, :, T + i], rtol=1e-5, atol=1e-5)
        torch.testing.assert_close(l1, lse[:, :, T + i], rtol=1e-6, atol=1e-5)


def test_empty_prompt():
    s = lte.shape(1, 2, 0, 64, 8, 4, lte.BF16)
    cache = lte.lte_cache_init_accum(s)
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn((1, 2, 64), generator=g, device="cuda").to(torch.bfloat16) for _ in range(3))
    for c, call in ((cache.clone(), lte.lte_attn_decode_accum), (lte.lte_cache4_pack(s, cache), lte.lte_attn_decode4_accum)):
        o, lse = call(s, c, q, k, v)
        assert torch.equal(o, v)                               # one row, as given: its weight is 1
        torch.testing.assert_close(lse, (q.float() * k.float()).sum(-1) / 8, rtol=1e-5, atol=1e-5)


def test_binding_refuses_what_it_would_read_past():
    r = Run("accum", "bf16", 1, 2, 2, 64, 16, 8, 60, 8)
    q, k, v = r.tokens()
    for bad in ((q[:, :2], k, v), (q, k[:, :1], v), (q, k, v[..., :32]), (q, torch.cat([k, k]), v)):
        with pytest.raises((ValueError, AssertionError)):
            r.call(*bad)
    for bad in ((q.float(), k, v), (q, k.float(), v), (q.cpu(), k, v), (q, k.transpose(1, 2), v)):
        with pytest.raises((ValueError, AssertionError)):
            r.call(*bad)
    with pytest.raises(ValueError):
        lte.lte_attn_decode_accum(r.s, r.cache[:-256].clone(), q, k, v)
    with pytest.raises(AssertionError):
        r.call(q, k, v, o1=torch.empty_like(q).float())
    with pytest.raises(lte.LteError):
        r.call(q, k, v, decay=1.5)
    with pytest.raises(lte.LteError):
        r.call(q, k, v, decay=float("nan"))
    with pytest.raises(TypeError):
        lte.lte_attn_decode4(r.s, None, r.cache, q, k, v)
