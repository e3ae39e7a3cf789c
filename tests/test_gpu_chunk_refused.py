"""A chunk on a cache that does not hold n_past tokens is reported and leaves the cache alone, whatever the workspace held before: the kernels behind
the one that finds it out work on a head without a pool."""
import pytest
import torch

from paper_2510_20787_b200 import lte

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("streaming", [False, True])
@pytest.mark.parametrize("dtype,d,W,R,T,M", [("bf16", 64, 24, 30, 200, 90), ("bf16", 128, 24, 30, 200, 9), ("bf16", 32, 20, 30, 200, 9),
                                             ("f32", 64, 24, 30, 200, 90), ("bf16", 64, 24, 400, 200, 60)])
def test_wrong_token_count_over_a_used_workspace(dtype, d, W, R, T, M, streaming):
    B, H = 2, 3
    g = torch.Generator(device="cuda").manual_seed(3)
    kind, dt = (lte.BF16, torch.bfloat16) if dtype == "bf16" else (lte.F32, torch.float32)
    n = lambda *size: torch.randn(size, generator=g, device="cuda").to(dt)  # noqa: E731
    s, s2 = lte.shape(B, H, T, d, W, R, kind), lte.shape(B, H, M, d, W, R, kind)
    c = lte.conv(torch.randn((H, 5, 2 * d), generator=g, device="cuda") * 0.05)
    k, v = n(B, H, T, d), n(B, H, T, d)
    z = lte.lte_scores(s, c, k, v)
    cache = lte.lte_cache_init(s, c, k, v, z, *lte.lte_select(s, z))
    size = lte.lte_workspace_bytes(lte.OP_CHUNK_STREAM if streaming else lte.OP_CHUNK, s2, c)
    q, k2, v2 = n(B, H, M, d), n(B, H, M, d), n(B, H, M, d)
    good = cache.clone()
    want = lte.lte_attn_prefill_chunk(s2, c, good, T, q, k2, v2, streaming=streaming)
    for fill in ("random", 7, 255):
        for n_past in (T - 1, T + 1, W, 3):
            ws = torch.randint(0, 256, (size,), generator=g, device="cuda", dtype=torch.uint8) if fill == "random" else torch.full((size,), fill, dtype=torch.uint8, device="cuda")
            keep = cache.clone()
            lte.lte_attn_prefill_chunk(s2, c, cache, n_past, q, k2, v2, ws=ws, streaming=streaming)
            assert lte.lte_device_status() == -6
            assert torch.equal(cache, keep)
            got = lte.lte_attn_prefill_chunk(s2, c, keep, T, q, k2, v2, ws=ws, streaming=streaming)   # the right count, over what the call left behind
            assert torch.equal(keep, good) and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
            assert lte.lte_device_status() == 0
