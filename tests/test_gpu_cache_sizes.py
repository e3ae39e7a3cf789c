"""The calls on ordinary caches refuse a cache that is shorter than the shape's, such as one in 4 bits, before anything is launched."""
import pytest
import torch

from paper_2510_20787_b200 import lte

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,torch_dtype", [(lte.BF16, torch.bfloat16), (lte.F32, torch.float32)])
def test_calls_on_ordinary_caches_refuse_short_ones(dtype, torch_dtype):
    B, H, T, d, W, R = 1, 2, 12, 64, 24, 300
    g = torch.Generator(device="cuda").manual_seed(1)
    n = lambda *size: torch.randn(size, generator=g, device="cuda")  # noqa: E731
    s = lte.shape(B, H, T, d, W, R, dtype)
    c = lte.conv(n(H, 5, 2 * d) * 0.05)
    stack = lte.conv_stack([n(H, d, 3, 2 * d), n(H, d // 2, 3, d), n(H, d // 4, 3, d // 2)], n(H, d // 4))
    k, v, z = n(B, H, T, d).to(torch_dtype), n(B, H, T, d).to(torch_dtype), n(B, H, T)
    idx, cnt = lte.lte_select(s, z)
    cache = lte.lte_cache_init(s, c, k, v, z, idx, cnt)
    four = lte.lte_cache4_pack(s, cache)
    one = lambda: n(B, H, d).to(torch_dtype)  # noqa: E731
    for short in (four, cache[:-256].clone()):
        keep = short.clone()
        for call in (lambda: lte.lte_cache_init(s, c, k, v, z, idx, cnt, cache=short), lambda: lte.lte_attn_decode(s, c, short, one(), one(), one()),
                     lambda: lte.lte_attn_prefill_chunk(s, c, short, T, k, k, v), lambda: lte.lte_cache_score(s, stack, short),
                     lambda: lte.lte_attn_decode_accum(s, short, one(), one(), one()), lambda: lte.lte_cache4_pack(s, short)):
            with pytest.raises(ValueError, match="shorter"):
                call()
        assert torch.equal(short, keep)
    lte.lte_attn_decode(s, c, torch.cat([cache, cache[:16]]), one(), one(), one())     # a longer one holds the shape's
    torch.cuda.synchronize()
    assert lte.lte_device_status() == 0


def test_no_list_is_needed_for_a_budget_of_none():
    """R = 0: lte_cache_init_accum takes no idx, as lte_cache_init does and lte.h says."""
    s = lte.shape(1, 2, 40, 64, 16, 0, lte.BF16)
    g = torch.Generator(device="cuda").manual_seed(2)
    k, v = (torch.randn((1, 2, 40, 64), generator=g, device="cuda").to(torch.bfloat16) for _ in "kv")
    a, cnt = torch.rand((1, 2, 40), generator=g, device="cuda"), torch.zeros((1, 2), dtype=torch.int32, device="cuda")
    with_list = lte.lte_cache_init_accum(s, k, v, a, torch.empty((1, 2, 0), dtype=torch.int32, device="cuda"), cnt)
    assert torch.equal(lte.lte_cache_init_accum(s, k, v, a, None, cnt), with_list)
    with pytest.raises(TypeError):
        lte.lte_cache_init_accum(lte.shape(1, 2, 40, 64, 16, 4, lte.BF16), k, v, a, None, cnt)
