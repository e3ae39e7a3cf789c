"""lte_attn_decode4 refuses a scorer of fewer heads or channels, whose weights it would read past their end."""
import pytest
import torch

from paper_2510_20787_b200 import lte
from tests.test_gpu_decode_accum import Run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scorer_of_fewer_heads_or_channels(dtype):
    r = Run("four learned", dtype, 1, 3, 1, 64, 40, 30, 300, 30)
    t = r.tokens()
    keep = r.cache.clone()
    for w, bias in ((r.w[:2].contiguous(), r.bias), (r.w[..., :64].contiguous(), r.bias), (r.w, r.bias[:2].contiguous()), (r.w[:1].contiguous(), None)):
        with pytest.raises(ValueError, match="scorer"):
            lte.lte_attn_decode4(r.s, lte.conv(w, bias), r.cache, *t)
    torch.cuda.synchronize()
    assert torch.equal(r.cache, keep)
    by_hand = lte.LteConv(1, r.K, 1, r.w.data_ptr(), r.bias.data_ptr())     # the struct without its tensors
    o, lse = lte.lte_attn_decode4(r.s, by_hand, r.cache.clone(), *t)
    more = lte.conv(torch.cat([r.w, r.w]), torch.cat([r.bias, r.bias]))     # of which the first heads count
    o3, l3 = lte.lte_attn_decode4(r.s, more, r.cache.clone(), *t)
    o2, l2 = lte.lte_attn_decode4(r.s, r.conv, r.cache, *t)
    assert torch.equal(o3, o2) and torch.equal(l3, l2)
    assert torch.equal(o, o2) and torch.equal(lse, l2)
    with pytest.raises(lte.LteError):
        lte.lte_attn_decode4(r.s, lte.conv(r.w[:, :6].contiguous(), r.bias), r.cache, *t)   # an even number of taps
