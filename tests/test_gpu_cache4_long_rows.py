"""Decode over 4-bit caches with many rows to a warp and attention spread over all of them: what is left of o after zero and code times step have
cancelled is small against either, and a sum that is rounded one way loses it."""
import numpy as np
import pytest
import torch

from paper_2510_20787_b200 import lte
from tests import rows_ref as ref
from tests.test_gpu_cache4_ranges import edited, key_with
from tests.test_gpu_decode_accum import Run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["four accum", "four learned"])
@pytest.mark.parametrize("H,G,d,W,R", [(2500, 1, 32, 768, 9000), (640, 2, 32, 768, 32000), (1300, 1, 64, 768, 15000), (600, 3, 64, 768, 8000), (400, 1, 128, 768, 32000),
                                       (2400, 1, 64, 300, 2000), (600, 9, 64, 100, 6000)])
def test_flat_attention_over_many_rows(kind, H, G, d, W, R):
    r = Run(kind, "bf16", 1, H, G, d, W, R, W + 3 * R, R)
    q, k, v = r.tokens(q_scale=0.05)
    which = [0, H // 2, H - 1]
    heads = torch.tensor(which, device="cuda")
    f = lambda t: None if t is None else t.double().cpu().numpy()  # noqa: E731
    state = ref.magnitudes(r.lay, r.cache, r.lay.state(r.cache, heads), heads)
    of = lambda t, e: t.reshape(H, -1, e)[heads]  # noqa: E731
    _, o64, _, bound = ref.step(r.s, r.lay, state, of(q, d), of(k, d), of(v, d), kind == "four accum", 1.0, f(r.w), f(r.bias), which)
    o, _ = r.call(q, k, v)
    off = np.abs(f(o.reshape(H, -1, d)[heads]).reshape(o64.shape) - o64)
    # Steps of 32 normal values lie around 4.1 / 15, codes around 7.5: with N weights near 1 / N the sum of w code step is near 2.05 (here at most 2.6).
    #   products with steps, each off by 2^-12 of it at most and one way as well as the other: 6 standard deviations of their sum, 6 2^-12 / sqrt(3) / sqrt(N) 2.6
    #   running sums, rounded towards zero by 2^-23 of them at most in each of the up to 32 (512 rows) + N / 512 products and sums in a row
    #   o rounded to bf16: half a step, 2^-9 of it, and as much for its being off already
    N = W + R
    most = 6 * 2.0 ** -12 / 3 ** 0.5 / N ** 0.5 * 2.6 + 2.0 ** -23 * 2.6 * (32 + N / 512) + 2.0 ** -8 * np.abs(o64)
    assert (off <= np.minimum(most, bound["o"])).all(), (float((off - most).max()), float(off.max()), float(np.abs(o64).mean()))


@pytest.mark.parametrize("kind", ["four accum", "four learned"])
@pytest.mark.parametrize("up", [True, False])
@pytest.mark.parametrize("H,G,d,W,R", [(2500, 1, 32, 100, 2500), (700, 2, 64, 700, 6000), (300, 3, 128, 500, 9000)])
def test_long_rows_whose_weights_and_values_run_against_each_other(H, G, d, W, R, up, kind):
    """Logits that rise by 90 in all while values fall by 2^100, and the other way round: references and scales move while there are second sums."""
    def edit(k, v, q):
        x = torch.linspace(-1, 1, W + R, device="cuda") * (1 if up else -1)
        v *= torch.exp2(-50 * x).to(v.dtype)[:, None]
        one = key_with(q, 45.0).float()
        k.copy_(0.2 * k.float() + x[:, None] * one[:, None])
    r, tokens = edited(kind, "bf16", 1, H, G, d, W, R, edit)
    r.step(tokens=tokens, decay=0.9, which=[0, H // 2, H - 1])
