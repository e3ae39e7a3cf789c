"""Decode steps over caches in 4 bits whose rows, groups of channels and queries differ widely in size: every step against the same step in
64 bits, within the bounds of the ordinary cases (an error of o of 2^-12 of the sum of weight times code times step, in the group of the channel)."""
import pytest
import torch

from paper_2510_20787_b200 import lte
from tests.test_gpu_decode_accum import Run

pytestmark = pytest.mark.gpu

# (B, H, d, W, R): a warp a head, several warps, clusters; none of the layouts is swizzled
SHAPES = [(60, 40, 32, 20, 44), (1, 2, 32, 40, 60), (1, 3, 64, 150, 250), (30, 40, 64, 200, 100), (1, 2, 128, 60, 100), (1, 8, 128, 700, 1000)]


def edited(kind, dtype, B, H, G, d, W, R, edit):
    """A run on a full cache whose keys and values [heads, W + R, d] `edit` has changed, and its next tokens: the query heads 0, 2, .. of a group are
    about the same, 1, 3, .. their opposite."""
    r = Run(kind, dtype, B, H, G, d, W, R, W + 3 * R, R)
    q, k1, v1 = r.tokens()
    q = q.view(B, H, G, d)
    sign = torch.tensor([1.0, -1.0] * G, device="cuda")[:G, None]
    q = ((q[:, :, :1] + 0.1 * q) * sign).to(q.dtype).view(B, H * G, d)
    plain = lte.lte_cache4_unpack(r.s, r.cache)
    part = lambda name: plain[256:].view(B * H, -1)[:, r.plain.at[name][0]:r.plain.at[name][1]].view(r.dt).view(B * H, W + R, d)  # noqa: E731
    edit(part("k"), part("v"), q.view(B * H, G, d)[:, 0])
    r.cache = lte.lte_cache4_pack(r.s, plain)
    return r, (q, k1, v1)


def key_with(q, logit):
    """A key whose scaled product with q is `logit`."""
    x = q.double()
    return (x * (logit * x.shape[-1] ** 0.5 / (x * x).sum(-1, keepdim=True))).to(q.dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["four accum", "four learned"])
@pytest.mark.parametrize("power", [10, 20, 26, 30, 45, 100])
@pytest.mark.parametrize("shape", SHAPES)
def test_a_row_of_large_values_that_weighs_nothing(shape, power, kind, dtype):
    """One row in four places of the head, values 2^power times the others': with weights of e^-50 for some query heads and, being their opposite's,
    nearly all the weight for others."""
    B, H, d, W, R = shape
    which = [0, 1, B * H - 1]
    for row in (0, 9, W, W + R - 1):                           # (n = W + 3 R: the row that leaves is another one)
        for G in (1, 3):
            def edit(k, v, q):
                v[:, row] *= 2.0 ** power
                k[:, row] = key_with(q, -50.0)
            r, tokens = edited(kind, dtype, B, H, G, d, W, R, edit)
            r.step(tokens=tokens, decay=0.9, which=which)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["four accum", "four learned"])
@pytest.mark.parametrize("power", [10, 20, 30, 60])
@pytest.mark.parametrize("shape", [x for x in SHAPES if x[2] > 32])
def test_groups_of_channels_of_different_size(shape, power, kind, dtype):
    """The first 32 channels of one row, or of every row, 2^power times the others: what the other channels come to does not depend on them."""
    B, H, d, W, R = shape
    which = [0, 1, B * H - 1]
    for rows in (slice(None), slice(7, 8), slice(W, None)):
        def edit(k, v, q):
            v[:, rows, :32] *= 2.0 ** power
        r, tokens = edited(kind, dtype, B, H, 2, d, W, R, edit)
        r.step(tokens=tokens, decay=0.9, which=which)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["four accum", "four learned"])
@pytest.mark.parametrize("up", [True, False])
@pytest.mark.parametrize("shape", SHAPES)
def test_weights_and_values_that_run_against_each_other(shape, up, kind, dtype):
    """Logits that rise along the rows by 90 in all while values fall by 2^100, and the other way round: the reference of the weights and the scale of the
    products move all the time, in opposite directions."""
    B, H, d, W, R = shape
    which = [0, 1, B * H - 1]

    def edit(k, v, q):
        x = torch.linspace(-1, 1, W + R, device="cuda", dtype=torch.float64) * (1 if up else -1)
        v *= torch.exp2(-50 * x).to(v.dtype)[:, None]
        k.copy_(0.2 * k + torch.stack([key_with(q, 45.0 * float(y)) for y in x], dim=1))
    r, tokens = edited(kind, dtype, B, H, 3, d, W, R, edit)
    r.step(tokens=tokens, decay=0.9, which=which)


@pytest.mark.parametrize("kind", ["four accum", "four learned"])
@pytest.mark.parametrize("size", [1e-30, 1e-20, 1e20, 1e30])
def test_values_small_and_large(size, kind):
    for shape in SHAPES:
        def edit(k, v, q):
            v *= size
        r, (q, k1, v1) = edited(kind, "bf16", *shape[:2], 2, *shape[2:], edit)
        r.step(tokens=(q, k1, (v1.double() * size).to(v1.dtype)), which=[0, 1, shape[0] * shape[1] - 1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["four accum", "four learned"])
@pytest.mark.parametrize("power", [117, 110, 60, -60, -110, -117])
def test_keys_and_queries_of_opposite_size(power, kind, dtype):
    """Keys 2^power times, queries 2^-power times their ordinary size: logits of the ordinary size."""
    for shape in SHAPES:
        for G in (1, 3):
            def edit(k, v, q):
                k *= 2.0 ** power
            r, (q, k1, v1) = edited(kind, dtype, *shape[:2], G, *shape[2:], edit)
            if r.conv is not None:                             # (a scorer whose logits of such keys are ordinary)
                r.w[..., :r.s.d] *= 2.0 ** -power
            r.step(tokens=(q * 2.0 ** -power, k1 * 2.0 ** power, v1), decay=0.9, which=[0, 1, shape[0] * shape[1] - 1])
