"""What paged_attn keeps of its weights, products and sums: 32 bits, whatever the
type of the cache, and one rounding of the result."""
import numpy as np
import pytest
import torch

from paper_2106_04718_amd import api, workloads

from _gpu import device, say, to_f64

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def bf16(x):
    """Rounded to bf16, as float64."""
    bits = workloads.f32_to_bf16_bits(np.asarray(x, np.float32))
    return (bits.astype(np.uint32) << 16).view(np.float32).astype(np.float64)


@pytest.mark.parametrize("D", [16, 32, 64, 128])
def test_weights_keep_their_bits_where_values_cancel(D):
    """Three positions: two of weight 1, one of weight w = exp(-s), their values such
    that a + b cancels w c but for some 2^-17 of it.  What is left shows the bits of w
    behind its sixteenth."""
    R, H, page = 4, 8, 16
    rng = np.random.default_rng(D)
    s = bf16(rng.uniform(0.3, 1.0, (R, H)))
    w = np.exp(-s)[..., None]
    c = bf16(rng.uniform(1, 2, (R, H, D)))
    a = bf16(-w * c)
    b = bf16(-w * c - a)
    q, K, V = np.zeros((R, H, D)), np.zeros((R, H, page, D)), np.zeros((R, H, page, D))
    q[..., 0], K[:, :, 1, 0] = s, -1.0          # scores 0, -s, 0: exact
    V[:, :, 0], V[:, :, 1], V[:, :, 2] = a, c, b
    t = lambda x: torch.from_numpy(x).float().to(BF16).to(device())
    say(f"[paged bits] D={D}")
    out = to_f64(api.paged_attn(t(q), t(K), t(V), torch.arange(R, dtype=torch.int32, device=device())[:, None],
                                torch.full((R,), 3, dtype=torch.int32, device=device()), scale=1.0))
    want = (a + b + w * c) / (2 + w)
    terms = (np.abs(a) + np.abs(b) + w * c) / (2 + w)
    # In steps of 2^-24 of the terms: 2 for the score in base 2 (two roundings of at most
    # 1.45, times ln 2), 2 for exp2 (a step of fp32), 16 for the sums (nine products,
    # each addition cut off or rounded).  Weights of 17 bits are off by up to 64 of w c,
    # half of the terms.
    assert (np.abs(out - want) <= 2.0 ** -8 * np.abs(want) + 20 * 2.0 ** -24 * terms).all(), \
        np.max((np.abs(out - want) - 2.0 ** -8 * np.abs(want)) / (2.0 ** -24 * terms))
