"""What paged_chunk_attn keeps of its weights, products and sums: 32 bits, whatever the type
of the cache and however the work is divided, and one rounding of the result."""
import numpy as np
import pytest
import torch

from paper_2106_04718_amd import api

from _gpu import device, say

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def bf16(x):
    """Rounded to bf16, as float64."""
    return torch.from_numpy(np.asarray(x)).to(BF16).double().numpy()


@pytest.mark.parametrize("D", [16, 32, 64, 128])
@pytest.mark.parametrize("R,T,behind", [(4, 1, 0), (3, 40, 0), (2, 150, 20), (1, 5, 9000), (1, 90, 6000)])
def test_weights_keep_their_bits_where_values_cancel(D, R, T, behind):
    """The first three positions, two of weight 1 and one of weight w = exp(-s), have values such that
    a + b cancels w c but for some 2^-17 of it: what is left shows the bits of w behind its
    sixteenth.  The `behind` ones behind them and the tokens' own have values of 0 and a weight of 0."""
    Hkv, G, page = 4, 2, 16
    rng = np.random.default_rng(D + T)
    L = 3 + behind + T - 1
    cols = -(-L // page)
    s = bf16(rng.uniform(0.3, 1.0, (R, Hkv)))
    w = np.exp(-s)[..., None]
    c = bf16(rng.uniform(1, 2, (R, Hkv, D)))
    a = bf16(-w * c)
    b = bf16(-w * c - a)
    q, K, V = np.zeros((R, T, Hkv, G, D)), np.zeros((R, cols, Hkv, page, D)), np.zeros((R, cols, Hkv, page, D))
    q[..., 0], q[..., 1] = s[:, None, :, None], 1.0
    K[..., 1] = -30000.0                               # scores of -30000, whose exponential is 0
    K[:, 0, :, :3, 1], K[:, 0, :, 1, 0] = 0.0, -1.0    # scores 0, -s, 0: exact
    V[:, 0, :, 0], V[:, 0, :, 1], V[:, 0, :, 2] = a, c, b
    dev = device()
    t = lambda x: torch.from_numpy(x).float().to(BF16).to(dev)
    i = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)
    say(f"[chunk bits] D={D} R={R} T={T} behind={behind}")
    out = api.paged_chunk_attn(t(q).view(R * T, Hkv * G, D), t(K).view(R * cols, Hkv, page, D), t(V).view(R * cols, Hkv, page, D),
                               i(np.arange(R * cols).reshape(R, cols)), i([L] * R), i(np.arange(R + 1) * T), scale=1.0)
    got = out.double().cpu().numpy().reshape(R, T, Hkv, G, D)
    want = ((a + b + w * c) / (2 + w))[:, None, :, None]
    terms = ((np.abs(a) + np.abs(b) + w * c) / (2 + w))[:, None, :, None]
    # In steps of 2^-24 of the terms: 2 for the score in base 2 (the factor's and the product's
    # rounding, of at most 1.45, times ln 2), 2 for exp2 (a step of fp32), 16 for the sums (five products
    # that are not 0, each addition cut off or rounded; those of nothing add nothing).  Weights of 17
    # bits are off by up to 64 of w c, half of the terms.
    tol = 2.0 ** -8 * np.abs(want) + 20 * 2.0 ** -24 * terms
    assert (np.abs(got - want) <= tol).all(), np.max((np.abs(got - want) - 2.0 ** -8 * np.abs(want)) / (2.0 ** -24 * terms))
