"""Rotary positions of more tokens than a dimension of a launch holds: 2^24 workgroups of 256
lanes, four tokens each."""
import pytest
import torch

from paper_2106_04718_amd import api

from _gpu import device, say

pytestmark = pytest.mark.gpu


def test_more_tokens_than_one_dimension_holds():
    dev, N, D = device(), (1 << 26) + 5, 16
    say(f"[rotary grid] {N} tokens")
    x = torch.randint(-1000, 1000, (N, 1, D), dtype=torch.int16, device=dev).to(torch.bfloat16)
    pos = torch.arange(N, device=dev).int() % 4
    freq = torch.full((D // 2,), torch.pi / 2, dtype=torch.float64, device=dev)   # quarter turns
    out = api.rotary(x, pos, freq)
    torch.cuda.synchronize()
    half = D // 2
    for p in range(4):
        a, b = x[p::4, :, :half], x[p::4, :, half:]
        want = ((a, b), (-b, a), (-a, -b), (b, -a))[p]
        got = out[p::4]
        # exact, but for 1000 times a cosine of 0 to some steps of fp64 where the other element is 0
        for g, w in ((got[..., :half], want[0]), (got[..., half:], want[1])):
            assert float((g.float() - w.float()).abs().max()) <= 1000 * 2.0 ** -48, p
