"""Paged calls of more workgroups than a dimension of a launch holds: 2^24 of 256
lanes.  The runtime refuses no more than that: it launches what 32 bits leave of
the number, so a call that counts on one dimension does nearly nothing and says
that it did."""
import pytest
import torch

from paper_2106_04718_amd import api

from _gpu import device, say

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def noise(*shape):
    """Finite bf16 values, made on the device."""
    return torch.randint(-1000, 1000, shape, dtype=torch.int16, device=device()).to(BF16)


@pytest.mark.parametrize("offsets", [True, False])
def test_append_of_more_tokens_than_one_dimension_holds(offsets):
    N, D, page = (1 << 26) + 5, 16, 1024   # four tokens a workgroup
    say(f"[paged grid] append of {N} tokens")
    dev = device()
    P = -(-N // page)
    k, v = noise(N, 1, D), noise(N, 1, D)
    K, V = torch.zeros(P, 1, page, D, dtype=BF16, device=dev), torch.zeros(P, 1, page, D, dtype=BF16, device=dev)
    if offsets:   # two rows, the second behind the first's pages
        first = page * (P // 2)
        table = torch.zeros(2, P, dtype=torch.int32, device=dev)
        table[0, :P // 2] = torch.arange(P // 2, device=dev)
        table[1, :P - P // 2] = torch.arange(P // 2, P, device=dev)
        start = torch.zeros(2, dtype=torch.int32, device=dev)
        off = torch.tensor([0, first, N], dtype=torch.int32, device=dev)
    else:         # token r alone is row r's: slot r % page of page r / page
        n = torch.arange(N, device=dev)
        table, start, off = (n // page).int()[:, None].expand(N, 1).contiguous(), (n % page).int(), None
    api.paged_append(K, V, k, v, table, start, off)
    torch.cuda.synchronize()
    for C, x in ((K, k), (V, v)):
        same = torch.equal(C.view(-1, D)[:N], x.view(N, D))
        assert same, "not every token is in its slot"
        assert not C.view(-1, D)[N:].any()


@pytest.mark.parametrize("R", [(1 << 24) - 1000, 1 << 24])
def test_attention_of_more_rows_than_one_dimension_holds(R):
    """Rows of one position: each result is that position's value, bit for bit.  Up to
    a few thousand workgroups more than rows are launched."""
    say(f"[paged grid] attention of {R} rows")
    dev, P, page, D = device(), 512, 256, 16
    q, K, V = noise(R, 1, D), noise(P, 1, page, D), noise(P, 1, page, D)
    r = torch.arange(R, device=dev)
    table, kv_len = (r % P).int()[:, None], (r % 3 != 1).int()
    out = torch.full((R, 1, D), -1.0, dtype=BF16, device=dev)
    api.paged_attn(q, K, V, table, kv_len, out=out)
    torch.cuda.synchronize()
    want = V[(r % P), :, 0] * kv_len[:, None, None].to(BF16)
    same = torch.equal(out, want)   # -0.0 of a masked row equals 0
    assert same, "not every row is attended"
