"""paged_resize's refused rows: their tokens reach no page of another row, whatever the table held
behind the rows' pages."""
import numpy as np
import pytest
import torch

from paper_2106_04718_amd import api

from _gpu import device, say
from test_gpu_resize import check, state

pytestmark = pytest.mark.gpu

I32 = torch.int32


@pytest.mark.parametrize("page", [1, 16])
@pytest.mark.parametrize("R", [1, 70, 1024, 2500])
def test_tables_that_name_pages_behind_their_rows(R, page):
    """Entries behind a row's pages name pages of others, as in a table of zeros: a row that wants
    them and gets none has -1 there, others keep what they had."""
    rng = np.random.default_rng(R + page)
    cols = 150
    d = state(R, rng.integers(0, 40 * page, R), page, cols, R)
    behind = np.arange(cols) >= -(-d["kv_len"][:, None] // page)
    d["table"] = np.where(behind, rng.integers(0, len(d["free_pages"]), (R, cols)), d["table"]).astype(np.int32)
    want = d["kv_len"] + rng.integers(0, 90 * page, R)
    want[rng.random(R) < 0.3] -= 5 * page
    want[rng.random(R) < 0.1] = 2**31 - 1      # past the table
    want[rng.random(R) < 0.1] = 0
    n = int(np.minimum(np.maximum(want.astype(np.int64) - d["kv_len"], 0), 100 * page).sum())
    check(d, want, page, min(n, 100_000), "entries of other rows", ld=3)


def test_appended_tokens_of_refused_rows_stay_in_their_last_page():
    dev = device()
    Hkv, D, page, P = 2, 64, 16, 8
    i = lambda *a: torch.tensor(a, dtype=I32, device=dev)
    table = torch.zeros(3, 6, dtype=I32, device=dev)     # zeros behind the rows' pages: page 0 is the first row's
    table[0, 0], table[1, 0], table[2, 0] = 0, 3, 5
    kv_len, free, count = i(16, 10, 16), i(1, 2, 4, 0, 0, 0, 0, 0), i(3)
    start, off, slots = i(0, 0, 0), i(0, 0, 0, 0), torch.zeros(300, dtype=torch.int64, device=dev)
    api.paged_resize(table, kv_len, i(33, 90, 70), free, count, page, start=start, offsets=off, slots=slots)
    say("[resize refused] append")
    K = torch.zeros(P, Hkv, page, D, dtype=torch.bfloat16, device=dev)
    V = torch.zeros_like(K)
    k = torch.ones(300, Hkv, D, dtype=torch.bfloat16, device=dev)
    api.paged_append(K, V, k, k, table, start, off)
    torch.cuda.synchronize()
    assert kv_len.tolist() == [33, 10, 16] and count.item() == 1 and off.tolist() == [0, 17, 97, 151]
    assert table.tolist() == [[0, 4, 2, 0, 0, 0], [3, -1, -1, -1, -1, -1], [5, -1, -1, -1, -1, 0]]
    assert (slots[17:] == -1).all() and slots[:17].tolist() == [*range(64, 80), 32]
    for C in (K, V):
        wrote = (C != 0).any(3).any(1)      # of every page, its places
        want = torch.zeros_like(wrote)
        want[4] = want[2, 0] = True         # the granted row's tokens
        want[3, 10:] = True                 # behind the end of the second row, in its last page
        assert torch.equal(wrote, want)


def test_a_refused_rows_token_left_out_of_the_attention_of_one_token():
    """Lengths of 0 for rows that got no page: nothing of theirs is written, and their results are 0."""
    dev = device()
    Hq, Hkv, D, page, P = 4, 2, 64, 16, 6
    g = torch.Generator(device=dev).manual_seed(2)
    r = lambda *s: torch.randn(*s, device=dev, generator=g).bfloat16()
    i = lambda *a: torch.tensor(a, dtype=I32, device=dev)
    K, V = r(P, Hkv, page, D), r(P, Hkv, page, D)
    keep = K.clone(), V.clone()
    table = torch.full((3, 4), -1, dtype=I32, device=dev)
    table[0, 0], table[1, 0], table[2, 0] = 0, 3, 5
    kv_len, free, count = i(16, 16, 9), i(4, 0, 0, 0, 0, 0), i(1)
    want = kv_len + 1
    api.paged_resize(table, kv_len, want, free, count, page)
    say("[resize refused] one token")
    q, k, v = r(3, Hq, D), r(3, Hkv, D), r(3, Hkv, D)
    out = api.paged_attn(q, K, V, table, torch.where(kv_len == want, kv_len, 0), k=k, v=v)
    torch.cuda.synchronize()
    assert kv_len.tolist() == [17, 16, 10] and not out[1].any() and out[0].any() and out[2].any()
    for C, was, x in ((K, keep[0], k), (V, keep[1], v)):
        was[4, :, 0], was[5, :, 9] = x[0], x[2]
        assert torch.equal(C, was)
