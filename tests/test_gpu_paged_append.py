"""paged_append where its kernels change: tokens of few bytes stand side by side in
a workgroup (up to 64 chunks of 16 bytes each), many tokens go four at a time.
Compared bit for bit with an indexed assignment, at sizes around both rules."""
import numpy as np
import pytest
import torch

from paper_2106_04718_amd import api

from _gpu import device, say

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def check(lens, Hkv, D, page, dtype, lead=0, trail=0, seed=0, bad=()):
    rng = np.random.default_rng(seed)
    lens = np.asarray(lens, np.int64)
    R, N = len(lens), lead + int(lens.sum()) + trail
    say(f"[append sizes] R={R} N={N} Hkv={Hkv} D={D} page={page} {dtype}")
    start = rng.integers(0, 2 * page, R)
    need = np.where(lens > 0, -(-(start + lens) // page), 0)
    P, cols = int(need.sum()) + 3, max(1, int(need.max(initial=0)))
    ids, at = rng.permutation(P), 0
    table = np.full((R, cols), -1, np.int32)
    for r in np.flatnonzero(need):
        table[r, :need[r]] = ids[at:at + need[r]]
        at += need[r]
    for r in bad:
        table[r, 0] = P   # no page: the tokens there go nowhere
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(device())
    gen = torch.Generator(device=device()).manual_seed(seed)
    noise = lambda *s: torch.randn(*s, device=device(), dtype=dtype, generator=gen)
    K, V, k, v = noise(P, Hkv, page, D), noise(P, Hkv, page, D), noise(N, Hkv, D), noise(N, Hkv, D)
    wK, wV = K.clone(), V.clone()
    off = lead + np.concatenate([[0], np.cumsum(lens)])
    row = dev(np.repeat(np.arange(R), lens))
    n = torch.arange(len(row), device=device()) + lead
    pos = dev(start)[row] + n - dev(off)[row]
    pg = dev(table)[row, pos // page].long()
    ok = (pg >= 0) & (pg < P)
    wK[pg[ok], :, (pos % page)[ok]] = k[n[ok]]
    wV[pg[ok], :, (pos % page)[ok]] = v[n[ok]]
    api.paged_append(K, V, k, v, dev(table), dev(start.astype(np.int32)), dev(off.astype(np.int32)))
    torch.cuda.synchronize()
    same = torch.equal(K, wK) and torch.equal(V, wV)
    assert same, f"R={R} N={N} Hkv={Hkv} D={D}"


# chunks of a token: 2, 6, 40, 56, 64 side by side; 72, 128 and 320 one behind another
@pytest.mark.parametrize("Hkv,D,dtype", [(1, 16, BF16), (3, 16, BF16), (5, 64, BF16), (7, 32, F32), (4, 128, BF16),
                                         (9, 64, BF16), (8, 128, BF16), (10, 128, F32)])
@pytest.mark.parametrize("turns", [0.4, 1, 1.1])
def test_around_the_number_of_tokens_that_go_four_at_a_time(Hkv, D, dtype, turns):
    per = Hkv * D * (2 if dtype == BF16 else 4) // 16
    side = 256 // per if per <= 64 else 1
    n = int(2048 * side * turns)
    parts = np.array([1, 0, 3, 700, 5, 0, 0, 1000, 2, 333])
    lens = parts * n // parts.sum()
    lens[3] += n - 7 - lens.sum()
    check(lens, Hkv, D, 16, dtype, lead=3, trail=4, seed=per, bad=[4])        # n tokens, seven of no row
    check(lens, Hkv, D, 7, dtype, seed=per + 1)


@pytest.mark.parametrize("Hkv,D", [(1, 16), (2, 64), (8, 128)])
def test_rows_without_tokens_between_rows_with_some(Hkv, D):
    lens = np.zeros(60_000, np.int64)
    lens[[0, 1, 2, 17, 18, 30_000, 59_998]] = [1, 2, 3, 2049, 2, 3001, 5]     # borders inside groups of four
    check(lens, Hkv, D, 16, BF16)
    lens[:] = 0
    lens[59_999] = 9001
    check(lens, Hkv, D, 16, BF16, lead=1)
    check(np.random.default_rng(1).integers(0, 2, 30_000), Hkv, D, 16, BF16, trail=9)   # ones and none
