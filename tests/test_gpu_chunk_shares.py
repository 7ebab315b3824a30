"""paged_chunk_attn where its work is divided differently, against float64 on the GPU.

The rule that gives workgroups whole tiles or shares of all tiles is worked out here too, so
that a case is known to reach the branch that it is meant for."""
import numpy as np
import pytest
import torch

from paper_2106_04718_amd import api

from _gpu import bits, device, say

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
UNIT, START, LEAST = 128, 128, 512


def rule(new, cached, Hq, Hkv, D, dtype, cap):
    """(whole tiles or not, parts of every tile of a head)."""
    bf16 = dtype == BF16
    width = (128 if D >= 32 else 32) if bf16 else 32 if D <= 64 else 16
    places = 256 * (3 if D <= (64 if bf16 else 32) else 2)
    shares = places // Hkv if Hkv <= places // 8 else 2 * places // Hkv
    columns, rows, G = sum(new) * (Hq // Hkv), min(len(new), sum(new)), Hq // Hkv
    shares = max(1, min(shares, (columns // width + rows) * (-(-cap // UNIT) + 1)))
    borders, units, longest = [0], [], 0
    for n, c in zip(new, cached):
        tiles = -(-n * G // width)
        for i in range(tiles):
            flat = c // 2 >= n
            work = lambda j: j * (c + n // 2 + START) if flat else j * (c + START) + int(j * (j + 1) * (0.5 * width / G))
            borders.append(borders[-1] + work(i + 1) - work(i))
            units.append(max(1, -(-min(c + (min((i + 1) * width, n * G) - 1) // G + 1, cap) // UNIT)))
        if tiles:
            longest = max(longest, max(1, -(-min(n + c, cap) // UNIT)))
    share = -(-borders[-1] // shares)
    time = longest * UNIT + START
    if len(units) > shares:
        time = 1.05 * max(time, share)
    whole = len(new) <= 256 and time <= 1.12 * max(share, LEAST) + 3 * START
    if whole:
        return True, [1] * len(units)
    share, parts = max(share, LEAST), []
    for t0, t1, u in zip(borders, borders[1:], units):
        at = lambda x: 0 if x <= t0 else u if x >= t1 else min(u, int(u * ((x - t0) / (t1 - t0)) + 0.5))
        first, last = t0 // share, (t1 - 1) // share
        if last > first and at(share * (first + 1)) == 0:
            first += 1
        if last > first and at(share * last) == u:
            last -= 1
        parts.append(last - first + 1)
    return False, parts


def make(seed, new, cached, Hq, Hkv, D, page, dtype):
    dev, rng = device(), np.random.default_rng(seed)
    gen = torch.Generator(device=dev).manual_seed(seed)
    noise = lambda *s: torch.randn(*s, device=dev, dtype=dtype, generator=gen)
    lens = np.asarray(new, np.int64) + np.asarray(cached, np.int64)
    need = -(-lens // page)
    P, cols = int(need.sum()) + 3, max(1, int(need.max()))
    ids, table, at = rng.permutation(P), rng.integers(0, P, (len(lens), cols)).astype(np.int32), 0
    for r, n in enumerate(need):
        table[r, :n] = ids[at:at + n]
        at += n
    t = lambda a: torch.from_numpy(np.asarray(a, np.int32)).to(dev)
    return dict(q=noise(int(sum(new)), Hq, D), K=noise(P, Hkv, page, D), V=noise(P, Hkv, page, D), table=t(table), kv_len=t(lens),
                offsets=t(np.concatenate([[0], np.cumsum(new)])))


def want(d):
    """(out, the softmax-weighted mean of |v|) in float64."""
    Hkv, D = d["K"].shape[1], d["q"].shape[2]
    G = d["q"].shape[1] // Hkv
    out = torch.zeros(d["q"].shape, dtype=torch.float64, device=d["q"].device)
    mean = torch.zeros_like(out)
    off = d["offsets"].tolist()
    for r, L in enumerate(d["kv_len"].tolist()):
        if off[r + 1] == off[r]:
            continue
        pages = d["table"][r, :-(-L // d["K"].shape[2])].long()
        k, v = (C[pages].transpose(0, 1).reshape(Hkv, -1, D)[:, :L].double() for C in (d["K"], d["V"]))
        q = d["q"][off[r]:off[r + 1]].double().view(-1, Hkv, G, D).permute(1, 2, 0, 3)
        at = torch.arange(L - q.shape[2], L, device=q.device)
        s = torch.matmul(q, k.transpose(1, 2).contiguous()[:, None]) * D ** -0.5
        s = s.masked_fill(torch.arange(L, device=q.device) > at[:, None], float("-inf"))
        w = torch.softmax(s, -1)
        for y, x in ((out, v), (mean, v.abs())):
            y[off[r]:off[r + 1]] = torch.matmul(w, x[:, None]).permute(2, 0, 1, 3).reshape(-1, Hkv * G, D)
    return out, mean


def check(d, what, **kw):
    say(f"[chunk shares] {what}: q{tuple(d['q'].shape)} K{tuple(d['K'].shape)} lens {d['kv_len'].tolist()[:6]}")
    out = api.paged_chunk_attn(d["q"], d["K"], d["V"], d["table"], d["kv_len"], d["offsets"], **kw)
    torch.cuda.synchronize()
    ref, mean = want(d)
    bf16, D, L = d["q"].dtype == BF16, d["q"].shape[2], int(d["kv_len"].max())
    # |q . k| scale of the drawn normal values: at most |q| |k| / sqrt(D)
    dot = float(d["q"].double().norm(dim=-1).max() * d["K"].double().norm(dim=-1).max()) * D ** -0.5
    eps = 2.0 ** -24
    rel = 2 * dot * (D + 8) * eps + (L + 64) * eps + (2.0 ** -17 if bf16 else 0)
    tol = (2.0 ** -8 if bf16 else eps) * ref.abs() + 2 * rel * mean + 1e-38
    err = (out.double() - ref).abs()
    assert (err <= tol).all(), f"{what}: off by {float((err / tol).max())} of the bound"
    again = api.paged_chunk_attn(d["q"], d["K"], d["V"], d["table"], d["kv_len"], d["offsets"], **kw)
    assert np.array_equal(bits(out), bits(again)), f"{what}: the same bits again"


CASES = {
    # name: (new, cached, Hq, Hkv, D, page, dtype, whole tiles, most parts of a tile at least)
    "one tile in very many parts": ([5], [120_000], 4, 1, 128, 64, BF16, False, 200),
    "groups of parts, fp32": ([3], [30_000], 2, 2, 64, 16, F32, False, 17),
    "parts of wide tiles": ([300], [9000], 8, 2, 128, 16, BF16, False, 9),
    "whole tiles in several turns": ([300, 20, 900, 1] * 6, [0, 50, 0, 7] * 6, 24, 24, 64, 16, BF16, True, 1),
    "whole tiles, fp32": ([200, 3, 120] * 9, [0, 40, 200] * 9, 16, 16, 32, 8, F32, True, 1),
    "shares that begin and end within tiles": ([129, 1, 1, 77, 5] * 5, [900, 3000, 60, 2000, 4000] * 5, 8, 4, 128, 16, BF16, False, 2),
    "the same, narrow heads": ([129, 1, 1, 77, 5] * 5, [900, 3000, 60, 2000, 4000] * 5, 6, 6, 16, 16, BF16, False, 2),
    "the same, heads of 32": ([129, 1, 1, 77, 5] * 5, [900, 3000, 60, 2000, 4000] * 5, 10, 2, 32, 16, BF16, False, 2),
    "a long prompt from nothing": ([3000], [0], 2, 1, 64, 32, BF16, False, 1),
    "equal tiles of a late piece": ([512], [7680], 16, 4, 128, 16, BF16, False, 2),
    "70 heads": ([40, 3], [600, 2500], 70, 70, 32, 16, BF16, False, 2),
    "300 heads": ([9, 1], [40, 700], 300, 300, 16, 16, BF16, True, 1),
    "600 heads, fp32": ([2, 33], [800, 10], 600, 600, 16, 16, F32, True, 1),
    "1600 heads": ([2, 33], [100, 10], 1600, 1600, 16, 16, BF16, True, 1),
    "more rows than are looked at": ([4] * 300 + [200], [300] * 300 + [5000], 4, 2, 64, 16, BF16, False, 2),
    "more rows, fp32, many heads": ([2] * 400, [50] * 400, 40, 40, 16, 16, F32, False, 1),
}


@pytest.mark.parametrize("name", CASES)
def test_every_division(name):
    new, cached, Hq, Hkv, D, page, dtype, whole, parts = CASES[name]
    d = make(len(name), new, cached, Hq, Hkv, D, page, dtype)
    got = rule(new, cached, Hq, Hkv, D, dtype, d["table"].shape[1] * page)
    assert got[0] == whole and max(got[1]) >= parts, (got[0], max(got[1]))
    check(d, name)


def test_more_heads_than_one_dimension_of_a_launch_holds():
    """One token of one position: each result is that position's value, bit for bit."""
    dev, H, D = device(), (1 << 24) + 77, 16
    say(f"[chunk shares] {H} heads")
    ints = lambda *s: torch.randint(-1000, 1000, s, dtype=torch.int16, device=dev).to(BF16)
    q, K, V = ints(1, H, D), ints(1, H, 1, D), ints(1, H, 1, D)
    i = lambda *a: torch.tensor(a, dtype=torch.int32, device=dev)
    out = api.paged_chunk_attn(q, K, V, i([0]), i(1), i(0, 1))
    torch.cuda.synchronize()
    assert torch.equal(out, V.view(1, H, D))


@pytest.mark.parametrize("offsets", [[0, 9, 2, 20], [3, 0, 25, 20], [-5, 4, 30, 12], [20, 20, 20, 0]])
@pytest.mark.parametrize("dtype,D", [(BF16, 128), (F32, 16)])
def test_offsets_that_decrease_touch_nothing_else(dtype, D, offsets):
    """They are no valid input; what is written then lies within out and the workspace."""
    d = make(50, [8, 6, 6], [700, 30, 2000], 4, 2, D, 16, dtype)
    need = api.paged_chunk_attn_workspace_bytes(20, 3, 4, 2, 16, d["table"].shape[1], D, dtype)
    room = torch.zeros(need + 4096, dtype=torch.uint8, device=device())
    room[need:] = 123
    wide = torch.full((24, 4, D), 9.0, dtype=dtype, device=device())
    off = torch.tensor(offsets, dtype=torch.int32, device=device())
    say(f"[chunk shares] offsets {offsets}")
    api.paged_chunk_attn(d["q"], d["K"], d["V"], d["table"], d["kv_len"], off, out=wide[2:22], workspace=room[:need])
    torch.cuda.synchronize()
    assert (room[need:] == 123).all() and (wide[:2] == 9).all() and (wide[22:] == 9).all()


@pytest.mark.parametrize("D", [16, 32, 64, 128])
def test_weights_keep_their_bits_where_values_cancel(D):
    """Three positions: two of weight 1, one of weight w = exp(-s), their values such that a + b
    cancels w c but for some 2^-17 of it."""
    R, H, page = 4, 8, 16
    rng = np.random.default_rng(D)
    bf16 = lambda x: torch.from_numpy(np.asarray(x)).to(BF16).double().numpy()
    s = bf16(rng.uniform(0.3, 1.0, (R, H)))
    w = np.exp(-s)[..., None]
    c = bf16(rng.uniform(1, 2, (R, H, D)))
    a = bf16(-w * c)
    b = bf16(-w * c - a)
    q, K, V = np.zeros((R, H, D)), np.zeros((R, H, page, D)), np.zeros((R, H, page, D))
    q[..., 0], K[:, :, 1, 0] = s, -1.0          # scores 0, -s, 0: exact
    V[:, :, 0], V[:, :, 1], V[:, :, 2] = a, c, b
    dev = device()
    t = lambda x: torch.from_numpy(x).float().to(BF16).to(dev)
    say(f"[chunk bits] D={D}")
    out = api.paged_chunk_attn(t(q), t(K), t(V), torch.arange(R, dtype=torch.int32, device=dev)[:, None],
                               torch.full((R,), 3, dtype=torch.int32, device=dev), torch.arange(R + 1, dtype=torch.int32, device=dev),
                               scale=1.0).double().cpu().numpy()
    ref = (a + b + w * c) / (2 + w)
    terms = (np.abs(a) + np.abs(b) + w * c) / (2 + w)
    # A weight in [2^e, 2^(e+1)) is the sum of two bf16 parts.  The first is off by at most half a
    # step, 2^(e-8); what is left lies below that, in a binade from 2^(e-9) or less, whose half step is
    # at most 2^(e-9) 2^-8: 2^-17 of the weight.  In steps of 2^-24 of the terms: 2 for the score in
    # base 2, 2 for exp2, 16 for the sums.
    tol = 2.0 ** -8 * np.abs(ref) + 2.0 ** -17 * w * c / (2 + w) + 20 * 2.0 ** -24 * terms
    assert (np.abs(out - ref) <= tol).all(), np.max(np.abs(out - ref) / tol)
