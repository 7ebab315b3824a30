"""GPU parity of paged_chunk_attn (several new tokens per row) with the fp64 form.

Cache slots that no token attends hold NaN, so a read of one shows."""
import math

import numpy as np
import pytest
import torch

from oracle import paged
from paper_2106_04718_amd import _native as N
from paper_2106_04718_amd import api, workloads

from _gpu import bits, device, say, to_f64
from test_gpu_paged import dev_of, draw, nan_like

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def make(seed, new, cached, Hq, Hkv, D, page, dtype, sigma=1.0, lead=0, trail=0, extra_cols=0):
    """Rows of `cached` positions and `new` tokens behind them, pages in random order, NaN in
    every slot that no row attends; `lead` and `trail` tokens of no row around them."""
    rng = np.random.default_rng(seed)
    new, cached = np.asarray(new, np.int64), np.asarray(cached, np.int64)
    lens = new + cached
    need = -(-lens // page)
    P = int(need.sum()) + 5
    cols = max(1, int(need.max(initial=0))) + extra_cols
    ids, at = rng.permutation(P), 0
    table = rng.integers(0, P, (len(new), cols)).astype(np.int32)   # columns behind a row name pages of others
    K, V = nan_like((P, Hkv, page, D), dtype), nan_like((P, Hkv, page, D), dtype)
    for r in range(len(new)):
        table[r, :need[r]] = ids[at:at + need[r]]
        at += need[r]
        for j in range(need[r]):
            n = min(page, lens[r] - j * page)
            K[table[r, j], :, :n] = draw(rng, (Hkv, n, D), dtype, sigma)
            V[table[r, j], :, :n] = draw(rng, (Hkv, n, D), dtype)
    off = lead + np.concatenate([[0], np.cumsum(new)])
    q = draw(rng, (int(off[-1]) + trail, Hq, D), dtype, sigma)
    return dict(q=q, K=K, V=V, table=table, kv_len=lens.astype(np.int32), offsets=off.astype(np.int32))


def bound(d, ref, mean, scale):
    """Of |out - ref|: half a step of the output's type, and what fp32 can lose of the terms p v
    of a sum: by a score of D products and its scaling, twice (its own and the maximum's); by
    exp2 and the sums over the keys; and 2^-17 by bf16 weights in two parts."""
    q, k = (np.nan_to_num(paged._f64(d[x]), posinf=0, neginf=0) for x in "qK")   # tokens and slots of nobody hold NaN
    dot = np.sqrt((q ** 2).sum(-1).max(initial=0)) * np.sqrt((k ** 2).sum(-1).max(initial=0)) * abs(scale)
    D, L = q.shape[-1], min(int(d["kv_len"].max(initial=0)), d["table"].shape[1] * d["K"].shape[2])
    eps = 2.0 ** -24
    bf16 = d["q"].dtype == np.uint16
    rel = 2 * dot * (D + 8) * eps + (L + 64) * eps + (2.0 ** -17 if bf16 else 0)
    return (2.0 ** -8 if bf16 else eps) * np.abs(ref) + 2 * rel * mean + 1e-38


def run(d, what, scale=None, **kw):
    say(f"[paged chunk] {what}: q{d['q'].shape} K{d['K'].shape} lens {d['kv_len'].tolist()[:8]} of {np.diff(d['offsets']).tolist()[:8]}")
    t = {x: dev_of(d[x]) for x in d}
    out = kw.pop("out", None)
    if out is None:
        out = torch.full_like(t["q"], 7.0)
    api.paged_chunk_attn(t["q"], t["K"], t["V"], t["table"], t["kv_len"], t["offsets"], out=out, scale=scale, **kw)
    torch.cuda.synchronize()
    return out, t


def check(d, what, scale=None, **kw):
    out, t = run(d, what, scale, **kw)
    ref, mean = paged.paged_chunk_attn(d["q"], d["K"], d["V"], d["table"], d["kv_len"], d["offsets"], scale)
    got = to_f64(out)
    nobody = np.isnan(ref).all((1, 2))
    assert (got[nobody] == 7.0).all(), f"{what}: tokens of no row are left as they were"
    got, ref, mean = got[~nobody], ref[~nobody], mean[~nobody]
    err, tol = np.abs(got - ref), bound(d, ref, mean, d["q"].shape[-1] ** -0.5 if scale is None else scale)
    assert np.isfinite(got).all() and (err <= tol).all(), f"{what}: off by {np.max(err / tol)} of the bound"
    return out


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [16, 32, 64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(4, 4), (8, 2), (3, 1)])
def test_types_widths_and_shared_heads(dtype, D, Hq, Hkv):
    check(make(D + Hq, [1, 3, 0, 20, 5, 150], [0, 33, 7, 200, 64, 10], Hq, Hkv, D, 16, dtype), "widths")


@pytest.mark.parametrize("G", [1, 2, 3, 5, 7, 8, 15, 16, 17, 31, 33, 48, 130])
def test_query_heads_per_key_value_head(G):
    check(make(G, [7, 40, 1], [70, 5, 0], 2 * G, 2, 64, 16, BF16), f"G={G}")
    check(make(G, [7, 9], [0, 50], G, 1, 32, 8, F32), f"G={G}")


@pytest.mark.parametrize("page", [1, 2, 3, 5, 7, 16, 24, 100, 128, 257])
def test_page_sizes(page):
    check(make(page, [1, 30, 130, 4], [31, 1, 20, 296], 4, 2, 64, page, BF16), f"page={page}")
    check(make(page, [1, 33, 9], [1, 7, 250], 2, 2, 32, page, F32), f"page={page}")


@pytest.mark.parametrize("dtype,Hq,Hkv,D", [(BF16, 4, 1, 64), (BF16, 1, 1, 128), (F32, 2, 1, 16)])
def test_every_length_around_the_tiles(dtype, Hq, Hkv, D):
    new = [0, 1, 2, 7, 8, 9, 15, 16, 17, 31, 32, 33, 34, 63, 64, 65, 66, 127, 128, 129, 160]
    for cached in (0, 1, 31, 64, 100):
        check(make(cached, new, [cached] * len(new), Hq, Hkv, D, 16, dtype), f"{cached} cached")


@pytest.mark.parametrize("dtype,new,cached", [(BF16, [5], [4000]), (BF16, [1, 40, 2], [20, 3000, 0]), (F32, [3, 1], [2500, 2]),
                                              (BF16, [4] * 3, [2045] * 3), (BF16, [40, 1], [2600, 2600])])
def test_few_tokens_of_long_rows(dtype, new, cached):
    check(make(len(new), new, cached, 8, 2, 64, 64, dtype, sigma=0.5), "long rows")


def test_many_rows():
    rng = np.random.default_rng(5)
    new, cached = rng.integers(0, 4, 700), rng.integers(0, 40, 700)
    new[345], cached[345] = 50, 1500
    check(make(9, new, cached, 4, 2, 32, 16, BF16), "one long row among 700")
    check(make(10, np.ones(2000, int), np.zeros(2000, int), 2, 1, 16, 16, BF16), "2000 rows of one position")
    check(make(11, [0] * 300 + [3] + [0] * 300, [9] * 601, 2, 1, 16, 16, F32), "one row with tokens")


def test_one_token_per_row_is_the_attention_of_one_token():
    d = make(12, [1] * 6, [0, 5, 31, 700, 64, 1500], 8, 2, 128, 16, BF16)
    t = {x: dev_of(d[x]) for x in d}
    got = to_f64(check(d, "one token"))
    one = to_f64(api.paged_attn(t["q"], t["K"], t["V"], t["table"], t["kv_len"]))
    ref, mean = paged.paged_chunk_attn(d["q"], d["K"], d["V"], d["table"], d["kv_len"], d["offsets"])
    assert (np.abs(got - one) <= 2 * bound(d, ref, mean, 128 ** -0.5)).all()


def test_tokens_of_no_row_are_left_alone():
    d = make(13, [5, 0, 70], [3, 9, 100], 4, 2, 64, 16, BF16, lead=3, trail=40)
    d["q"][:3] = d["q"][-40:] = workloads.BF16_NAN
    check(d, "padded")


def test_tokens_that_attend_nothing():
    d = make(14, [5, 40, 3, 2], [4, 10, 0, 0], 4, 2, 64, 16, BF16)
    d["kv_len"] = np.array([2, 20, 0, -5], np.int32)   # shorter than the tokens: the first ones come before position 0
    out = to_f64(check(d, "before the beginning"))
    assert not out[:3].any() and not out[5:25].any() and not out[45:].any() and out[25:45].any()
    d = make(15, [4, 33], [0, 0], 4, 2, 64, 16, F32)
    d["table"][:] = -1
    assert not to_f64(check(d, "no pages")).any()


def test_bad_pages_and_lengths_past_the_table():
    d = make(16, [10, 36, 33, 4], [90, 54, 31, 60], 4, 2, 64, 16, BF16)
    d["K"], d["V"] = (np.where(x == workloads.BF16_NAN, np.uint16(0x3f80), x) for x in (d["K"], d["V"]))
    d["table"][0, 2] = -1                      # one page in the middle
    d["table"][1, :] = [d["K"].shape[0], -7, 2**31 - 1, -2**31, -1, -1, -1][:d["table"].shape[1]]   # every page
    d["table"][2, 3] = d["K"].shape[0]         # the last page
    d["kv_len"][3] = 2**31 - 1                 # far past the table: every token attends all of it
    out = to_f64(check(d, "bad pages"))
    assert not out[10:46].any()


@pytest.mark.parametrize("dtype,new,cached,Hq", [(BF16, 6, 40, 4), (BF16, 90, 20, 4), (F32, 40, 30, 2), (BF16, 3, 0, 1), (BF16, 200, 0, 1)])
def test_infinities_and_nan_behind_a_token_do_not_reach_it(dtype, new, cached, Hq):
    d = make(17, [new], [cached], Hq, 1, 64, 16, dtype)
    at = cached + new // 2
    pg, sl = d["table"][0, at // 16], at % 16
    f32 = lambda x: np.float32(x) if dtype == F32 else workloads.f32_to_bf16_bits(np.array([x], np.float32))[0]
    d["V"][pg, 0, sl, 5], d["V"][pg, 0, sl, 40], d["V"][pg, 0, sl, 63] = f32(np.inf), f32(-np.inf), f32(np.nan)
    last = cached + new - 1
    d["K"][d["table"][0, last // 16], 0, last % 16, 3] = f32(np.nan)   # a NaN key of the last token
    out, _ = run(d, "infinities and NaN")
    got = to_f64(out)
    clean = dict(d, V=d["V"].copy(), K=d["K"].copy())
    clean["V"][pg, 0, sl] = f32(1.0)
    clean["K"][d["table"][0, last // 16], 0, last % 16] = f32(1.0)
    ref, mean = paged.paged_chunk_attn(*(clean[x] for x in ("q", "K", "V", "table", "kv_len", "offsets")))
    first = new // 2
    assert (np.abs(got - ref) <= bound(clean, ref, mean, 0.125))[:first].all(), "tokens before it"
    # those that attend it: an infinity or NaN, as documented (0 of a weight's parts times it)
    assert not (got[first:-1, :, 5] < np.inf).any() and not (got[first:-1, :, 40] > -np.inf).any() and np.isnan(got[first:-1, :, 63]).all()
    others = [x for x in range(64) if x not in (5, 40, 63)]
    assert np.isfinite(got[:-1, :, others]).all() and np.isnan(got[-1]).all()


def test_large_scores_and_scales():
    check(make(18, [30, 5], [370, 72], 4, 2, 64, 16, F32, sigma=20.0), "scores of hundreds")
    check(make(19, [40, 5], [370, 72], 4, 2, 64, 16, BF16), "scale 0", scale=0.0)
    check(make(20, [40, 5], [370, 72], 4, 2, 64, 16, BF16), "negative scale", scale=-0.3)
    d = make(21, [40], [260], 1, 1, 64, 16, F32)
    d["q"][:] = 1e4
    d["K"][:] = np.where(np.isnan(d["K"]), np.nan, -1e4).astype(np.float32)   # every score very low
    check(d, "all scores equal and very low")


@pytest.mark.parametrize("dtype,new", [(BF16, [5, 1, 3]), (BF16, [50, 0, 130]), (F32, [9, 1, 30])])
def test_strides(dtype, new):
    """Token-major pages, keys and values interleaved, q cut from one projection, a table
    with a leading dimension: the same bits."""
    Hq, Hkv, D, page = 4, 2, 64, 16
    d = make(22, new, [50, 1, 130], Hq, Hkv, D, page, dtype)
    want, _ = run(d, "contiguous")
    dev = device()
    kv = torch.empty(d["K"].shape[0], page, 2, Hkv, D, dtype=dtype, device=dev)
    K, V = kv[:, :, 0].transpose(1, 2), kv[:, :, 1].transpose(1, 2)
    K.copy_(dev_of(d["K"])), V.copy_(dev_of(d["V"]))
    qkv = torch.empty(len(d["q"]), Hq + 2 * Hkv, D, dtype=dtype, device=dev)
    q = qkv[:, :Hq]
    q.copy_(dev_of(d["q"]))
    table = torch.full((3, 40), -1, dtype=torch.int32, device=dev)
    table[:, :d["table"].shape[1]] = dev_of(d["table"])
    out = api.paged_chunk_attn(q, K, V, table[:, :d["table"].shape[1]], dev_of(d["kv_len"]), dev_of(d["offsets"]))
    torch.cuda.synchronize()
    assert np.array_equal(bits(out), bits(want))
    # one K for all heads and V the same array: a cache that is read alone may be expanded
    wide = torch.randn(9, 1, page, D, device=dev).to(dtype).expand(9, Hkv, page, D)
    one = lambda C: api.paged_chunk_attn(q, C, C, table[:, :3] * 0, torch.full_like(dev_of(d["kv_len"]), 40), dev_of(d["offsets"]))
    assert np.array_equal(bits(one(wide)), bits(one(wide.contiguous())))


def test_the_same_call_twice_gives_the_same_bits_and_any_workspace_serves():
    big = make(23, [5, 300, 1], [6000, 40, 700], 8, 2, 64, 16, BF16)
    small = make(24, [30, 2], [300, 2], 4, 4, 32, 8, F32)
    many = make(25, [2] * 300, [40] * 300, 4, 2, 32, 16, BF16)
    need = lambda d: api.paged_chunk_attn_workspace_bytes(len(d["q"]), len(d["kv_len"]), d["q"].shape[1], d["K"].shape[1], d["K"].shape[2],
                                                          d["table"].shape[1], d["q"].shape[2], F32 if d["q"].dtype == np.float32 else BF16)
    sets = (big, small, many)
    ws = api.new_workspace(max(need(d) for d in sets), device())
    first = [bits(run(x, "fresh workspace")[0]) for x in sets]
    for _ in range(3):   # sizes that alternate in one workspace
        for x, want in zip(sets, first):
            assert np.array_equal(bits(run(x, "shared workspace", workspace=ws)[0]), want)


def test_cache_behind_32_bits():
    """A page table that reaches past 4 GiB of a cache."""
    dev = device()
    P, Hkv, page, D = 70_000, 4, 128, 128          # 9.2 GB in bf16
    K = torch.empty(P, Hkv, page, D, dtype=BF16, device=dev)
    V = torch.empty_like(K)
    for new in ([3, 1], [40, 100]):
        d = make(26, new, [300, 129], 8, Hkv, D, page, BF16)
        far = np.array([P - 1, 0, 40_000, 33_000, 65_535, 16_384, 32_768, 8192, 1, 2, 3, 4], np.int32)[:d["K"].shape[0]]
        K[torch.from_numpy(far).long().to(dev)] = dev_of(d["K"])
        V[torch.from_numpy(far).long().to(dev)] = dev_of(d["V"])
        want, _ = run(d, "near pages")
        out = api.paged_chunk_attn(dev_of(d["q"]), K, V, dev_of(far[d["table"]]), dev_of(d["kv_len"]), dev_of(d["offsets"]))
        torch.cuda.synchronize()
        assert np.array_equal(bits(out), bits(want))


def test_empty_calls():
    dev = device()
    K = torch.zeros(2, 2, 16, 64, dtype=BF16, device=dev)
    e = lambda *s, t=BF16: torch.empty(*s, dtype=t, device=dev)
    z = lambda *s: torch.zeros(*s, dtype=torch.int32, device=dev)
    assert api.paged_chunk_attn(e(0, 4, 64), K, K, z(3, 1), z(3), z(4)).shape == (0, 4, 64)
    out = torch.full((2, 4, 64), 3.0, dtype=BF16, device=dev)
    api.paged_chunk_attn(e(2, 4, 64), K, K, z(0, 1), z(0), z(1), out=out)     # no rows: nobody's tokens
    assert (out == 3).all()
    api.paged_chunk_attn(e(2, 4, 64), K, K, z(2, 0), z(2) + 9, torch.tensor([0, 1, 2], dtype=torch.int32, device=dev), out=out)
    assert not out.any()   # a table without columns


def test_debug_mode_rejects_lengths_outside_the_table():
    d = make(27, [4, 4], [16, 60], 4, 2, 64, 16, BF16)
    t = {x: dev_of(d[x]) for x in d}
    call = lambda n: api.paged_chunk_attn(t["q"], t["K"], t["V"], t["table"], torch.tensor(n, dtype=torch.int32, device=device()), t["offsets"])
    with api.validate_lengths():
        call([20, 64])
        for bad in ([20, 65], [-1, 64]):
            with pytest.raises(N.NativeError, match="kv_len"):
                call(bad)


@pytest.mark.parametrize("change,needle", [
    (dict(q=lambda x: x["q"].float()), "q must be"), (dict(q=lambda x: x["q"][0]), "dimensions"),
    (dict(V=lambda x: x["V"].transpose(0, 1).contiguous().transpose(0, 1)), "same shape and strides"),
    (dict(table=lambda x: x["table"].long()), "table must be"), (dict(kv_len=lambda x: x["kv_len"][:1]), "kv_len must be"),
    (dict(offsets=lambda x: x["offsets"][:2]), "offsets must be"), (dict(offsets=lambda x: x["offsets"].cpu()), "GPU tensor"),
    (dict(offsets=lambda x: x["offsets"].long()), "offsets must be"),
    (dict(out=lambda x: x["q"]), "overlaps"), (dict(out=lambda x: x["q"].float()), "out must match"),
    (dict(workspace=lambda x: torch.zeros(8, dtype=torch.uint8, device=x["q"].device)), "workspace of 8 bytes"),
    (dict(q=lambda x: x["q"][:, :3].contiguous()), "multiple of Hkv"), (dict(scale=lambda x: math.inf), "scale"),
    (dict(table=lambda x: x["table"][:1]), "kv_len must be"),
])
def test_refusals_of_the_front_end(change, needle):
    d = make(40, [20, 5], [3, 4], 4, 2, 64, 16, BF16)
    x = {n: dev_of(a) for n, a in d.items()}
    x.update({n: f(x) for n, f in change.items()})
    with pytest.raises((ValueError, N.NativeError), match=needle):
        api.paged_chunk_attn(x.pop("q"), x.pop("K"), x.pop("V"), x.pop("table"), x.pop("kv_len"), x.pop("offsets"), **x)
