"""paged_chunk_attn where the offsets count more tokens than there are: those that there are keep
their positions, as paged_resize numbers them and paged_append writes them."""
import numpy as np
import pytest
import torch

from oracle import paged
from paper_2106_04718_amd import _native as N
from paper_2106_04718_amd import api

from _gpu import bits, device, say, to_f64
from test_gpu_paged_chunk import bound, check, make

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("count", [1, 5, 30, 31, 100, 190, 249])
@pytest.mark.parametrize("dtype,D", [(BF16, 64), (BF16, 128), (F32, 32), (BF16, 16)])
def test_rows_whose_last_tokens_are_not_given(dtype, D, count):
    d = make(count, [30, 0, 160, 60], [200, 5, 40, 700], 4, 2, D, 16, dtype)
    d["q"] = d["q"][:count]
    check(d, f"{count} of 250 tokens")


@pytest.mark.parametrize("dtype,new,cached,count", [(BF16, [5], [6000], 2), (BF16, [2000], [100], 40), (F32, [600], [0], 9), (BF16, [9], [0], 4),
                                                (BF16, [2] * 400 + [900], [40] * 400 + [30], 850)])
def test_long_rows_and_many(dtype, new, cached, count):
    d = make(len(new), new, cached, 4, 2, 64, 16, dtype)
    d["q"] = d["q"][:count]
    check(d, f"{count} of {sum(new)} tokens")


def test_a_step_of_fewer_tokens_than_the_rows_take():
    """Rows grow by more than is computed now: resize, append and attention agree on every token's
    place."""
    dev = device()
    g = torch.Generator(device=dev).manual_seed(1)
    r = lambda *s: torch.randn(*s, device=dev, generator=g).bfloat16()
    R, Hq, Hkv, D, page, cols = 3, 4, 2, 64, 16, 20
    i = lambda *a: torch.tensor(a, dtype=torch.int32, device=dev)
    grow = [7, 90, 100]
    q, k, v = r(197, Hq, D), r(197, Hkv, D), r(197, Hkv, D)
    outs = []
    for count in (197, 130):
        say(f"[chunk offsets] {count} of 197 tokens")
        K, V = torch.zeros(64, Hkv, page, D, dtype=BF16, device=dev), torch.zeros(64, Hkv, page, D, dtype=BF16, device=dev)
        table, kv_len, free, count = torch.full((R, cols), -1, dtype=torch.int32, device=dev), i(0, 0, 0), torch.arange(64, device=dev).int(), i(64)
        start, off, pos = i(0, 0, 0), i(0, 0, 0, 0), torch.zeros(count, dtype=torch.int32, device=dev)
        api.paged_resize(table, kv_len, i(*grow), free, count, page, start=start, offsets=off, positions=pos)
        assert off.tolist() == [0, 7, 97, 197] and pos[97:].tolist() == list(range(count - 97))
        api.paged_append(K, V, k[:count], v[:count], table, start, off)
        out = api.paged_chunk_attn(q[:count], K, V, table, kv_len, off)
        torch.cuda.synchronize()
        d = dict(q=bits(q[:count]), K=bits(K), V=bits(V), table=table.cpu().numpy(), kv_len=kv_len.cpu().numpy())
        ref, mean = paged.paged_chunk_attn(d["q"], d["K"], d["V"], d["table"], d["kv_len"], off.cpu().numpy())
        err, tol = np.abs(to_f64(out) - ref), bound(d, ref, mean, D ** -0.5)
        assert (err <= tol).all(), np.max(err / tol)
        assert torch.equal(out[7], v[7].repeat_interleave(2, 0))   # a row's first token attends itself alone
        outs.append(ref)
    assert np.array_equal(outs[0][:130], outs[1])


def test_debug_mode_rejects_offsets_that_decrease():
    d = make(30, [4, 4, 2], [16, 60, 0], 4, 2, 64, 16, BF16)
    t = {x: torch.from_numpy(d[x].view(np.int16) if d[x].dtype == np.uint16 else d[x]).to(device()) for x in d}
    q, K, V = (t[x].view(BF16) for x in "qKV")
    call = lambda *off: api.paged_chunk_attn(q, K, V, t["table"], t["kv_len"], torch.tensor(off, dtype=torch.int32, device=device()))
    say("[chunk offsets] debug mode")
    call(0, 8, 4, 10)      # outside of it: nothing else is touched
    with api.validate_lengths():
        call(0, 4, 8, 10)
        call(2, 2, 2, 900)     # tokens of no row, rows of none, more than there are
        for bad, needle in (((0, 8, 4, 10), r"offsets\[1\] = 8 is above offsets\[2\] = 4"), ((0, 4, 8, 7), "above"), ((1, 0, 0, 0), "above")):
            with pytest.raises(N.NativeError, match=needle):
                call(*bad)
