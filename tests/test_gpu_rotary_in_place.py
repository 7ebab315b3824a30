"""rotary in place stores nothing behind the turned elements: what another stream writes there
meanwhile stays."""
import pytest
import torch

from paper_2106_04718_amd import api

from _gpu import bits, device, say

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("tokens", [40, 30_000])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,D,rot", [(BF16, 32, 6), (BF16, 128, 20), (BF16, 64, 32), (F32, 32, 6), (F32, 64, 20), (F32, 16, 14)])
def test_the_rest_of_a_head_is_another_streams(dtype, D, rot, interleaved, tokens):
    """One stream turns the first elements back and forth by half turns, another adds 1 to the rest: each
    finds its own as if it were alone."""
    dev, H, times = device(), 6, 20
    say(f"[rotary in place] {tokens} tokens D={D} rot={rot} {'pairs' if interleaved else 'halves'} {dtype}")
    g = torch.Generator(device=dev).manual_seed(rot)
    x = torch.randint(-99, 99, (tokens, 2 * H, D), device=dev, generator=g).to(dtype)
    q, k = x[:, :H], x[:, H:]
    want = x.clone()
    want[..., rot:] += times
    pos = torch.zeros(tokens, dtype=torch.int32, device=dev)
    freq = api.rotary_frequencies(rot, device=dev)
    k_out = torch.zeros(tokens, H, D, dtype=dtype, device=dev)
    turn, add = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for i in range(times):
        with torch.cuda.stream(turn):     # negated, and back: exact
            if i % 2:
                api.rotary(q, pos, freq, k=k, out=q, k_out=k, interleaved=interleaved, magnitude=-1.0)
            else:
                api.rotary(q, pos, freq, out=q, interleaved=interleaved, magnitude=-1.0)
                api.rotary(k, pos, freq, out=k, interleaved=interleaved, magnitude=-1.0)
        with torch.cuda.stream(add):
            x[..., rot:] += 1
    torch.cuda.synchronize()
    assert torch.equal(x, want)
    # queries in place, keys not: all of the keys' output is written, nothing of the queries' rest
    for i in range(times):
        with torch.cuda.stream(turn):
            api.rotary(q, pos, freq, k=k, out=q, k_out=k_out, interleaved=interleaved, magnitude=-1.0)
        with torch.cuda.stream(add):
            q[..., rot:] += 1
    torch.cuda.synchronize()
    want[:, :H, rot:] += times
    assert torch.equal(x, want)
    assert torch.equal(k_out[..., :rot], -k[..., :rot]) and torch.equal(k_out[..., rot:], k[..., rot:])
