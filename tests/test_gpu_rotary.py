"""GPU parity of rotary positions with the fp64 form."""
import numpy as np
import pytest
import torch

from oracle import paged
from paper_2106_04718_amd import _native as N
from paper_2106_04718_amd import api

from _gpu import bits, device, say, to_f64
from test_gpu_paged import dev_of, draw

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def bound(ref, pair, dtype, magnitude):
    """Half a step of the output's type, and of the magnitude of the pair: 2^-24 each for the angle
    behind its reduction (at most pi / 4, rounded), the series (some steps of 2^-24 of at most
    1: 4 of them), the magnitude's product and the two products and the sum (3)."""
    half = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
    return half * np.abs(ref) + 10 * 2.0 ** -24 * abs(magnitude) * pair


def pairs(x, half, interleaved):
    """Of every element the length of its pair (0 behind the pairs)."""
    x, out = paged._f64(x), np.zeros(x.shape)
    a = x[..., 0:2 * half:2] if interleaved else x[..., :half]
    b = x[..., 1:2 * half:2] if interleaved else x[..., half:2 * half]
    r = np.hypot(a, b)
    if interleaved:
        out[..., 0:2 * half:2], out[..., 1:2 * half:2] = r, r
    else:
        out[..., :half], out[..., half:2 * half] = r, r
    return out


def check(seed, N_, Hq, Hkv, D, rot, interleaved, dtype, far=4096, magnitude=1.0, freq=None, in_place=False, what=""):
    say(f"[rotary] {what} N={N_} H={Hq}+{Hkv} D={D} rot={rot} {'pairs' if interleaved else 'halves'} {dtype}")
    rng = np.random.default_rng(seed)
    q, k = draw(rng, (N_, Hq, D), dtype), draw(rng, (N_, Hkv, D), dtype)
    pos = rng.integers(-far, far, N_).astype(np.int32)
    freq = paged.rotary_frequencies(rot) if freq is None else freq
    tq, tk = (dev_of(x) if x.size else torch.empty(x.shape, dtype=dtype, device=device()) for x in (q, k))
    kw = dict(out=tq, k_out=tk) if in_place else {}
    out = api.rotary(tq, dev_of(pos), dev_of(freq), k=tk if Hkv else None, interleaved=interleaved, magnitude=magnitude,
                     **(kw if Hkv else {x: kw[x] for x in kw if x == "out"}))
    torch.cuda.synchronize()
    for got, x in zip(out if Hkv else (out,), (q, k)):
        ref = paged.rotary(x, pos, freq, interleaved, magnitude)
        err, tol = np.abs(to_f64(got) - ref), bound(ref, pairs(x, rot // 2, interleaved), dtype, magnitude)
        assert (err <= tol).all(), f"off by {np.max(err / np.maximum(tol, 1e-300))} of the bound"
        assert np.array_equal(to_f64(got)[..., rot:], paged._f64(x)[..., rot:])
    if not in_place:
        for t, x in ((tq, q), (tk, k)):
            assert np.array_equal(bits(t), x.view(bits(t).dtype))


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [16, 32, 64, 128])
def test_widths_and_parts_of_the_head(D, dtype, interleaved, in_place):
    for rot in sorted({0, 2, 4, 6, 10, 12, 14, D // 4, D // 2, D - 2, D}):
        check(D + rot, 5, 3, 2, D, rot, interleaved, dtype, in_place=in_place)


@pytest.mark.parametrize("N_,Hq,Hkv", [(1, 1, 0), (1, 32, 8), (7, 0, 3), (300, 12, 12), (2049, 3, 1), (2050, 1, 0), (3, 200, 40)])
def test_tokens_and_heads(N_, Hq, Hkv):
    check(N_, N_, Hq, Hkv, 64, 64, False, BF16)
    check(N_, N_, Hq, Hkv, 32, 20, True, F32)


@pytest.mark.parametrize("interleaved", [False, True])
def test_far_positions_keep_their_angles(interleaved):
    check(1, 40, 2, 1, 64, 64, interleaved, F32, far=2**31 - 1, what="far")
    check(2, 40, 2, 1, 64, 64, interleaved, F32, far=1 << 20, magnitude=1.25, freq=paged.rotary_frequencies(64, 5e5, 8.0, 8192))
    check(3, 40, 2, 1, 16, 16, interleaved, F32, far=9, freq=np.array([0.0, np.pi / 2, np.pi, -np.pi / 4, 3.0, 1e-9, 100.0, np.pi / 4]),
          what="quarter turns")
    check(4, 4, 1, 1, 16, 16, interleaved, BF16, magnitude=-0.5)


def test_turning_back_gives_the_vectors():
    g = torch.Generator(device=device()).manual_seed(3)
    x = torch.randn(50, 4, 128, device=device(), generator=g)
    pos = torch.randint(0, 1 << 20, (50,), device=device(), generator=g).int()
    freq = api.rotary_frequencies(128, device=device())
    back = api.rotary(api.rotary(x, pos, freq), -pos, freq)
    assert (back - x).abs().max() <= 40 * 2.0 ** -24 * x.abs().max() * 2 ** 0.5


def test_strides_and_a_projection_in_place():
    dev = device()
    g = torch.Generator(device=dev).manual_seed(4)
    for dtype in (BF16, F32):
        qkv = torch.randn(9, 8, 64, device=dev, generator=g).to(dtype)
        q, k, v = qkv.split([4, 2, 2], 1)
        pos, freq = torch.arange(9, device=dev).int(), api.rotary_frequencies(64, device=dev)
        want = api.rotary(q.clone(), pos, freq, k=k.clone())
        keep = v.clone()
        a, b = api.rotary(q, pos, freq, k=k, out=q, k_out=k)
        assert a is q and b is k and torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(v, keep)
        # heads of q, k and v in turn, [N, H, 3, D]; outputs head-major
        x = torch.randn(9, 4, 3, 64, device=dev, generator=g).to(dtype)
        want = api.rotary(x[:, :, 0].clone(), pos, freq, k=x[:, :, 1].clone())
        out = [torch.zeros(4, 9, 64, device=dev, dtype=dtype).transpose(0, 1) for _ in range(2)]
        api.rotary(x[:, :, 0], pos, freq, k=x[:, :, 1], out=out[0], k_out=out[1])
        api.rotary(x[:, :, 0], pos, freq, k=x[:, :, 1], out=x[:, :, 0], k_out=x[:, :, 1])
        for i in range(2):
            assert torch.equal(out[i], want[i]) and torch.equal(x[:, :, i], want[i])


def test_what_is_not_finite_stays_in_its_pair():
    dev = device()
    for inter in (False, True):
        x = torch.ones(2, 1, 64, device=dev)
        x[0, 0, 3], x[1, 0, 50] = float("inf"), float("nan")
        got = api.rotary(x, torch.tensor([5, 6], device=dev).int(), api.rotary_frequencies(40, device=dev), interleaved=inter)
        partner = 2 if inter else 23
        bad = torch.zeros(2, 64, dtype=torch.bool, device=dev)
        bad[0, 3] = bad[0, partner] = bad[1, 50] = True   # 50 lies behind the pairs: kept as it is
        assert torch.equal(~torch.isfinite(got[:, 0]), bad)


def test_frequencies():
    for rot, base, factor, context in ((0, 1e4, 1.0, 0), (2, 1e4, 1.0, 0), (64, 1e4, 4.0, 0), (128, 5e5, 8.0, 8192), (20, 100.0, 0.5, 64)):
        got = api.rotary_frequencies(rot, base, factor, context)
        want = paged.rotary_frequencies(rot, base, factor, context)
        assert got.dtype == torch.float64 and np.abs(got.numpy() - want).max(initial=0) <= 1e-14


@pytest.mark.parametrize("change,needle", [
    (dict(q=lambda x: x["q"].half()), "q must be"), (dict(q=lambda x: x["q"][0]), "dimensions"), (dict(k=lambda x: x["k"].float()), "k must be"),
    (dict(k=lambda x: x["k"][:3]), "shape mismatch"), (dict(positions=lambda x: x["positions"].long()), "positions must be"),
    (dict(positions=lambda x: x["positions"][:3]), "positions must be"), (dict(freq=lambda x: x["freq"].float()), "freq must be"),
    (dict(freq=lambda x: x["freq"].cpu()), "GPU tensor"), (dict(freq=lambda x: torch.cat([x["freq"]] * 2)), "rot=128"),
    (dict(out=lambda x: x["q"][:, :2]), "out must be"), (dict(out=lambda x: x["q"][:1].expand(4, 4, 64)), "on one another"),
    (dict(out=lambda x: x["k"].expand(4, 4, 64) if x["k"].shape[1] == 1 else torch.cat([x["k"]] * 2, 1)[:, :4].as_strided((4, 4, 64), (64, 64, 1))), "on one another"),
    (dict(k_out=lambda x: x["q"][:, :2]), "overlaps"), (dict(k=lambda x: None, k_out=lambda x: x["q"]), "go together"),
    (dict(q=lambda x: torch.cat([x["q"], x["q"][..., :1]], -1)[..., :64]), "multiples of 16"),
])
def test_refusals(change, needle):
    dev = device()
    x = dict(q=torch.zeros(4, 4, 64, dtype=BF16, device=dev), k=torch.zeros(4, 2, 64, dtype=BF16, device=dev),
             positions=torch.zeros(4, dtype=torch.int32, device=dev), freq=api.rotary_frequencies(64, device=dev))
    x.update({n: f(x) for n, f in change.items()})
    with pytest.raises((ValueError, N.NativeError), match=needle):
        api.rotary(x.pop("q"), x.pop("positions"), x.pop("freq"), **x)


def test_empty_calls():
    dev = device()
    e = lambda *s: torch.empty(*s, device=dev)
    i = torch.zeros(0, dtype=torch.int32, device=dev)
    a, b = api.rotary(e(0, 4, 64), i, api.rotary_frequencies(64, device=dev), k=e(0, 2, 64))
    assert a.shape == (0, 4, 64) and b.shape == (0, 2, 64)
    x = torch.ones(3, 2, 64, device=dev)
    assert torch.equal(api.rotary(x, torch.arange(3, device=dev).int(), api.rotary_frequencies(0, device=dev)), x)
