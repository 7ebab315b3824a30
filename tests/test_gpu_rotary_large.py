"""Rotary positions in calls of so many units that a lane has several, workgroups are numbered
along two dimensions and units past 2^31.

The sizes follow from the launch's rule, worked out here too, so that a case is known to reach
what it is meant for."""
import numpy as np
import pytest
import torch

from paper_2106_04718_amd import api

from _gpu import device, say

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
FEW, GRID_ROW = 1024 * 256, 1 << 20


def rule(N, H, D, rot, dtype, interleaved, in_place):
    """(units of a call, units of a workgroup, whether partners come from LDS)."""
    vec, pairs = (8 if dtype == BF16 else 4), rot // 2
    any_half = not interleaved and pairs % vec != 0
    whole = D // vec if any_half else D // (2 * vec)
    units = whole if any_half or not in_place else -(-pairs // vec)
    total = N * H * units
    batch = min((1 if total <= FEW else 2) * 256, H * units * (4096 // max(1, pairs) - 2))
    return total, batch, any_half


def want(x, pos, freq, rot, interleaved, magnitude):
    """In float64, and the length of every element's pair."""
    x = x.double()
    angle = pos.double()[:, None, None] * freq
    c, s = torch.cos(angle) * magnitude, torch.sin(angle) * magnitude
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    u, w, r = a * c - b * s, b * c + a * s, torch.hypot(a, b)
    join = (lambda y, z: torch.stack([y, z], -1).flatten(2)) if interleaved else (lambda y, z: torch.cat([y, z], -1))
    return torch.cat([join(u, w), x[..., rot:]], -1), torch.cat([join(r, r), torch.zeros_like(x[..., rot:])], -1)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D,rot,Hq,Hkv", [(64, 20, 12, 3), (128, 20, 8, 1), (128, 126, 5, 5), (64, 64, 32, 8), (32, 16, 7, 0), (16, 6, 40, 1), (128, 128, 3, 2)])
def test_several_units_a_lane(D, rot, Hq, Hkv, dtype, interleaved, in_place):
    dev = device()
    per = (Hq + Hkv) * (rule(1, 1, D, rot, dtype, interleaved, in_place)[0])
    N = 3 * FEW // per + 37
    N += N * per % 512 == 0           # the last workgroup's batch is not full
    total, batch, any_half = rule(N, Hq + Hkv, D, rot, dtype, interleaved, in_place)
    assert total > FEW and total % batch and any_half == (not interleaved and rot in (6, 20, 126))
    say(f"[rotary large] N={N} H={Hq}+{Hkv} D={D} rot={rot} {'pairs' if interleaved else 'halves'} {dtype} {'in place' if in_place else ''}")
    g = torch.Generator(device=dev).manual_seed(D + rot)
    x = torch.randn(N, Hq + Hkv, D, device=dev, generator=g).to(dtype)
    pos = torch.randint(-5000, 5000, (N,), device=dev, generator=g).int()
    freq, magnitude = api.rotary_frequencies(rot, device=dev), 1.25
    ref, pair = want(x, pos, freq, rot, interleaved, magnitude)
    q, k = x[:, :Hq], x[:, Hq:] if Hkv else None
    if in_place:
        api.rotary(q, pos, freq, k=k, out=q, k_out=k, interleaved=interleaved, magnitude=magnitude)
        got = x
    else:
        keep = x.clone()
        out = api.rotary(q, pos, freq, k=k, interleaved=interleaved, magnitude=magnitude)
        got = torch.cat(out, 1) if Hkv else out
        assert torch.equal(x, keep)
    torch.cuda.synchronize()
    # half a step of the type, and 10 steps of 2^-24 of the pair's length times the magnitude: the
    # angle (1), the series (4), the magnitude's product (1), two products and a sum (3), and the 64-bit sines'
    half = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
    err, tol = (got.double() - ref).abs(), half * ref.abs() + 10 * 2.0 ** -24 * magnitude * pair
    assert (err <= tol).all(), f"off by {float((err / tol.clamp(min=1e-300)).max())} of the bound"
    assert torch.equal(got[..., rot:].double(), ref[..., rot:])


@pytest.mark.parametrize("interleaved,D,rot", [(False, 16, 16), (True, 16, 16), (False, 32, 20)])
def test_workgroups_along_two_dimensions_and_units_past_2_to_the_31(interleaved, D, rot):
    """Quarter turns of whole numbers, in place: exact but for cosines of 0 to some steps of 64 bits."""
    dev, heads = device(), 1 << 16
    per = rule(1, heads, D, rot, BF16, interleaved, True)[0]
    N = (1 << 31) // per + 3
    total, batch, any_half = rule(N, heads, D, rot, BF16, interleaved, True)
    assert -(-total // batch) > GRID_ROW and total > 1 << 31 and any_half == (rot == 20)
    say(f"[rotary large] {N} tokens of {heads} heads of {D}, {total} units in {-(-total // batch)} workgroups")
    x = torch.empty(N, heads, D, dtype=BF16, device=dev)
    step = 256
    fill = lambda n0: ((torch.arange(n0, min(n0 + step, N), device=dev)[:, None, None] * 7 + torch.arange(heads, device=dev)[:, None] * 5
                        + torch.arange(D, device=dev) * 3) % 251 - 125).to(BF16)
    for n0 in range(0, N, step):
        x[n0:n0 + step] = fill(n0)
    pos = torch.arange(N, device=dev).int() % 4
    freq = torch.full((rot // 2,), torch.pi / 2, dtype=torch.float64, device=dev)
    api.rotary(x, pos, freq, out=x, interleaved=interleaved)
    torch.cuda.synchronize()
    c, s = torch.tensor([1, 0, -1, 0], device=dev), torch.tensor([0, 1, 0, -1], device=dev)
    for n0 in range(0, N, step):
        y, got = fill(n0).float(), x[n0:n0 + step].float()
        p = pos[n0:n0 + step].long()
        cc, ss = c[p].float()[:, None, None], s[p].float()[:, None, None]
        a, b = (y[..., 0:rot:2], y[..., 1:rot:2]) if interleaved else (y[..., :rot // 2], y[..., rot // 2:rot])
        u, w = (got[..., 0:rot:2], got[..., 1:rot:2]) if interleaved else (got[..., :rot // 2], got[..., rot // 2:rot])
        # 125 times a cosine of 0 to some steps of fp64
        assert float((u - (a * cc - b * ss)).abs().max()) <= 125 * 2.0 ** -48, n0
        assert float((w - (b * cc + a * ss)).abs().max()) <= 125 * 2.0 ** -48, n0
        assert torch.equal(got[..., rot:], y[..., rot:])
