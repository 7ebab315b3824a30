"""GPU parity of token_sample with its definition in fp64: equal tokens, and
log-probabilities to half a step of fp32.

The weights and sums are 64-bit on both sides, so a token could differ only
where u lies within some 1e-12 of a border between two tokens."""
import numpy as np
import pytest
import torch

from oracle import paged
from paper_2106_04718_amd import _native as N
from paper_2106_04718_amd import api, workloads

from _gpu import device, say

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def dev_of(a):
    a = np.ascontiguousarray(a)
    if a.dtype == np.uint16:
        return torch.from_numpy(a.view(np.int16)).to(device()).view(BF16)
    return torch.from_numpy(a).to(device())


def check(x, u, what, **kw):
    R = x.shape[0]
    u = np.asarray(u, np.float32)
    full = {n: np.broadcast_to(np.asarray(a, np.int32 if n == "top_k" else np.float32), (R,)).copy()
            for n, a in kw.items() if a is not None}
    say(f"[sample] {what}: {x.shape} {x.dtype} { {n: a[:4].tolist() for n, a in full.items()} }")
    tok, lp = api.token_sample(dev_of(x), dev_of(u), **{n: dev_of(a) for n, a in full.items()})
    torch.cuda.synchronize()
    tok, lp = tok.cpu().numpy(), lp.cpu().numpy().astype(np.float64)
    wt, wl = paged.token_sample(x, u, **full)
    assert np.array_equal(tok, wt), f"{what}: rows {np.flatnonzero(tok != wt)[:5]}: {tok[tok != wt][:5]}, want {wt[tok != wt][:5]}"
    ok = np.isnan(wl)
    assert np.array_equal(np.isnan(lp), ok), what
    # the fp32 rounding of the result, and 64-bit sums of up to V terms
    assert (np.abs(lp - wl)[~ok] <= 2.0 ** -24 * np.abs(wl[~ok]) + 1e-11).all(), what
    return tok, lp


def logits(seed, R, V, sd=2.0, dtype=F32, bans=0.02):
    rng = np.random.default_rng(seed)
    x = (rng.standard_normal((R, V)) * sd).astype(np.float32)
    if V > 8:
        x[np.arange(R)[:, None], rng.integers(0, V, (R, 6))] += (rng.random((R, 6)) * 8).astype(np.float32)
        x[rng.random((R, V)) < bans] = -np.inf
    x[:, rng.integers(0, V)] = 1.0
    return workloads.f32_to_bf16_bits(x) if dtype == BF16 else x, rng.random(R).astype(np.float32)


MODES = {
    "plain": {}, "T": dict(temperature=0.7), "hot": dict(temperature=3.0), "cold": dict(temperature=0.01),
    "k1": dict(top_k=1), "k50": dict(top_k=50), "k700": dict(top_k=700), "k3000": dict(top_k=2900, temperature=1.5),
    "p9": dict(top_p=0.9), "p5": dict(top_p=0.5, temperature=2.0), "p1e-6": dict(top_p=1e-6), "p0": dict(top_p=0.0),
    "p999": dict(top_p=0.9999, temperature=1.4), "m": dict(min_p=0.05), "m1": dict(min_p=1.0), "m0": dict(min_p=1e-6),
    "kp": dict(top_k=40, top_p=0.9), "kpm": dict(top_k=100, top_p=0.95, min_p=0.02, temperature=0.9),
    "pm": dict(top_p=0.99, min_p=0.01, temperature=1.7), "all off": dict(top_k=0, top_p=1.0, min_p=0.0, temperature=1.0),
    "greedy": dict(temperature=0.0, top_k=5, top_p=0.5),
}


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("mode", MODES)
def test_modes(mode, dtype):
    x, u = logits(len(mode), 24, 5003, dtype=dtype)
    check(x, u, mode, **MODES[mode])


@pytest.mark.parametrize("V", [1, 2, 3, 5, 63, 64, 65, 127, 255, 1000, 1023, 1024, 1025, 2047, 4096, 4099, 16385, 32128])
def test_vocabulary_sizes(V):
    for n, (mode, kw) in enumerate(MODES.items()):
        if n % 3 == V % 3:
            x, u = logits(V + n, 3, V, dtype=BF16 if n % 2 else F32)
            check(x, u, f"V={V} {mode}", **kw)


@pytest.mark.parametrize("V,R", [(50257, 9), (50264, 4), (65536, 2), (65537, 2), (131072, 3), (151936, 2), (262147, 1)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_large_vocabularies(V, R, dtype):
    for mode in ("T", "k50", "p9", "p5", "kpm", "m", "k3000", "greedy"):
        x, u = logits(V + len(mode), R, V, dtype=dtype)
        check(x, u, f"V={V} {mode}", **MODES[mode])


def test_every_row_has_its_own_settings():
    rng = np.random.default_rng(3)
    R = 300
    x, u = logits(4, R, 2501)
    check(x, u, "mixed", temperature=rng.choice([0, 0.5, 1, 2, -1, np.nan, np.inf], R),
          top_k=rng.choice([-3, 0, 1, 7, 400, 2501, 2**31 - 1], R), top_p=rng.choice([0, 0.3, 0.95, 1, 1.5, np.nan, -1], R),
          min_p=rng.choice([0, 0.1, 1, 2, np.nan, -1], R))


@pytest.mark.parametrize("R,V", [(32, 40001), (33, 40001), (7, 32769), (7, 32768), (3, 36864), (2, 36865), (32, 131072)])
def test_each_row_its_settings_around_the_sizes_where_the_kernels_change(R, V):
    """Up to 32 rows of more than 32768 logits go through kernels with a workgroup per
    slice of 4096, others through a workgroup per row."""
    rng = np.random.default_rng(R + V)
    x, u = logits(V - R, R, V, dtype=BF16 if V % 2 else F32)
    if R > 3:
        x = x.copy()
        x[1], x[2, V - 1] = (workloads.BF16_NAN if x.dtype == np.uint16 else np.nan), x[2, 0]
        x[3] = 0                                    # a row of one value: given up by the slices
        x[0, 4096:] = x[0, 4096]                    # all but a slice equal
    kw = dict(temperature=rng.choice([0, 0.5, 0.8, 1, 2, -1, np.inf], R), top_k=rng.choice([0, 1, 7, 60, 190, 200, 1500, V], R),
              top_p=rng.choice([0, 0.3, 0.9, 0.95, 1, 1.5], R), min_p=rng.choice([0, 0, 0.1, 1], R))
    check(x, u, "mixed", **kw)
    for off in ("top_k", "top_p", "min_p", "temperature"):
        check(x, u, f"without {off}", **{n: a for n, a in kw.items() if n != off})
    check(x, u, "top_p alone", top_p=kw["top_p"])
    check(x, u, "min_p alone", min_p=kw["min_p"])


def test_slices_of_bans_alone_and_few_finite_logits():
    rng = np.random.default_rng(21)
    x = np.full((6, 50000), -np.inf, np.float32)
    for r, n in enumerate((1, 3, 40, 900, 5000, 30000)):
        x[r, rng.choice(50000, n, replace=False)] = rng.standard_normal(n).astype(np.float32)
    u = rng.random(6).astype(np.float32)
    for mode, kw in MODES.items():
        check(x, u, f"few finite, {mode}", **kw)


def test_candidates_of_every_slice_exceed_the_list():
    """Top-k of 190 over 32 slices: several thousand candidates, bounded once more."""
    x, u = logits(22, 2, 131072, sd=1.0)
    for k in (150, 190, 192, 193):
        check(x, u, f"k={k}", top_k=k)
        check(x, u, f"k={k}", top_k=k, top_p=0.8, min_p=0.02)


def test_many_rows():
    x, u = logits(5, 3000, 77)
    check(x, u, "3000 rows", top_k=9, top_p=0.9)


def test_u_at_its_ends_and_outside():
    x, _ = logits(6, 1, 4000)
    us = np.array([0.0, 2.0 ** -30, 1 - 2.0 ** -24, 1.0, 2.0, -1.0, np.nan, np.inf, -np.inf], np.float32)
    for kw in ({}, dict(top_k=30), dict(top_p=0.8), dict(min_p=0.1)):
        check(np.repeat(x, len(us), 0), us, "ends of u", **kw)


@pytest.mark.parametrize("V", [2, 100, 3001, 70000])
def test_equal_logits(V):
    """Whole rows of one value, and few different values: the cut falls inside
    equal logits, whose first indices are kept."""
    u = np.linspace(0, 0.999, 6).astype(np.float32)
    same = np.full((6, V), -3.5, np.float32)
    rng = np.random.default_rng(V)
    few = rng.choice(np.array([0, -0.0, -1, 2, -np.inf], np.float32), (6, V))
    few[:, 0] = 2
    low = np.full((6, V), np.finfo(np.float32).min, np.float32)
    for kw in ({}, dict(top_k=max(1, V // 3)), dict(top_p=0.37), dict(top_k=max(1, V // 2), top_p=0.61), dict(min_p=1.0), dict(temperature=0.0)):
        check(same, u, "one value", **kw)
        check(few, u, "few values", **kw)
        check(low, u, "the lowest value", **kw)


def test_values_that_crowd_a_few_floats():
    """Logits that differ in their last bits alone, and around zero."""
    rng = np.random.default_rng(8)
    base = np.float32(17.0)
    x = (base.view(np.int32) + rng.integers(0, 40, (8, 30000)).astype(np.int32)).view(np.float32)
    tiny = (rng.standard_normal((8, 30000)) * 1e-30).astype(np.float32)
    u = rng.random(8).astype(np.float32)
    for kw in ({}, dict(top_k=3000), dict(top_k=1), dict(top_p=0.4), dict(top_p=0.9, top_k=20000), dict(min_p=0.9999999)):
        check(x, u, "last bits", **kw)
        check(tiny, u, "around zero", **kw)


def test_far_values_and_a_wide_range():
    rng = np.random.default_rng(9)
    x = (rng.standard_normal((6, 5000)) * 1e30).astype(np.float32)
    u = rng.random(6).astype(np.float32)
    for kw in ({}, dict(top_k=10), dict(top_p=0.5), dict(temperature=1e30, top_p=0.9), dict(temperature=1e38), dict(temperature=1e-38)):
        check(x, u, "1e30", **kw)
    x = np.concatenate([np.full((6, 4000), -1e9, np.float32), logits(10, 6, 1000)[0]], 1)
    for kw in ({}, dict(top_k=500), dict(top_k=1500), dict(top_p=0.9), dict(min_p=0.01)):
        check(x, u, "masked by -1e9", **kw)


def test_rows_without_a_distribution_and_bans():
    x, u = logits(11, 8, 3003)
    x[0, 17] = np.nan
    x[1, 3002] = np.inf
    x[2] = -np.inf
    x[3] = -np.inf
    x[3, 2999] = -5      # one token left
    x[4, :-1] = np.nan
    x[5] = np.nan
    for kw in ({}, dict(top_k=4), dict(top_p=0.2), dict(min_p=0.3), dict(temperature=0.0)):
        tok, _ = check(x, u, "no distribution", **kw)
        assert tok[[0, 1, 2, 4, 5]].tolist() == [-1] * 5 and tok[3] == 2999
    x, u = logits(12, 64, 700, bans=0.97)
    for kw in ({}, dict(top_k=50), dict(top_p=0.9)):
        tok, _ = check(x, u, "mostly banned", **kw)
        assert np.isfinite(x[np.arange(64), tok]).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shift", [1, 2, 3])
def test_row_strides_and_alignment(dtype, shift):
    x, u = logits(13, 5, 1003, dtype=dtype)
    big = torch.full((5, 1203), float("nan"), dtype=dtype, device=device())
    view = big[:, shift:shift + 1003]
    view.copy_(dev_of(x))
    for kw in ({}, dict(top_k=20, top_p=0.9), dict(top_p=0.7)):
        full = {n: torch.full((5,), a, dtype=torch.int32 if n == "top_k" else F32, device=device()) for n, a in kw.items()}
        got = api.token_sample(view, dev_of(u), **full)
        want = api.token_sample(dev_of(x), dev_of(u), **full)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert np.array_equal(got[0].cpu().numpy(), paged.token_sample(x, u, **{n: t.cpu().numpy() for n, t in full.items()})[0])


def test_reused_workspace_and_repeated_calls():
    ws = api.new_workspace(max(api.token_sample_workspace_bytes(R, V, t) for R, V, t in ((1, 131072, F32), (40, 9001, BF16), (2, 60000, F32))), device())
    cases = [(logits(14, 1, 131072), dict(top_p=0.9)), (logits(15, 40, 9001, dtype=BF16), dict(top_k=50)),
             (logits(16, 1, 131072), {}), (logits(17, 2, 60000), dict(top_k=30))]
    for rep in range(3):
        for (x, u), kw in cases:
            full = {n: torch.full((len(u),), a, dtype=torch.int32 if n == "top_k" else F32, device=device()) for n, a in kw.items()}
            tok, _ = api.token_sample(dev_of(x), dev_of(u), workspace=ws, **full)
            torch.cuda.synchronize()
            assert np.array_equal(tok.cpu().numpy(), paged.token_sample(x, u, **{n: t.cpu().numpy() for n, t in full.items()})[0])


@pytest.mark.parametrize("change,needle", [
    (dict(logits=lambda x: x["logits"].half()), "float32 or bfloat16"), (dict(logits=lambda x: x["logits"].t()), "contiguous rows"),
    (dict(logits=lambda x: x["logits"].cpu()), "GPU tensor"), (dict(u=lambda x: x["u"].double()), "u must be"),
    (dict(u=lambda x: x["u"][:2]), "u must be"), (dict(top_k=lambda x: x["u"]), "top_k must be"),
    (dict(temperature=lambda x: 0.5), "temperature must be"), (dict(top_p=lambda x: x["u"].cpu()), "top_p must be"),
    (dict(out=lambda x: (x["u"], x["u"])), "out must be"), (dict(out=lambda x: (x["u"],)), "out must be"),
    (dict(out=lambda x: (x["u"].int(), x["u"])), "overlaps"), (dict(workspace=lambda x: x["u"][:1]), "workspace"),
])
def test_refusals_of_the_front_end(change, needle):
    dev = device()
    x = dict(logits=torch.zeros(3, 50, device=dev), u=torch.zeros(3, device=dev))
    x.update({n: f(x) for n, f in change.items()})
    with pytest.raises((ValueError, N.NativeError), match=needle):
        api.token_sample(x.pop("logits"), x.pop("u"), **x)
