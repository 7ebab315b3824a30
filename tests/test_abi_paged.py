"""The paged cache's and the sampling's entry points reject invalid arguments on
the host, before any HIP call (the fake pointers are never dereferenced)."""
import pytest

from paper_2106_04718_amd import _native as N

F = 1 << 24
BIG = 1 << 40


def append(**kw):
    a = dict(K=BIG, V=2 * BIG, ps=2 * 16 * 64, hs=16 * 64, ss=64, P=9, page=16, k=F, v=2 * F, ts=128, ks=64, N=5,
             table=3 * F, ld=4, cols=4, start=4 * F, offsets=5 * F, R=3, Hkv=2, D=64, dtype=N.FS_BF16)
    a.update(kw)
    return N.lib().fs_paged_append(*a.values(), None)


def attn(**kw):
    a = dict(q=F, qr=512, qh=64, K=BIG, V=2 * BIG, ps=2 * 16 * 64, hs=16 * 64, ss=64, P=9, page=16, table=3 * F, ld=4,
             cols=4, kv_len=4 * F, k=None, v=None, ns=128, nh=64, scale=0.125, out=5 * F, R=3, Hq=8, Hkv=2, D=64,
             dtype=N.FS_BF16, ws=4 * BIG, ws_bytes=1 << 32)
    a.update(kw)
    return N.lib().fs_paged_attn(*a.values(), None)


def sample(**kw):
    a = dict(logits=F, ld=100, R=3, V=100, dtype=N.FS_F32, u=2 * F, T=3 * F, k=4 * F, p=5 * F, m=6 * F, tok=7 * F,
             lp=8 * F, ws=BIG, ws_bytes=1 << 32)
    a.update(kw)
    return N.lib().fs_token_sample(*a.values(), None)


INVALID, UNSUPPORTED = N.FS_ERR_INVALID_ARG, N.FS_ERR_UNSUPPORTED
CACHE = [
    (dict(R=-1), INVALID, "negative"), (dict(Hkv=-2), INVALID, "negative"), (dict(P=-1), INVALID, "negative"),
    (dict(cols=-1), INVALID, "negative"), (dict(P=0), INVALID, "P=0"), (dict(page=0), INVALID, "page=0"),
    (dict(ld=3), INVALID, "ld_table"), (dict(D=48), UNSUPPORTED, "D=48"), (dict(dtype=2), UNSUPPORTED, "dtype"),
    (dict(K=None), INVALID, "null"), (dict(V=None), INVALID, "null"), (dict(table=None), INVALID, "null"),
    (dict(K=BIG + 8), INVALID, "aligned"), (dict(table=3 * F + 2), INVALID, "aligned"),
    (dict(ss=68), INVALID, "multiples of 16"), (dict(hs=1028), INVALID, "multiples of 16"),
    (dict(ps=2052), INVALID, "multiples of 16"), (dict(ps=-2048), INVALID, "negative stride"),
    (dict(P=1 << 30, ps=1 << 40), UNSUPPORTED, "64 GiB"), (dict(P=40_000_000), UNSUPPORTED, "64 GiB"),
    (dict(page=1 << 20, cols=4096, ld=4096, P=1), UNSUPPORTED, "positions"),
]


@pytest.mark.parametrize("kw,status,needle", CACHE + [
    (dict(N=-1), INVALID, "negative"), (dict(offsets=None), INVALID, "without offsets"), (dict(k=None), INVALID, "null"),
    (dict(v=None), INVALID, "null"), (dict(start=None), INVALID, "null"), (dict(k=F + 4), INVALID, "aligned"),
    (dict(offsets=5 * F + 1), INVALID, "aligned"), (dict(ts=132), INVALID, "multiples of 16"),
    (dict(ks=-64), INVALID, "negative stride"), (dict(k=BIG + 64), INVALID, "overlaps"),
    (dict(table=2 * BIG + 64), INVALID, "overlaps"), (dict(start=BIG), INVALID, "overlaps"),
    (dict(Hkv=1 << 22, hs=0), UNSUPPORTED, "heads"), (dict(N=2**31 - 1, Hkv=64, hs=64 * 16, ps=64 * 64 * 16), UNSUPPORTED, "too many tokens"),
])
def test_append_rejects(kw, status, needle):
    assert append(**kw) == status
    assert needle in N.last_error()


@pytest.mark.parametrize("kw,status,needle", CACHE + [
    (dict(Hq=-8), INVALID, "negative"), (dict(Hq=7), INVALID, "multiple of Hkv"), (dict(Hkv=0), INVALID, "multiple of Hkv"),
    (dict(R=1 << 22), UNSUPPORTED, "2^24"), (dict(q=None), INVALID, "null"), (dict(out=None), INVALID, "null"),
    (dict(kv_len=None), INVALID, "null"), (dict(k=7 * F), INVALID, "go together"), (dict(v=7 * F), INVALID, "go together"),
    (dict(q=F + 8), INVALID, "aligned"), (dict(k=7 * F, v=8 * F + 4), INVALID, "aligned"), (dict(kv_len=4 * F + 1), INVALID, "aligned"),
    (dict(qr=516), INVALID, "multiples of 16"), (dict(qh=-64), INVALID, "negative stride"),
    (dict(k=7 * F, v=8 * F, ns=130), INVALID, "multiples of 16"),
    (dict(scale=float("inf")), INVALID, "scale"), (dict(scale=float("nan")), INVALID, "scale"),
    (dict(out=F), INVALID, "out overlaps"), (dict(out=BIG), INVALID, "out overlaps"), (dict(out=4 * F), INVALID, "out overlaps"),
    (dict(k=BIG, v=8 * F), INVALID, "overlaps"), (dict(q=BIG, k=7 * F, v=8 * F), INVALID, "the cache overlaps"),
    (dict(ws=None), INVALID, "workspace"), (dict(ws_bytes=8), INVALID, "workspace"), (dict(ws=4 * BIG + 4), INVALID, "aligned"),
    (dict(ws=BIG), INVALID, "workspace overlaps"),
])
def test_attn_rejects(kw, status, needle):
    assert attn(**kw) == status
    assert needle in N.last_error()


@pytest.mark.parametrize("kw,status,needle", [
    (dict(R=-1), INVALID, "negative"), (dict(V=-3), INVALID, "negative"), (dict(V=0), INVALID, "V=0"),
    (dict(dtype=5), UNSUPPORTED, "dtype"), (dict(V=(1 << 24) + 1, ld=1 << 25), UNSUPPORTED, "2^24"),
    (dict(R=(1 << 20) + 1), UNSUPPORTED, "2^20"), (dict(ld=99), INVALID, "ld_logits"), (dict(ld=-1, R=1), INVALID, "ld_logits"),
    (dict(ld=1 << 50), UNSUPPORTED, "ld_logits"), (dict(logits=None), INVALID, "null"), (dict(u=None), INVALID, "null"),
    (dict(tok=None), INVALID, "null"), (dict(lp=None), INVALID, "null"), (dict(logits=F + 2), INVALID, "aligned"),
    (dict(logits=F + 1, dtype=N.FS_BF16), INVALID, "aligned"), (dict(p=5 * F + 2), INVALID, "aligned"),
    (dict(tok=7 * F + 1), INVALID, "aligned"), (dict(tok=F + 4), INVALID, "overlaps"), (dict(lp=2 * F), INVALID, "overlaps"),
    (dict(lp=7 * F + 8), INVALID, "outputs overlap"), (dict(ws=None), INVALID, "workspace"), (dict(ws_bytes=0), INVALID, "workspace"),
    (dict(ws=BIG + 8), INVALID, "aligned"), (dict(ws=F), INVALID, "workspace overlaps"), (dict(ws=7 * F), INVALID, "workspace overlaps"),
])
def test_sample_rejects(kw, status, needle):
    assert sample(**kw) == status
    assert needle in N.last_error()


def test_empty_calls_return_ok_without_launch():
    none = dict(K=None, V=None, table=None)
    assert append(N=0, k=None, v=None, **none) == N.FS_OK
    assert append(R=0, **none) == N.FS_OK and append(Hkv=0, **none) == N.FS_OK
    assert attn(R=0, ws=None, **none) == N.FS_OK and attn(Hq=0, ws=None, **none) == N.FS_OK
    assert sample(R=0, logits=None, ws=None) == N.FS_OK
    assert N.last_error() == ""


def test_workspace_queries():
    f, g = N.lib().fs_paged_attn_workspace_bytes, N.lib().fs_token_sample_workspace_bytes
    bad = 2**64 - 1
    assert f(0, 8, 2, 16, 4, 64, N.FS_BF16) == 0 and g(0, 100, N.FS_F32) == 0
    assert 0 < f(3, 8, 2, 16, 4, 64, N.FS_BF16) < bad and 0 < g(3, 100, N.FS_F32) < bad
    for call in (f(3, 7, 2, 16, 4, 64, N.FS_BF16), f(3, 8, 2, 0, 4, 64, N.FS_BF16), f(3, 8, 2, 16, 4, 65, N.FS_BF16),
                 f(3, 8, 2, 1 << 20, 4096, 64, N.FS_BF16), f(-1, 8, 2, 16, 4, 64, N.FS_F32), g(3, 0, N.FS_F32), g(3, 100, 7)):
        assert call == bad
