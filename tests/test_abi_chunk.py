"""The entry points of growing rows, rotary positions and the attention of several new tokens
reject invalid arguments on the host, before any HIP call (the fake pointers are never
dereferenced)."""
import ctypes

import pytest

from paper_2106_04718_amd import _native as N
from test_abi_paged import BIG, CACHE, F, INVALID, UNSUPPORTED


def resize(**kw):
    a = dict(table=F, ld=4, cols=4, kv_len=2 * F, want=3 * F, R=3, page=16, free=4 * F, count=5 * F, P=9, start=6 * F,
             offsets=7 * F, positions=8 * F, slots=9 * F, N=5, ws=10 * F, ws_bytes=1 << 20)
    a.update(kw)
    return N.lib().fs_paged_resize(*a.values(), None)


def rotary(**kw):
    a = dict(q=F, qt=256, qh=64, k=2 * F, kt=128, kh=64, positions=3 * F, freq=4 * F, rot=64, inter=0, magnitude=1.0, qo=5 * F,
             qot=256, qoh=64, ko=6 * F, kot=128, koh=64, N=5, Hq=4, Hkv=2, D=64, dtype=N.FS_BF16)
    a.update(kw)
    return N.lib().fs_rotary(*a.values(), None)


def chunk(**kw):
    a = dict(q=F, qt=512, qh=64, K=BIG, V=2 * BIG, ps=2 * 16 * 64, hs=16 * 64, ss=64, P=9, page=16, table=3 * F, ld=4, cols=4,
             kv_len=4 * F, offsets=6 * F, scale=0.125, out=5 * F, N=7, R=3, Hq=8, Hkv=2, D=64, dtype=N.FS_BF16, ws=4 * BIG,
             ws_bytes=1 << 32)
    a.update(kw)
    return N.lib().fs_paged_chunk_attn(*a.values(), None)


def frequencies(**kw):
    out = (ctypes.c_double * 8)()
    a = dict(freq=ctypes.addressof(out), rot=16, base=1e4, factor=4.0, context=100, fast=32.0, slow=1.0)
    a.update(kw)
    return N.lib().fs_rotary_frequencies(*a.values())


@pytest.mark.parametrize("kw,status,needle", [
    (dict(R=-1), INVALID, "negative"), (dict(N=-1), INVALID, "negative"), (dict(cols=-1), INVALID, "negative"),
    (dict(P=-1), INVALID, "negative"), (dict(ld=-1), INVALID, "negative"), (dict(page=0), INVALID, "page=0"),
    (dict(ld=3), INVALID, "ld_table"), (dict(R=(1 << 20) + 1), UNSUPPORTED, "2^20"),
    (dict(page=1 << 20, cols=4096, ld=4096), UNSUPPORTED, "positions"), (dict(R=1 << 20, cols=2048, ld=2048, page=1), UNSUPPORTED, "a table"),
    (dict(table=None), INVALID, "null"), (dict(kv_len=None), INVALID, "null"), (dict(want=None), INVALID, "null"),
    (dict(free=None), INVALID, "null"), (dict(count=None), INVALID, "null"), (dict(ws=None), INVALID, "workspace"),
    (dict(ws_bytes=8), INVALID, "workspace"), (dict(ws=10 * F + 4), INVALID, "workspace must be 16"), (dict(table=F + 2), INVALID, "table must be 4"),
    (dict(slots=9 * F + 4), INVALID, "slots must be 8"), (dict(start=3 * F), INVALID, "start overlaps want"),
    (dict(kv_len=3 * F + 8), INVALID, "kv_len overlaps want"), (dict(free=F), INVALID, "free_pages overlaps table"),
    (dict(slots=8 * F), INVALID, "slots overlaps positions"), (dict(ws=2 * F), INVALID, "workspace overlaps kv_len"),
    (dict(count=4 * F + 8), INVALID, "free_count overlaps free_pages"),
])
def test_resize_rejects(kw, status, needle):
    assert resize(**kw) == status
    assert needle in N.last_error()


@pytest.mark.parametrize("kw,status,needle", [
    (dict(N=-1), INVALID, "negative"), (dict(Hq=-1), INVALID, "negative"), (dict(Hkv=-1), INVALID, "negative"),
    (dict(D=48), UNSUPPORTED, "D=48"), (dict(dtype=2), UNSUPPORTED, "dtype"), (dict(rot=63), INVALID, "rot=63"),
    (dict(rot=66), INVALID, "rot=66"), (dict(rot=-2), INVALID, "rot=-2"), (dict(inter=2), INVALID, "interleaved=2"),
    (dict(Hq=1 << 17), UNSUPPORTED, "2^17"),
    (dict(N=2**31 - 1, Hq=100, qt=6400, qot=6400), UNSUPPORTED, "too many tokens"), (dict(q=None), INVALID, "null"), (dict(k=None), INVALID, "null"),
    (dict(qo=None), INVALID, "null"), (dict(ko=None), INVALID, "null"), (dict(positions=None), INVALID, "null"),
    (dict(freq=None), INVALID, "null"), (dict(positions=3 * F + 2), INVALID, "aligned"), (dict(freq=4 * F + 4), INVALID, "aligned"),
    (dict(q=F + 8), INVALID, "16-byte"), (dict(ko=6 * F + 2), INVALID, "16-byte"), (dict(qt=260), INVALID, "multiples of 16"),
    (dict(koh=68), INVALID, "multiples of 16"), (dict(qt=-256), INVALID, "negative stride"), (dict(qt=1 << 62), UNSUPPORTED, "too large"),
    (dict(qot=0), INVALID, "on one another"), (dict(qoh=0), INVALID, "on one another"), (dict(qoh=56), INVALID, "on one another"),
    (dict(qot=64, qoh=64), INVALID, "on one another"), (dict(qo=F + 16), INVALID, "overlaps"), (dict(qo=F, qot=512), INVALID, "overlaps"),
    (dict(qo=2 * F), INVALID, "overlaps"), (dict(ko=F), INVALID, "overlaps"), (dict(ko=5 * F), INVALID, "overlaps"),
    (dict(qo=3 * F), INVALID, "positions or freq"), (dict(ko=4 * F), INVALID, "positions or freq"),
    # cut from one projection, but into one another's rows
    (dict(qt=512, kt=512, q=F, k=F + 2 * 256, qo=F, qot=512, ko=F + 2 * 128, kot=512), INVALID, "overlaps"),
    (dict(qt=512, kt=512, q=F, k=F + 2 * 448, qo=F, qot=512, ko=F + 2 * 448, kot=512), INVALID, "overlaps"),
])
def test_rotary_rejects(kw, status, needle):
    assert rotary(**kw) == status
    assert needle in N.last_error()


@pytest.mark.parametrize("kw,status,needle", CACHE + [
    (dict(N=-1), INVALID, "negative"), (dict(Hq=-8), INVALID, "negative"), (dict(Hq=7), INVALID, "multiple of Hkv"),
    (dict(Hkv=0), INVALID, "multiple of Hkv"), (dict(N=1 << 26), UNSUPPORTED, "2^28"), (dict(R=(1 << 24) + 1), UNSUPPORTED, "2^24"),
    (dict(q=None), INVALID, "null"), (dict(out=None), INVALID, "null"), (dict(kv_len=None), INVALID, "null"),
    (dict(offsets=None), INVALID, "null"), (dict(q=F + 8), INVALID, "aligned"), (dict(out=5 * F + 8), INVALID, "aligned"),
    (dict(kv_len=4 * F + 1), INVALID, "aligned"), (dict(offsets=6 * F + 2), INVALID, "aligned"), (dict(qt=516), INVALID, "multiples of 16"),
    (dict(qh=-64), INVALID, "negative stride"), (dict(qt=1 << 62), UNSUPPORTED, "too large"), (dict(scale=float("inf")), INVALID, "scale"),
    (dict(scale=float("nan")), INVALID, "scale"), (dict(scale=3e38), INVALID, "scale"), (dict(out=F), INVALID, "out overlaps"),
    (dict(out=BIG), INVALID, "out overlaps"), (dict(out=4 * F), INVALID, "out overlaps"), (dict(out=6 * F), INVALID, "out overlaps"),
    (dict(ws=None), INVALID, "workspace"), (dict(ws_bytes=8), INVALID, "workspace"), (dict(ws=4 * BIG + 4), INVALID, "aligned"),
    (dict(ws=BIG), INVALID, "workspace overlaps"), (dict(ws=5 * F), INVALID, "workspace overlaps"),
])
def test_chunk_attn_rejects(kw, status, needle):
    assert chunk(**kw) == status
    assert needle in N.last_error()


@pytest.mark.parametrize("kw,needle", [
    (dict(rot=15), "rot=15"), (dict(rot=-2), "rot=-2"), (dict(base=0.0), "base"), (dict(base=float("inf")), "base"),
    (dict(factor=-1.0), "factor"), (dict(factor=float("nan")), "factor"), (dict(context=-1), "context"), (dict(fast=1.0), "fast"),
    (dict(slow=-1.0), "slow"), (dict(fast=float("nan")), "fast"), (dict(freq=None), "null"),
])
def test_frequencies_reject(kw, needle):
    assert frequencies(**kw) == INVALID
    assert needle in N.last_error()


def test_a_cache_that_is_read_alone_may_be_expanded():
    """These get as far as the workspace, which is missing."""
    for change in (dict(V=BIG), dict(ps=0), dict(hs=0), dict(ss=0)):
        assert chunk(ws=None, **change) == INVALID and "workspace" in N.last_error(), change


def test_empty_calls_return_ok_without_launch():
    none = dict(K=None, V=None, table=None)
    assert chunk(N=0, q=None, ws=None, **none) == N.FS_OK and chunk(R=0, ws=None, **none) == N.FS_OK
    assert chunk(Hq=0, ws=None, **none) == N.FS_OK
    assert rotary(N=0, q=None, freq=None) == N.FS_OK and rotary(Hq=0, Hkv=0, q=None, k=None) == N.FS_OK
    assert resize(R=0, N=0, table=None, ws=None) == N.FS_OK
    assert frequencies(rot=0, freq=None) == N.FS_OK
    assert N.last_error() == ""


def test_workspace_queries():
    f, g = N.lib().fs_paged_chunk_attn_workspace_bytes, N.lib().fs_paged_resize_workspace_bytes
    bad = 2**64 - 1
    for x in (f(0, 3, 8, 2, 16, 4, 64, N.FS_BF16), f(3, 0, 8, 2, 16, 4, 64, N.FS_BF16), f(3, 3, 0, 2, 16, 4, 64, N.FS_BF16), g(0, 0)):
        assert x == 0
    assert 0 < f(3, 3, 8, 2, 16, 4, 64, N.FS_BF16) < bad and 0 < g(3, 100) < bad and 0 < g(0, 5) < bad
    for call in (f(3, 3, 7, 2, 16, 4, 64, N.FS_BF16), f(3, 3, 8, 2, 0, 4, 64, N.FS_BF16), f(3, 3, 8, 2, 16, 4, 65, N.FS_BF16),
                 f(3, 3, 8, 2, 1 << 20, 4096, 64, N.FS_BF16), f(-1, 3, 8, 2, 16, 4, 64, N.FS_F32), g(-1, 5), g((1 << 20) + 1, 5)):
        assert call == bad
