"""GPU parity of paged_resize with the rules taken one page at a time: whole numbers,
the same bit for bit."""
import numpy as np
import pytest
import torch

from oracle import paged
from paper_2106_04718_amd import _native as N
from paper_2106_04718_amd import api

from _gpu import device, say

pytestmark = pytest.mark.gpu

I32, I64 = torch.int32, torch.int64


def state(seed, held, page, cols, spare):
    rng = np.random.default_rng(seed)
    held = np.asarray(held, np.int64)
    need = -(-held // page)
    P = int(need.sum()) + spare
    ids = rng.permutation(P).astype(np.int32)
    table = np.full((len(held), cols), -1, np.int32)
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = ids[at:at + n]
        at += n
    free = rng.integers(-9, P + 9, P).astype(np.int32)   # what lies behind the top does not matter
    free[:P - at] = ids[at:]
    return dict(table=table, kv_len=held.astype(np.int32), free_pages=free, free_count=P - at)


def dev_of(a, dtype=I32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(device(), dtype)


def call(d, want, page, n, workspace=None, outputs=("start", "offsets", "positions", "slots"), ld=0):
    R, cols = d["table"].shape
    wide = torch.full((R, cols + ld), 77, dtype=I32, device=device())
    wide[:, :cols] = dev_of(d["table"])
    t = dict(table=wide[:, :cols], kv_len=dev_of(d["kv_len"]), want=dev_of(want), free_pages=dev_of(d["free_pages"]),
             free_count=dev_of([d["free_count"]]))
    made = dict(start=torch.full((R,), 55, dtype=I32, device=device()), offsets=torch.full((R + 1,), 55, dtype=I32, device=device()),
                positions=torch.full((n,), 55, dtype=I32, device=device()), slots=torch.full((n,), 55, dtype=I64, device=device()))
    made = {x: made[x] for x in outputs}
    api.paged_resize(t["table"], t["kv_len"], t["want"], t["free_pages"], t["free_count"], page, workspace=workspace, **made)
    torch.cuda.synchronize()
    assert (wide[:, cols:] == 77).all()
    return {**t, **made}


def check(d, want, page, n, what, **kw):
    say(f"[resize] {what}: R={len(want)} page={page} N={n}")
    want = np.asarray(want, np.int64).astype(np.int32)
    got = call(d, want, page, n, **kw)
    ref = paged.paged_resize(d["table"], d["kv_len"], want, d["free_pages"], d["free_count"], page, n)
    for x, y in got.items():
        if x != "want":
            w = np.atleast_1d(np.asarray(ref[x]))
            g = y.cpu().numpy()
            if x == "free_pages":   # as far as it is kept
                g, w = g[:ref["free_count"]], w[:ref["free_count"]]
            assert np.array_equal(g, w), f"{what}: {x}"
    return dict(table=ref["table"], kv_len=ref["kv_len"], free_pages=got["free_pages"].cpu().numpy(), free_count=ref["free_count"])


@pytest.mark.parametrize("page", [1, 2, 3, 7, 16, 100])
@pytest.mark.parametrize("R", [1, 2, 63, 64, 65, 300, 1023, 1024, 1025, 3000])
def test_random_steps(page, R):
    """Rows grow, shrink, end and begin; in some steps the pages do not last."""
    rng = np.random.default_rng(R + page)
    cols = 12
    d = state(R, rng.integers(0, cols * page // 2 + 1, R), page, cols, 2 * R)
    for step in range(4):
        want = rng.integers(-2, cols * page + 2, R)
        same = rng.random(R) < 0.3
        want[same] = d["kv_len"][same]
        n = int(np.maximum(want - d["kv_len"], 0).sum())
        d = check(d, want, page, [n, n + 5, max(0, n - 3), 0][step], f"step {step}")


def test_growing_again_at_once_finds_the_same_pages():
    d = state(1, [40, 100, 7, 64], 16, 20, 30)
    more = [300, 100, 0, 90]
    a = check(d, more, 16, 400, "there")
    b = check(a, [40, 100, 7, 64], 16, 400, "and back")
    # the row that had ended takes the page that it gave back, and the free ones are as they were
    assert np.array_equal(b["table"], d["table"]) and b["free_count"] == d["free_count"]
    assert np.array_equal(b["free_pages"][:b["free_count"]], d["free_pages"][:d["free_count"]])


def test_pages_that_do_not_last():
    d = state(2, [16, 16, 16, 16, 16], 16, 10, 5)
    d = check(d, [48, 80, 16, 20, 33], 16, 200, "the second and those behind it get none")   # 2, 4, 0, 1, 2 of 5
    assert d["kv_len"].tolist() == [48, 16, 16, 16, 16] and d["free_count"] == 3
    d = check(d, [0, 200, 16, 32, 64], 16, 300, "a row past the table takes nothing from the others")
    assert d["kv_len"].tolist() == [0, 16, 16, 32, 64]
    check(d, [2**31 - 1] * 5, 16, 100, "far past the table, offsets at their end")


def test_states_that_an_earlier_mistake_left():
    d = state(3, [40, 30, 100], 16, 8, 6)
    d["table"][0, 1], d["table"][2, 5], d["table"][2, 6] = -1, 1000, -2**31   # not given back
    d = check(d, [3, 60, 10], 16, 60, "entries that name no page")
    d = state(4, [40, 30, 100], 16, 8, 6)
    d["kv_len"][:] = [-7, 2**31 - 1, 100]
    check(d, [20, 30, 2**31 - 1], 16, 60, "lengths outside the table")
    for count in (-3, 2**31 - 1):
        d = state(5, [40, 30], 16, 8, 6)
        d["free_count"] = count
        d["free_pages"] = np.arange(len(d["free_pages"]), dtype=np.int32)
        check(d, [90, 90], 16, 200, f"a count of {count}")
    d = state(6, [64, 64], 16, 8, 0)
    d["table"][1] = d["table"][0]             # pages of two rows, given back twice: no more than there are
    d["free_count"] = 5
    check(d, [0, 0], 16, 3, "given back twice")


def test_long_rows_and_large_calls():
    check(state(7, [0], 16, 9000, 9000), [140_000], 16, 140_000, "one long prompt")
    check(state(8, [140_000], 16, 9000, 10), [5], 16, 0, "which ends")
    rng = np.random.default_rng(9)
    held = rng.integers(0, 900, 5000)
    check(state(9, held, 16, 70, 200_000), held + rng.integers(0, 200, 5000), 16, 500_000, "5000 rows")


def test_a_table_of_almost_2_to_the_31_entries_returned_at_once():
    """Counts of returned pages step past 2^31 here."""
    cols = 715_827_882
    say(f"[resize] 3 rows of {cols} pages")
    dev = device()
    table = torch.full((3, cols), -1, dtype=I32, device=dev)
    table[0, 0], table[1, 400_000_000], table[2, cols - 1] = 5, 7, 3
    kv_len, free = torch.full((3,), cols, dtype=I32, device=dev), torch.full((8,), 9, dtype=I32, device=dev)
    count = torch.zeros(1, dtype=I32, device=dev)
    api.paged_resize(table, kv_len, torch.zeros(3, dtype=I32, device=dev), free, count, 1)
    assert not kv_len.any() and count.item() == 3
    assert free.tolist() == [3, 7, 5, 9, 9, 9, 9, 9]   # the last row's last page first
    assert all(bool((row == -1).all()) for row in table)


def test_outputs_that_are_not_asked_for_and_a_leading_dimension():
    d = state(10, [40, 0, 7], 16, 30, 60)
    for outputs in ((), ("start",), ("offsets", "slots"), ("positions",)):
        check(d, [400, 50, 0], 16, 500, f"only {outputs}", outputs=outputs, ld=5)
    ws = torch.randint(0, 255, (api.paged_resize_workspace_bytes(3, 500),), dtype=torch.uint8, device=device())
    for _ in range(2):   # whatever the workspace holds
        check(d, [400, 50, 0], 16, 500, "a used workspace", workspace=ws)


def test_no_rows():
    dev = device()
    z = lambda *s: torch.zeros(*s, dtype=I32, device=dev)
    pos, slots, off, count = z(5) + 9, torch.zeros(5, dtype=I64, device=dev), z(1) + 3, z(1) + 2
    api.paged_resize(z(0, 4), z(0), z(0), z(8), count, 16, offsets=off, positions=pos, slots=slots)
    assert not pos.any() and (slots == -1).all() and off.item() == 0 and count.item() == 2
    api.paged_resize(z(0, 4), z(0), z(0), z(8), count, 16)
    api.paged_resize(z(2, 0), z(2), z(2), z(0), count * 0, 16, positions=pos, slots=slots)   # no columns and no pages


def test_a_captured_call_replayed():
    dev = device()
    d = state(11, [40, 100, 7, 64], 16, 20, 60)
    t = {x: dev_of(np.atleast_1d(d[x])) for x in d}
    want, back = dev_of([300, 101, 0, 65]), dev_of(d["kv_len"])
    start, off, slots = (torch.zeros(n, dtype=ty, device=dev) for n, ty in ((4, I32), (5, I32), (300, I64)))
    ws = api.new_workspace(api.paged_resize_workspace_bytes(4, 300), dev)

    def step(w):
        api.paged_resize(t["table"], t["kv_len"], w, t["free_pages"], t["free_count"], 16, start=start, offsets=off, slots=slots, workspace=ws)

    step(want)
    torch.cuda.synchronize()
    first = [x.clone() for x in (t["table"], t["kv_len"], t["free_count"], start, off, slots)]
    step(back)
    g = torch.cuda.CUDAGraph()
    say("[resize] capture")
    with torch.cuda.graph(g):
        step(want)
    for rep in range(3):
        say(f"[resize] replay {rep}")
        g.replay()
        torch.cuda.synchronize()
        for x, y in zip((t["table"], t["kv_len"], t["free_count"], start, off, slots), first):
            assert torch.equal(x, y)
        step(back)


@pytest.mark.parametrize("change,needle", [
    (dict(table=lambda x: x["table"].long()), "table must be"), (dict(table=lambda x: x["table"].t()), "contiguous rows"),
    (dict(kv_len=lambda x: x["kv_len"][:2]), "kv_len must be"), (dict(want=lambda x: x["want"].long()), "want must be"),
    (dict(want=lambda x: x["want"].cpu()), "GPU tensor"), (dict(free_pages=lambda x: x["free_pages"].view(2, 4)), "free_pages must be"),
    (dict(free_count=lambda x: x["free_pages"][:2]), "free_count must be"), (dict(page=lambda x: 0), "page=0"),
    (dict(start=lambda x: x["want"]), "start overlaps want"), (dict(kv_len=lambda x: x["want"]), "kv_len overlaps want"),
    (dict(offsets=lambda x: x["want"].clone()), "offsets must be"), (dict(slots=lambda x: x["want"]), "slots must be"),
    (dict(positions=lambda x: torch.zeros(3, dtype=I32, device=x["want"].device), slots=lambda x: torch.zeros(4, dtype=I64, device=x["want"].device)), "slots must be"),
    (dict(workspace=lambda x: torch.zeros(8, dtype=torch.uint8, device=x["want"].device)), "workspace of 8 bytes"),
])
def test_refusals(change, needle):
    z = lambda *s: torch.zeros(*s, dtype=I32, device=device())
    x = dict(table=z(3, 4), kv_len=z(3), want=z(3), free_pages=z(8), free_count=z(1), page=16)
    x.update({n: f(x) for n, f in change.items()})
    with pytest.raises((ValueError, N.NativeError), match=needle):
        api.paged_resize(**x)
