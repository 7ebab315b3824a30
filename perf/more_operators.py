"""The operators that take prompts and drafts through a paged cache, measured for
speed: cases, their inputs, one pass in a plain form and through the public entry
points, and what each pass cannot do without.

  resize  ``paged_resize``: rows of a paged cache grow and shrink.  Pages are taken
          from a list of free ones and given back, and every new token gets its
          position and its slot of the cache.
  rotary  ``rotary``: queries and keys turned by their positions, in half or
          interleaved pairs, all of the head or its first part, with frequencies
          scaled for long contexts.
  chunk   ``paged_chunk_attn``: causal attention of several new tokens per row over
          the pages of that row, with shared key-value heads.

Sizes are those of the workload configurations (BART and GPT2 shaped) and generic
ones around them.  Pages lie in random order, as an allocator leaves them; lengths
are spread evenly over their range.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
ESIZE = {"bf16": 2, "f32": 4}


def listed():
    big = dict(Hq=32, Hkv=8, D=128, dtype="bf16")
    return [
        # One interactive request whose beginning is cached: the new tokens of a
        # short question.  Latency.
        dict(name="chunk_short", kind="chunk", R=1, ones=0, lo=16, hi=16, c_lo=100, c_hi=100, page=16, **big),
        # A batch in which every request has four drafted tokens verified beside its last one.
        dict(name="chunk_draft", kind="chunk", R=32, ones=0, lo=5, hi=5, c_lo=200, c_hi=4096, page=16, **big),
        # One piece of a long prompt, the pieces before it cached.
        dict(name="chunk_piece", kind="chunk", R=1, ones=0, lo=512, hi=512, c_lo=7680, c_hi=7680, page=16, **big),
        # A server's step: one token of most requests, pieces of a few prompts among them.
        dict(name="chunk_mixed", kind="chunk", R=40, ones=36, lo=129, hi=512, c_lo=200, c_hi=4096, page=16, **big),
        # The prompts of a GPT2-shaped batch (12 heads x 64, every head its own keys), nothing cached.
        dict(name="chunk_gpt2", kind="chunk", R=32, ones=0, lo=1, hi=1164, c_lo=0, c_hi=0, page=32, Hq=12, Hkv=12, D=64,
             dtype="bf16"),
        # A large piece late in a long document: the largest call.
        dict(name="chunk_long", kind="chunk", R=1, ones=0, lo=2048, hi=2048, c_lo=30500, c_hi=30500, page=64, **big),
        # BART-large-shaped heads in single precision, as an accuracy run uses them.
        dict(name="chunk_f32", kind="chunk", R=8, ones=0, lo=1, hi=257, c_lo=400, c_hi=1024, page=32, Hq=16, Hkv=16, D=64,
             dtype="f32"),
        # One token of every request of a large batch.
        dict(name="rotary_step", kind="rotary", N=256, rot=128, inter=False, far=4096, factor=1.0, **big),
        # The tokens of a batch of prompts late in long contexts, frequencies scaled for these.
        dict(name="rotary_prompt", kind="rotary", N=16384, rot=128, inter=False, far=1 << 20, factor=8.0, **big),
        # Interleaved pairs in the first half of the head, in single precision.
        dict(name="rotary_part", kind="rotary", N=5001, Hq=16, Hkv=16, D=64, rot=32, inter=True, far=8192, factor=1.0,
             dtype="f32"),
        # Every request of a batch reserves places for drafted tokens, and gives back those not accepted.
        dict(name="resize_step", kind="resize", R=256, page=16, lo=200, hi=4096, a_lo=1, a_hi=8, done=0, spare=600),
        # A large batch in which a quarter of the rows ends, the others take prompts, and new rows take
        # the ended ones' place.
        dict(name="resize_rows", kind="resize", R=1500, page=16, lo=1, hi=1500, a_lo=1, a_hi=400, done=4, spare=50000),
    ]


MAX_FLOPS = 4 * 2048 * 31524 * 32 * 128   # of the longest listed call
MAX_SCORES = 40 * 32 * 512 * 4608          # scores of a listed plain pass, all rows as long as the longest


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["chunk", "chunk", "chunk", "rotary", "rotary", "resize"])
    if kind == "resize":
        R, hi = _log_int(rng, 1, 1500), _log_int(rng, 1, 4096)
        a_hi = _log_int(rng, 1, 400)
        return dict(kind=kind, R=R, page=rng.choice([1, 16, 16, 32, 64, 100]), lo=1, hi=hi, a_lo=rng.choice([0, 1]), a_hi=a_hi,
                    done=rng.choice([0, 2, 4, 7]), spare=_log_int(rng, 1, 50000))
    Hkv, G = rng.choice([(1, 16), (2, 8), (4, 8), (8, 4), (8, 8), (4, 3), (8, 5), (12, 1), (16, 1), (16, 2)])
    D, dtype = rng.choice([64, 128, 128]), rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind == "rotary":
        N = min(_log_int(rng, 1, 16384), 16384 * 40 * 128 * 2 // ((G + 1) * Hkv * D * ESIZE[dtype]))
        rot = rng.choice([D, D, D, D // 2, D // 4, 20, 6])
        return dict(kind=kind, N=N, Hq=Hkv * G, Hkv=Hkv, D=D, rot=rot, inter=rng.random() < 0.4, far=_log_int(rng, 64, 1 << 20),
                    factor=rng.choice([1.0, 1.0, 2.0, 8.0]), dtype=dtype)
    hi = _log_int(rng, 1, 2048)
    c_hi = rng.choice([0, _log_int(rng, 1, 30500), _log_int(rng, 1, 30500)])
    c = dict(kind=kind, R=_log_int(rng, 1, 128), ones=0, lo=rng.choice([1, max(1, hi // 3), hi]), hi=hi,
             c_lo=rng.choice([0, c_hi // 2, c_hi]), c_hi=c_hi, page=rng.choice([16, 16, 32, 64, 256]), Hq=Hkv * G, Hkv=Hkv, D=D,
             dtype=dtype)
    few = 8 if dtype == "f32" else 1   # single precision goes at an eighth of the rate
    while c["R"] > 1 and (work(c)["flops"] * few > MAX_FLOPS or c["R"] * c["Hq"] * hi * (hi + c_hi) > MAX_SCORES):
        c["R"] -= 1
    while work(c)["flops"] * few > MAX_FLOPS or c["Hq"] * c["hi"] * (c["hi"] + c_hi) > MAX_SCORES:
        c["hi"] = c["hi"] * 3 // 4
        c["lo"] = min(c["lo"], c["hi"])
    if rng.random() < 0.3:
        c["ones"] = rng.randint(0, c["R"] - 1)
    return c


# ---- inputs -------------------------------------------------------------------

def _spread(lo, hi, R):
    """Lengths spread evenly over [lo, hi], one per row (the middle for one row)."""
    if R == 1:
        return np.array([(lo + hi) // 2], np.int64)
    return lo + (np.arange(R, dtype=np.int64) * (hi - lo)) // max(1, R - 1)


def _chunk_lens(case):
    """New tokens and cached positions of each row, in an order that belongs to the case."""
    new = np.concatenate([np.ones(case["ones"], np.int64), _spread(case["lo"], case["hi"], case["R"] - case["ones"])])
    order = np.random.default_rng([case["R"], case["hi"]]).permutation(case["R"])
    return new, _spread(case["c_lo"], case["c_hi"], case["R"])[order]


def _resize_lens(case):
    """Positions held by each row, and the lengths wanted of it by the first of two calls."""
    held = _spread(case["lo"], case["hi"], case["R"])
    order = np.random.default_rng([case["R"], case["hi"], 1]).permutation(case["R"])
    want = held + _spread(case["a_lo"], case["a_hi"], case["R"])[order]
    if case["done"]:
        want[::case["done"]] = 0
    return held, want


def _pages(lens, page, rng, spare=8, more=0):
    """A table of pages in random order for rows of these lengths, and the ids of the others."""
    need = -(-lens // page)
    ids = rng.permutation(int(need.sum()) + spare)
    table = np.full((len(lens), max(1, int(need.max()) + more)), -1, np.int32)
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = ids[at:at + n]
        at += n
    return table, ids[at:]


def _frequencies(case):
    """Turning speed of every pair in radians a position (fp64): base 10000, and with a factor the
    slow pairs' divided by it, the fast ones' kept, those between mixed."""
    i = np.arange(case["rot"] // 2, dtype=np.float64)
    f = 10000.0 ** (-2 * i / case["rot"])
    if case["factor"] == 1.0:
        return f
    turns = 4096 * f / (2 * math.pi)
    keep = np.clip((turns - 1) / (32 - 1), 0, 1)
    return f / case["factor"] * (1 - keep) + f * keep


def prepare(case, seed):
    rng = np.random.default_rng([seed & 0x7fffffff, 13])
    gen = torch.Generator(device=DEV).manual_seed(seed & 0x7fffffff)
    dev = lambda a, t=np.int32: torch.from_numpy(np.ascontiguousarray(a).astype(t)).to(DEV)
    st = {"case": case, "kind": case["kind"]}
    if case["kind"] == "resize":
        R, page = case["R"], case["page"]
        held, want = _resize_lens(case)
        more = np.maximum(-(-want // page) - -(-held // page), 0)
        table, free = _pages(held, page, rng, int(more.sum()) + case["spare"], int(more.max()))
        back = np.maximum(held - want, 0)
        N = int(max(np.maximum(want - held, 0).sum(), back.sum())) + 3   # both calls' tokens, padded
        P = int((-(-held // page)).sum()) + len(free)
        stack = np.zeros(P, np.int32)
        stack[:len(free)] = free
        out = lambda: dict(start=torch.empty(R, dtype=torch.int32, device=DEV),
                           offsets=torch.empty(R + 1, dtype=torch.int32, device=DEV),
                           positions=torch.empty(N, dtype=torch.int32, device=DEV),
                           slots=torch.empty(N, dtype=torch.int64, device=DEV))
        st.update(table=dev(table), kv_len=dev(held), want=dev(want), back=dev(held), free=dev(stack), count=dev([len(free)]),
                  first=out(), second=out())
        if own:
            from paper_2106_04718_amd import api
            st["workspace"] = api.new_workspace(api.paged_resize_workspace_bytes(R, N), DEV)
        return st
    dt = DT[case["dtype"]]
    normal = lambda *s: torch.randn(*s, device=DEV, dtype=dt, generator=gen)
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    if case["kind"] == "rotary":
        N = case["N"]
        q, k = normal(N, Hq, D), normal(N, Hkv, D)
        st.update(q=q, k=k, positions=dev(rng.integers(0, case["far"], N)), freq=dev(_frequencies(case), np.float64),
                  magnitude=0.1 * math.log(case["factor"]) + 1.0, out=(torch.empty_like(q), torch.empty_like(k)))
        return st
    new, cached = _chunk_lens(case)
    page, R, N = case["page"], case["R"], int(new.sum())
    table, free = _pages(new + cached, page, rng)
    P = int((-(-(new + cached) // page)).sum()) + len(free)
    q = normal(N, Hq, D)
    st.update(q=q, K=normal(P, Hkv, page, D), V=normal(P, Hkv, page, D), table=dev(np.maximum(table, 0)), kv_len=dev(new + cached),
              offsets=dev(np.concatenate([[0], np.cumsum(new)])), longest=int(new.max()), out=torch.empty_like(q))
    if own:
        from paper_2106_04718_amd import api
        st["workspace"] = api.new_workspace(
            api.paged_chunk_attn_workspace_bytes(N, R, Hq, Hkv, page, table.shape[1], D, dt), DEV)
    return st


# ---- one pass -----------------------------------------------------------------

def run(st):
    if own:
        return _run_own(st)
    return {"resize": _resize, "rotary": _rotary, "chunk": _chunk}[st["kind"]](st)


def _run_own(st):
    from paper_2106_04718_amd import api
    if st["kind"] == "resize":
        for want, o in ((st["want"], st["first"]), (st["back"], st["second"])):
            api.paged_resize(st["table"], st["kv_len"], want, st["free"], st["count"], st["case"]["page"], start=o["start"],
                             offsets=o["offsets"], positions=o["positions"], slots=o["slots"], workspace=st["workspace"])
        return _resize_outputs(st)
    if st["kind"] == "rotary":
        return api.rotary(st["q"], st["positions"], st["freq"], k=st["k"], interleaved=st["case"]["inter"],
                          magnitude=st["magnitude"], out=st["out"][0], k_out=st["out"][1])
    return api.paged_chunk_attn(st["q"], st["K"], st["V"], st["table"], st["kv_len"], st["offsets"], out=st["out"],
                                workspace=st["workspace"])


def _resize_outputs(st):
    """What both calls leave: the second takes the lengths back, and every page to where it was."""
    return st["table"], st["kv_len"], st["free"], st["count"], st["first"], st["second"]


def _resize(st):
    _resize_once(st, st["want"], st["first"])
    _resize_once(st, st["back"], st["second"])
    return _resize_outputs(st)


def _resize_once(st, want, o):
    table, page, P = st["table"].long(), st["case"]["page"], st["free"].shape[0]
    R, cols = table.shape
    held, want = st["kv_len"].long(), want.long()
    has, need = -(-held // page), -(-want // page)
    col = torch.arange(cols, device=DEV)
    # pages behind the rows' new ends go on the stack, the last row's last one first
    back = ((col >= need[:, None]) & (col < has[:, None])).view(-1)
    i = torch.cumsum(back, 0) - 1
    count = st["count"].long()
    at = torch.where(back, count + back.sum() - 1 - i, P)
    stack = torch.cat([st["free"], st["free"].new_zeros(1)])
    stack.scatter_(0, at, table.view(-1).int())
    count = count + back.sum()
    # rows that grow take from its end, in their order, as long as it lasts
    more = torch.where(want <= cols * page, (need - has).clamp(min=0), 0)
    run_sum = torch.cumsum(more, 0)
    ok = (want <= cols * page) & ((more == 0) | (run_sum <= count))
    take = (col >= has[:, None]) & (col < need[:, None]) & ok[:, None]
    j = (run_sum - more)[:, None] + col - has[:, None]
    table = torch.where(back.view(R, cols), -1, table)
    table = torch.where(take, stack[(count - 1 - j).clamp(0, P)].long(), table)
    st["free"].copy_(stack[:P])
    st["count"].copy_(count - (more * ok).sum())
    st["table"].copy_(table)
    st["kv_len"].copy_(torch.where(ok, want, held))
    o["start"].copy_(held)
    off = torch.cat([held.new_zeros(1), torch.cumsum((want - held).clamp(min=0), 0)])
    o["offsets"].copy_(off)
    n = torch.arange(o["slots"].shape[0], device=DEV)
    row = (torch.searchsorted(off, n, right=True) - 1).clamp(0, R - 1)
    pos = held[row] + n - off[row]
    live = n < off[-1]
    pg = table[row, (pos // page).clamp(0, cols - 1)]
    o["positions"].copy_(torch.where(live, pos, 0))
    o["slots"].copy_(torch.where(live & ok[row] & (pg >= 0), pg * page + pos % page, -1))


def _rotary(st):
    rot, inter = st["case"]["rot"], st["case"]["inter"]
    angle = st["positions"].double()[:, None] * st["freq"]
    c = (torch.cos(angle) * st["magnitude"]).float()[:, None]
    s = (torch.sin(angle) * st["magnitude"]).float()[:, None]
    x, o = torch.cat([st["q"], st["k"]], 1).float(), None
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if inter else (x[..., :rot // 2], x[..., rot // 2:rot])
    turned = a * c - b * s, b * c + a * s
    turned = torch.stack(turned, -1).flatten(2) if inter else torch.cat(turned, -1)
    o = torch.cat([turned, x[..., rot:]], -1)
    st["out"][0].copy_(o[:, :st["case"]["Hq"]])
    st["out"][1].copy_(o[:, st["case"]["Hq"]:])
    return st["out"]


def _chunk(st):
    c = st["case"]
    R, Hq, Hkv, D, T = c["R"], c["Hq"], c["Hkv"], c["D"], st["longest"]
    G = Hq // Hkv
    off, kv = st["offsets"].long(), st["kv_len"].long()
    n = off[1:] - off[:-1]
    # rows padded to the longest one's tokens
    t = torch.arange(T, device=DEV)
    index = (off[:-1, None] + t).clamp(max=st["q"].shape[0] - 1)
    rows = lambda C: C[st["table"].long()].permute(0, 2, 1, 3, 4).reshape(R, Hkv, -1, D).float()
    q = st["q"][index].float().view(R, T, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(R, Hkv, G * T, D)
    k = rows(st["K"])
    s = torch.matmul(q, k.transpose(2, 3)).div_(math.sqrt(D)).view(R, Hkv, G, T, -1)
    del k, q
    pos = (kv - n)[:, None] + t
    seen = torch.arange(s.shape[-1], device=DEV) <= pos[:, :, None]
    s.masked_fill_(~seen[:, None, None], -math.inf)
    s.sub_(s.amax(-1, keepdim=True)).exp_()
    total = s.sum(-1).view(R, Hkv, G * T, 1)
    o = torch.matmul(s.view(R, Hkv, G * T, -1), rows(st["V"])).div_(total)
    o = o.view(R, Hkv, G, T, D).permute(0, 3, 1, 2, 4).reshape(R * T, Hq, D)
    # every token's place among the padded ones
    i = torch.arange(st["q"].shape[0], device=DEV)
    row = torch.searchsorted(off, i, right=True) - 1
    st["out"].copy_(o[row * T + i - off[row]])
    return st["out"]


# ---- the same from the definitions, in 64 bits -----------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    return {"resize": _exact_resize, "rotary": _exact_rotary, "chunk": _exact_chunk}[case["kind"]](st)


def _exact_resize(st):
    """Whole numbers: the calls row by row and page by page."""
    page, table = st["case"]["page"], st["table"].cpu().numpy()
    cap = table.shape[1] * page
    kv = st["kv_len"].tolist()
    buffer, count = st["free"].tolist(), int(st["count"])
    outs = []
    for want, o in ((st["want"].tolist(), st["first"]), (st["back"].tolist(), st["second"])):
        N, start = len(o["slots"]), list(kv)
        off, pos, slot = [0], [0] * N, [-1] * N
        for r in reversed(range(len(kv))):
            for j in reversed(range(-(-want[r] // page), -(-kv[r] // page))):
                buffer[count] = int(table[r, j])
                count += 1
                table[r, j] = -1
        full = False
        for r, w in enumerate(want):
            has, need = -(-kv[r] // page), -(-w // page)
            given = w <= cap
            if given and need > has:
                full = full or need - has > count
                given = not full
                for j in range(has, need if given else has):
                    count -= 1
                    table[r, j] = buffer[count]
            for p in range(kv[r], w):
                pos[off[-1] + p - kv[r]] = p
                if given:
                    slot[off[-1] + p - kv[r]] = int(table[r, p // page]) * page + p % page
            off.append(off[-1] + max(0, w - kv[r]))
            kv[r] = w if given else kv[r]
        t = lambda a, ty=torch.int32: torch.tensor(a, dtype=ty, device=DEV)
        outs.append(dict(start=t(start), offsets=t(off), positions=t(pos), slots=t(slot, torch.int64)))
    return t(table), t(kv), t(buffer), t([count]), outs[0], outs[1]


def _exact_rotary(st):
    rot, inter = st["case"]["rot"], st["case"]["inter"]
    turn = torch.polar(torch.full_like(st["freq"], st["magnitude"]).expand(len(st["positions"]), -1).contiguous(),
                       torch.outer(st["positions"].double(), st["freq"]))[:, None]

    def of(x):
        x = x.double()
        pairs = x[..., :rot].unflatten(-1, (rot // 2, 2) if inter else (2, rot // 2))
        pairs = pairs if inter else pairs.transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        return torch.cat([(z if inter else z.transpose(-1, -2)).flatten(-2), x[..., rot:]], -1)

    return of(st["q"]), of(st["k"])


def _exact_chunk(st):
    c = st["case"]
    G, D, page = c["Hq"] // c["Hkv"], c["D"], c["page"]
    out = torch.zeros(st["q"].shape, device=DEV, dtype=torch.float64)
    off = st["offsets"].tolist()
    for r, L in enumerate(st["kv_len"].tolist()):
        pages = st["table"][r, :-(-L // page)].long()
        first = L - (off[r + 1] - off[r])
        for g in range(c["Hkv"]):
            k, v = (C[pages, g].reshape(-1, D)[:L].double() for C in (st["K"], st["V"]))
            for n0 in range(off[r], off[r + 1], 512):   # some tokens at a time
                n1 = min(off[r + 1], n0 + 512)
                q = st["q"][n0:n1, g * G:(g + 1) * G].double().transpose(0, 1)
                s = (q @ k.T) * D ** -0.5
                at = torch.arange(n0 - off[r] + first, n1 - off[r] + first, device=DEV)
                s = s.masked_fill(torch.arange(L, device=DEV) > at[:, None], -math.inf)
                out[n0:n1, g * G:(g + 1) * G] = (torch.softmax(s, -1) @ v).transpose(0, 1)
    return out


# ---- what a pass cannot do without -----------------------------------------------

def work(case):
    if case["kind"] == "resize":
        held, want = _resize_lens(case)
        page, tokens = case["page"], int(np.abs(want - held).sum())
        pages = int(np.abs(-(-want // page) - -(-held // page)).sum())
        # both calls: lengths read and written, the wanted ones, starts and offsets; a page moved there and
        # back; every token's position and slot
        return {"bytes": 2 * case["R"] * 20 + 2 * pages * 8 + tokens * 12, "flops": 0}
    e, D = ESIZE[case["dtype"]], case["D"]
    if case["kind"] == "rotary":
        heads = case["Hq"] + case["Hkv"]
        return {"bytes": case["N"] * (2 * heads * D * e + 4) + case["rot"] * 4, "flops": case["N"] * heads * case["rot"] * 3}
    new, cached = _chunk_lens(case)
    kv, page = new + cached, case["page"]
    seen = int((new * cached + new * (new + 1) // 2).sum())
    tables = 4 * int((-(-kv // page)).sum()) + 8 * case["R"]
    return {"bytes": 2 * int(kv.sum()) * case["Hkv"] * D * e + 2 * int(new.sum()) * case["Hq"] * D * e + tables,
            "flops": 4 * seen * case["Hq"] * D}
