"""The operators of sampled generation over a paged cache, measured for speed:
cases, their inputs, one pass in a plain form and through the public entry
points, and what each pass cannot do without.

  append  ``paged_append``: the keys and values of prompts, or of one token per
          row, into the pages that each row's table names.
  attn    ``paged_attn``: attention of one new token per row over the pages of
          that row, with shared key-value heads; with ``new`` the token's own
          key and value come in the same call and are written to the cache.
  sample  ``token_sample``: one token per row from its logits, by temperature,
          top-k, top-p and min-p, from given random numbers.

Sizes are those of the workload configurations (BART, T5, GPT2 and ProphetNet
shaped) and generic ones around them.  Pages lie in random order, as an
allocator leaves them; row lengths are spread evenly over [lo, hi].
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
ESIZE = {"bf16": 2, "f32": 4}


def listed():
    return [
        # One interactive request, 32 query heads on 8 key-value heads: latency,
        # and the row split over the whole chip.
        dict(name="attn_one", kind="attn", R=1, Hq=32, Hkv=8, D=128, page=16, lo=1500, hi=1500, dtype="bf16", new=True),
        # A serving batch of ragged conversations, each step writing its token.
        dict(name="attn_batch", kind="attn", R=64, Hq=32, Hkv=8, D=128, page=16, lo=200, hi=4096, dtype="bf16", new=True),
        # Few very long rows: the largest call.
        dict(name="attn_long", kind="attn", R=4, Hq=32, Hkv=8, D=128, page=64, lo=120000, hi=131072, dtype="bf16",
             new=False),
        # The GPT2-shaped decoder (12 heads x 64, every head its own keys).
        dict(name="attn_gpt2", kind="attn", R=128, Hq=12, Hkv=12, D=64, page=32, lo=1, hi=1164, dtype="bf16", new=True),
        # Many query heads on few key-value heads, pages larger than a short row.
        dict(name="attn_shared", kind="attn", R=40, Hq=64, Hkv=4, D=128, page=256, lo=33, hi=9001, dtype="bf16", new=False),
        # BART-large-shaped heads in single precision, as an accuracy run uses them.
        dict(name="attn_f32", kind="attn", R=32, Hq=16, Hkv=16, D=64, page=32, lo=400, hi=1024, dtype="f32", new=True),
        # One new token of every row of a large batch.
        dict(name="append_token", kind="append", R=256, Hkv=8, D=128, page=16, lo=1, hi=1, used=900, dtype="bf16"),
        # The prompts of a batch, ragged, some behind a cached beginning.
        dict(name="append_prompt", kind="append", R=24, Hkv=8, D=128, page=16, lo=1, hi=4001, used=130, dtype="bf16"),
        # One interactive request over a large vocabulary, nucleus sampling.
        dict(name="sample_one", kind="sample", R=1, V=131072, sd=2.0, T=0.8, k=0, p=0.9, m=0.0, mix=False, dtype="f32"),
        # The BART-shaped rows with the usual chat settings.
        dict(name="sample_bart", kind="sample", R=128, V=50264, sd=2.0, T=0.8, k=50, p=0.95, m=0.0, mix=False, dtype="f32"),
        # Rollouts: every row from the model's own distribution, GPT2's odd vocabulary.
        dict(name="sample_rollout", kind="sample", R=512, V=50257, sd=1.5, T=1.0, k=0, p=1.0, m=0.0, mix=False,
             dtype="bf16"),
        # A server's batch in which every request brings its own settings.
        dict(name="sample_mixed", kind="sample", R=256, V=151936, sd=2.0, T=0.8, k=64, p=0.9, m=0.05, mix=True,
             dtype="f32"),
    ]


MAX_KV_BYTES = 4 * 125536 * 8 * 128 * 2 * 2   # keys and values of the longest listed call
MAX_LOGITS = 256 * 151936


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "append", "sample", "sample"])
    if kind == "sample":
        V = rng.choice([30522, 32128, 50257, 50264, _log_int(rng, 1000, 160000), _log_int(rng, 1000, 160000)])
        R = min(_log_int(rng, 1, 512), MAX_LOGITS // V)
        return dict(kind=kind, R=R, V=V, sd=round(rng.uniform(1.0, 4.0), 3),
                    T=round(rng.uniform(0.5, 1.3), 3), k=rng.choice([0, 0, 1, 20, 50, 200, 1500]),
                    p=rng.choice([1.0, 1.0, 0.5, 0.9, 0.95, 0.99]), m=rng.choice([0.0, 0.0, 0.02, 0.1]),
                    mix=rng.random() < 0.4, dtype=rng.choice(["f32", "f32", "bf16"]))
    Hkv, G = rng.choice([(1, 16), (2, 8), (4, 8), (8, 4), (8, 8), (8, 3), (8, 5), (12, 1), (16, 1), (16, 2)])
    D = rng.choice([64, 128, 128])
    page = rng.choice([16, 16, 32, 64, 256])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    R = _log_int(rng, 1, 256)
    row = 2 * Hkv * D * ESIZE[dtype]
    if kind == "append":
        hi = 1 if rng.random() < 0.4 else _log_int(rng, 2, 4096)
        R = max(1, min(R, (256 << 20) // (row * hi)))
        return dict(kind=kind, R=R, Hkv=Hkv, D=D, page=page, lo=1, hi=hi, used=rng.randint(0, 1000), dtype=dtype)
    hi = _log_int(rng, 16, 32768)
    R = max(1, min(R, MAX_KV_BYTES // (row * hi)))
    return dict(kind=kind, R=R, Hq=Hkv * G, Hkv=Hkv, D=D, page=page, lo=rng.choice([1, max(1, hi // 4), hi]), hi=hi,
                dtype=dtype, new=rng.random() < 0.5)


# ---- inputs -------------------------------------------------------------------

def _spread(case):
    """Lengths spread evenly over [lo, hi], one per row (the middle for one row)."""
    lo, hi, R = case["lo"], case["hi"], case["R"]
    if R == 1:
        return np.array([(lo + hi) // 2], np.int64)
    return lo + (np.arange(R, dtype=np.int64) * (hi - lo)) // (R - 1)


def _pages(lens, page, rng):
    """A table of pages in random order for rows of these lengths, and the number of pages."""
    need = -(-lens // page)
    P = int(need.sum()) + 8
    ids = rng.permutation(P)
    table = np.zeros((len(lens), max(1, int(need.max()))), np.int32)
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = ids[at:at + n]
        at += n
    return table, P


def prepare(case, seed):
    rng = np.random.default_rng([seed & 0x7fffffff, 11])
    gen = torch.Generator(device=DEV).manual_seed(seed & 0x7fffffff)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
    R = case["R"]
    st = {"case": case, "kind": case["kind"]}
    if case["kind"] == "sample":
        V = case["V"]
        x = torch.randn(R, V, device=DEV, generator=gen) * case["sd"]
        # a step's few likely tokens stand above the rest, and some tokens are banned
        likely = torch.randint(0, V, (R, 64), device=DEV, generator=gen)
        x.scatter_add_(1, likely, 8 * torch.rand(R, 64, device=DEV, generator=gen))
        x.scatter_(1, torch.randint(0, V, (R, 5), device=DEV, generator=gen), -math.inf)
        st["logits"] = x.to(DT[case["dtype"]])
        st["u"] = torch.rand(R, device=DEV, generator=gen)
        k = np.full(R, case["k"], np.int32)
        p, m = np.full(R, case["p"], np.float32), np.full(R, case["m"], np.float32)
        T = np.full(R, case["T"], np.float32)
        if case["mix"]:
            on = rng.integers(0, 8, R)   # each request has its own settings on or off
            k, p, m = np.where(on & 1, k, 0), np.where(on & 2, p, 1.0), np.where(on & 4, m, 0.0)
            T = np.where(on == 7, 0.0, rng.uniform(0.5, 1.3, R))
        st.update(T=dev(T.astype(np.float32)), k=dev(k.astype(np.int32)), p=dev(p.astype(np.float32)),
                  m=dev(m.astype(np.float32)))
        st["out"] = (torch.empty(R, dtype=torch.int32, device=DEV), torch.empty(R, dtype=torch.float32, device=DEV))
        if own:
            from paper_2106_04718_amd import api
            st["workspace"] = api.new_workspace(api.token_sample_workspace_bytes(R, V, DT[case["dtype"]]), DEV)
        return st
    Hkv, D, page, dt = case["Hkv"], case["D"], case["page"], DT[case["dtype"]]
    normal = lambda *s: torch.randn(*s, device=DEV, dtype=dt, generator=gen)
    order = rng.permutation(R)
    lens = _spread(case)[order]
    if case["kind"] == "append":
        used = ((np.arange(R, dtype=np.int64) * 7919) % (case["used"] + 1))[order]   # tokens already cached
        table, P = _pages(used + lens, page, rng)
        st.update(start=dev(used.astype(np.int32)), offsets=dev(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)),
                  k=normal(int(lens.sum()), Hkv, D), v=normal(int(lens.sum()), Hkv, D))
    else:
        table, P = _pages(lens, page, rng)
        st.update(kv_len=dev(lens.astype(np.int32)), q=normal(R, case["Hq"], D),
                  out=torch.empty(R, case["Hq"], D, device=DEV, dtype=dt))
        if case["new"]:
            st.update(k=normal(R, Hkv, D), v=normal(R, Hkv, D))
        if own:
            from paper_2106_04718_amd import api
            st["workspace"] = api.new_workspace(
                api.paged_attn_workspace_bytes(R, case["Hq"], Hkv, page, table.shape[1], D, dt), DEV)
    st.update(K=normal(P, Hkv, page, D), V=normal(P, Hkv, page, D), table=dev(table))
    return st


# ---- one pass -----------------------------------------------------------------

def run(st):
    if own:
        return _run_own(st)
    return {"append": _append, "attn": _attn, "sample": _sample}[st["kind"]](st)


def _run_own(st):
    from paper_2106_04718_amd import api
    if st["kind"] == "append":
        api.paged_append(st["K"], st["V"], st["k"], st["v"], st["table"], st["start"], offsets=st["offsets"])
        return st["K"], st["V"]
    if st["kind"] == "attn":
        new = st["case"]["new"]
        api.paged_attn(st["q"], st["K"], st["V"], st["table"], st["kv_len"], out=st["out"], workspace=st["workspace"],
                       k=st["k"] if new else None, v=st["v"] if new else None)
        return (st["out"], st["K"], st["V"]) if new else st["out"]
    return api.token_sample(st["logits"], st["u"], temperature=st["T"], top_k=st["k"], top_p=st["p"], min_p=st["m"],
                            out=st["out"], workspace=st["workspace"])


def _put(st, row, pos, k, v):
    """k, v of tokens at positions `pos` of rows `row` into their pages."""
    page = st["case"]["page"]
    pg = st["table"][row, pos // page].long()
    st["K"][pg, :, pos % page] = k
    st["V"][pg, :, pos % page] = v


def _append(st):
    off = st["offsets"].long()
    n = torch.arange(st["k"].shape[0], device=DEV)
    row = torch.searchsorted(off, n, right=True) - 1
    _put(st, row, st["start"].long()[row] + n - off[row], st["k"], st["v"])
    return st["K"], st["V"]


def _attn(st):
    c = st["case"]
    R, Hq, Hkv, D, page = c["R"], c["Hq"], c["Hkv"], c["D"], c["page"]
    n = st["kv_len"].long()
    if c["new"]:
        _put(st, torch.arange(R, device=DEV), n - 1, st["k"], st["v"])
    rows = lambda C: C[st["table"].long()].permute(0, 2, 1, 3, 4).reshape(R, Hkv, -1, D).float()
    q = st["q"].float().view(R, Hkv, Hq // Hkv, D)
    k = rows(st["K"])
    s = torch.matmul(q, k.transpose(2, 3)) / math.sqrt(D)
    del k
    live = torch.arange(s.shape[-1], device=DEV) < n[:, None]
    s = s.masked_fill(~live[:, None, None], -math.inf)
    w = torch.exp(s - s.amax(-1, keepdim=True))
    o = torch.matmul(w, rows(st["V"])) / w.sum(-1, keepdim=True)
    st["out"].copy_(o.view(R, Hq, D))
    return (st["out"], st["K"], st["V"]) if c["new"] else st["out"]


def _sample(st):
    x, V = st["logits"].float(), st["case"]["V"]
    T, k, p, m = st["T"].double()[:, None], st["k"].long()[:, None], st["p"].double()[:, None], st["m"].double()[:, None]
    greedy = T == 0
    top, order = torch.sort(x, dim=1, descending=True, stable=True)
    d = top.double() - top[:, :1].double()
    w = torch.where(greedy, (d == 0).double(), torch.exp(d / torch.where(greedy, 1.0, T)))
    rank = torch.arange(V, device=DEV)
    w = torch.where((k <= 0) | (rank < k), w, 0.0)
    mass = torch.cumsum(w, 1)
    before = mass - w
    w = torch.where((before < p * mass[:, -1:]) | (p >= 1) | (rank == 0), w, 0.0)
    w = torch.where((w >= m) | (rank == 0), w, 0.0)
    w = torch.where(greedy & (rank > 0), 0.0, w)
    w = torch.zeros_like(w).scatter_(1, order, w)   # back into the order of the tokens
    run_sum = torch.cumsum(w, 1)
    total = run_sum[:, -1:]
    tok = ((run_sum > st["u"].double()[:, None] * total) & (w > 0)).double().argmax(1, keepdim=True)
    st["out"][0].copy_(tok[:, 0])
    st["out"][1].copy_(torch.log(w.gather(1, tok) / total)[:, 0])
    return st["out"]


# ---- the same from the definitions, in 64 bits -----------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    return {"append": _exact_append, "attn": _exact_attn, "sample": _exact_sample}[case["kind"]](st)


def _exact_append(st):
    page = st["case"]["page"]
    off, start, table = st["offsets"].tolist(), st["start"].tolist(), st["table"].tolist()
    K, V = st["K"].clone(), st["V"].clone()
    for r in range(st["case"]["R"]):
        i = 0
        while i < off[r + 1] - off[r]:   # one page at a time
            pos = start[r] + i
            n = min(page - pos % page, off[r + 1] - off[r] - i)
            for C, x in ((K, st["k"]), (V, st["v"])):
                C[table[r][pos // page], :, pos % page:pos % page + n] = x[off[r] + i:off[r] + i + n].transpose(0, 1)
            i += n
    return K, V


def _exact_attn(st):
    c = st["case"]
    G, D, page = c["Hq"] // c["Hkv"], c["D"], c["page"]
    out = torch.zeros(c["R"], c["Hq"], D, device=DEV, dtype=torch.float64)
    for r, n in enumerate(st["kv_len"].tolist()):
        pages = st["table"][r, :-(-n // page)].long()
        for h in range(c["Hkv"]):
            k, v = (C[pages, h].reshape(-1, D)[:n].double() for C in (st["K"], st["V"]))
            if c["new"]:
                k[n - 1], v[n - 1] = st["k"][r, h].double(), st["v"][r, h].double()
            s = (st["q"][r, h * G:(h + 1) * G].double() @ k.T) * D ** -0.5
            out[r, h * G:(h + 1) * G] = torch.softmax(s, -1) @ v
    return (out, None, None) if c["new"] else out


def _exact_sample(st):
    R = st["case"]["R"]
    tok, lp = torch.zeros(R, dtype=torch.int32, device=DEV), torch.zeros(R, dtype=torch.float64, device=DEV)
    x64, u = st["logits"].double(), st["u"].double()
    for r, (T, k, p, m) in enumerate(zip(st["T"].tolist(), st["k"].tolist(), st["p"].tolist(), st["m"].tolist())):
        x = x64[r]
        if T == 0:
            tok[r] = (x == x.max()).nonzero()[0, 0]
            continue
        order = torch.sort(x, descending=True, stable=True).indices
        w = torch.softmax(x / T, 0)
        if k > 0:
            order = order[:k]
        if p < 1:
            share = w[order] / w[order].sum()
            order = order[:max(1, int((torch.cumsum(share, 0) - share < p).sum()))]
        if m > 0:
            order = order[w[order] >= m * w[order[0]]]
        kept = torch.sort(order).values
        share = w[kept] / w[kept].sum()
        at = torch.searchsorted(torch.cumsum(share, 0), u[r], right=True).clamp(max=len(kept) - 1)
        tok[r], lp[r] = kept[at], torch.log(share[at])
    return tok, lp


# ---- what a pass cannot do without -----------------------------------------------

def work(case):
    R = case["R"]
    if case["kind"] == "sample":
        return {"bytes": R * (case["V"] * ESIZE[case["dtype"]] + 28), "flops": R * case["V"] * 2}
    e, lens = ESIZE[case["dtype"]], int(_spread(case).sum())
    rows = 2 * lens * case["Hkv"] * case["D"] * e
    if case["kind"] == "append":
        return {"bytes": 2 * rows + R * 8, "flops": 0}
    new = 2 * R * case["Hkv"] * case["D"] * e if case["new"] else 0
    tables = 4 * int((-(-_spread(case) // case["page"])).sum()) + 4 * R
    return {"bytes": rows + new + 2 * R * case["Hq"] * case["D"] * e + tables, "flops": 4 * lens * case["Hq"] * case["D"]}
