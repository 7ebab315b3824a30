"""Prompts and drafts through a paged cache as the operators are used together: rows grow,
queries and keys are turned by their positions, keys and values appended and attended, then
tokens drafted, verified together and partly given back, and rows end and begin.

The decoder is a toy of fixed random weights.  Its every operator is checked against the fp64
forms on the inputs that the run has at that point, and the whole run against its capture into
a graph, its repetition and a run on another stream, bit for bit."""
import numpy as np
import pytest
import torch

from oracle import paged
from paper_2106_04718_amd import api

from _gpu import bits, device, say, to_f64

pytestmark = pytest.mark.gpu

R, LAYERS, HQ, HKV, D, PAGE, COLS, P, VOCAB, DRAFT = 4, 2, 8, 2, 64, 16, 12, 40, 311, 4
# lengths wanted by each call, rows that end among them; pages do not last for the last row of the third
STEPS = [[30, 5, 60, 0], [90, 5, 63, 41], [94, 0, 67, 180], [70, 150, 66, 43]]
FREQ = dict(rot=48, base=10000.0, factor=4.0, context=64)


def f(t):
    return t.float().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


class Decoder:
    def __init__(self, dtype=torch.bfloat16, interleaved=False):
        dev = device()
        g = torch.Generator(device=dev).manual_seed(6)
        r = lambda *s, sd=1.0: (torch.randn(*s, device=dev, generator=g) * sd).to(dtype)
        dm = HQ * D
        self.interleaved, self.check = interleaved, False
        self.embed = r(VOCAB, dm)
        self.qkv = [r(dm, (HQ + 2 * HKV) * D, sd=dm ** -0.5) for _ in range(LAYERS)]
        self.o = [r(dm, dm, sd=dm ** -0.5) for _ in range(LAYERS)]
        self.freq = api.rotary_frequencies(**FREQ, device=dev)
        i = lambda *s: torch.zeros(*s, dtype=torch.int32, device=dev)
        self.N = N = 256
        self.kv = [torch.zeros(2, P, HKV, PAGE, D, device=dev, dtype=dtype) for _ in range(LAYERS)]
        self.table, self.len, self.want, self.free, self.count = i(R, COLS), i(R), i(R), i(P), i(1)
        self.start, self.off, self.pos = i(R), i(R + 1), i(N)
        self.slots = torch.zeros(N, dtype=torch.int64, device=dev)
        self.ids = torch.randperm(P, device=dev, generator=g).int()
        self.tokens = torch.randint(0, VOCAB, (len(STEPS), N), device=dev, generator=g)
        self.now = torch.zeros(N, dtype=torch.int64, device=dev)
        self.out = torch.zeros(N, HQ, D, device=dev, dtype=dtype)
        self.x = torch.zeros(N, dm, device=dev, dtype=dtype)
        self.ws = api.new_workspace(api.paged_chunk_attn_workspace_bytes(N, R, HQ, HKV, PAGE, COLS, D, dtype), dev)
        self.ws2 = api.new_workspace(api.paged_resize_workspace_bytes(R, N), dev)

    def begin(self):
        self.table.fill_(-1), self.len.zero_(), self.free.copy_(self.ids), self.count.fill_(P)
        self.out.zero_()
        for c in self.kv:
            c.zero_()

    def step(self):
        """What self.want asks for, with the tokens self.now, padded to N."""
        if self.check:
            before = [f(x) for x in (self.table, self.len, self.want, self.free)] + [int(self.count)]
        api.paged_resize(self.table, self.len, self.want, self.free, self.count, PAGE, start=self.start, offsets=self.off,
                         positions=self.pos, slots=self.slots, workspace=self.ws2)
        if self.check:
            ref = paged.paged_resize(*before, PAGE, self.N)
            for x, y in (("table", self.table), ("kv_len", self.len), ("start", self.start), ("offsets", self.off),
                         ("positions", self.pos), ("slots", self.slots)):
                assert np.array_equal(f(y), ref[x]), x
            assert int(self.count) == ref["free_count"]
        self.x.copy_(self.embed[self.now])
        for c, w, o in zip(self.kv, self.qkv, self.o):
            q, k, v = (self.x @ w).view(self.N, HQ + 2 * HKV, D).split([HQ, HKV, HKV], 1)
            if self.check:
                q0, k0 = f(q), f(k)
            api.rotary(q, self.pos, self.freq, k=k, out=q, k_out=k, interleaved=self.interleaved)
            if self.check:
                half = 2.0 ** -8 if q.dtype == torch.bfloat16 else 2.0 ** -24
                for got, x in ((q, q0), (k, k0)):
                    ref = paged.rotary(x, f(self.pos), self.freq.cpu().numpy(), self.interleaved)
                    assert (np.abs(to_f64(got) - ref) <= half * np.abs(ref) + 2.0 ** -20 * np.abs(x).max()).all()
                cache = f(c)
            api.paged_append(c[0], c[1], k, v, self.table, self.start, self.off)
            if self.check:
                K, V = paged.paged_append(cache[0], cache[1], f(k), f(v), f(self.table), f(self.start), f(self.off))
                assert np.array_equal(f(c[0]), K) and np.array_equal(f(c[1]), V)
                # every slot says where its token's key went
                s = f(self.slots)
                assert np.array_equal(K.transpose(0, 2, 1, 3).reshape(-1, HKV, D)[s[s >= 0]], f(k)[s >= 0])
            api.paged_chunk_attn(q, c[0], c[1], self.table, self.len, self.off, out=self.out, workspace=self.ws)
            if self.check:
                ref, mean = paged.paged_chunk_attn(f(q), K, V, f(self.table), f(self.len), f(self.off))
                own = ~np.isnan(ref).all((1, 2))
                # a half step of the type, and fp32 sums and scores of some hundred terms
                assert (np.abs(to_f64(self.out) - ref) <= half * np.abs(ref) + 1e-4 * mean)[own].all()
                assert own.sum() == min(self.N, int(self.off[-1]))
            self.x += self.out.view(self.N, -1) @ o

    def run(self, steps=len(STEPS)):
        self.begin()
        for t in range(steps):
            self.want.copy_(torch.tensor(STEPS[t], dtype=torch.int32, device=self.x.device))
            self.now.copy_(self.tokens[t])
            self.step()
        return self.state()

    def state(self):
        torch.cuda.synchronize()
        kept = int(self.count)
        return [bits(x).copy() for x in (self.table, self.len, self.free[:kept], self.start, self.off, self.pos, self.x, *self.kv)]


def same(a, b):
    return all(np.array_equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype,interleaved", [(torch.bfloat16, False), (torch.float32, True)])
def test_every_operator_of_a_run_against_the_definitions(dtype, interleaved):
    say(f"[prompts] {dtype}")
    d = Decoder(dtype, interleaved)
    d.check = True
    first = d.run()
    assert f(d.len).tolist() == [70, 150, 66, 43] and f(d.pos).any()
    d.check = False
    assert same(d.run(), first), "the same run again"


def test_a_run_on_another_stream():
    d = Decoder()
    first = d.run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        second = d.run()
    torch.cuda.current_stream().wait_stream(s)
    assert same(first, second)


def test_two_runs_on_two_streams_at_once():
    a, b = Decoder(), Decoder()
    want = a.run()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for d, s in zip((a, b), streams):
        with torch.cuda.stream(s):
            d.begin()
    for t in range(len(STEPS)):
        for d, s in zip((a, b), streams):
            with torch.cuda.stream(s):
                d.want.copy_(torch.tensor(STEPS[t], dtype=torch.int32, device=device()))
                d.now.copy_(d.tokens[t])
                d.step()
    torch.cuda.synchronize()
    assert same(a.state(), want) and same(b.state(), want)


def test_one_captured_step_serves_every_step():
    """Lengths, tokens and pages are on the device, so a step captured once is every step."""
    d = Decoder()
    want = d.run()
    g = torch.cuda.CUDAGraph()
    say("[prompts] capture")
    with torch.cuda.graph(g):
        d.step()
    torch.cuda.synchronize()
    for rep in range(3):
        d.begin()
        for t in range(len(STEPS)):
            say(f"[prompts] replay {rep}, step {t}")
            d.want.copy_(torch.tensor(STEPS[t], dtype=torch.int32, device=device()))
            d.now.copy_(d.tokens[t])
            if (rep + t) % 3 == 1:
                d.step()      # eagerly, in the same workspaces
            else:
                g.replay()
        assert same(d.state(), want), f"replay {rep}"


def test_two_graphs_of_different_sizes_share_a_workspace():
    dev = device()
    g = torch.Generator(device=dev).manual_seed(9)
    r = lambda *s: torch.randn(*s, device=dev, generator=g).bfloat16()
    sets = []
    for new, length in (((5, 60, 1), 2500), ((3,), 6000)):
        rows, cols = len(new), -(-length // PAGE)
        off = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device=dev)
        sets.append(dict(q=r(sum(new), HQ, D), K=r(rows * cols, HKV, PAGE, D), V=r(rows * cols, HKV, PAGE, D),
                         table=torch.randperm(rows * cols, device=dev, generator=g).view(rows, cols).int(), off=off,
                         n=torch.full((rows,), length, dtype=torch.int32, device=dev), out=r(sum(new), HQ, D)))
    ws = api.new_workspace(max(api.paged_chunk_attn_workspace_bytes(len(s["q"]), len(s["n"]), HQ, HKV, PAGE, s["table"].shape[1], D)
                               for s in sets), dev)

    def call(s, w):
        api.paged_chunk_attn(s["q"], s["K"], s["V"], s["table"], s["n"], s["off"], out=s["out"], workspace=w)

    def result(s):
        torch.cuda.synchronize()
        return bits(s["out"]).copy()

    want = []
    for s in sets:
        call(s, torch.zeros_like(ws))
        want.append(result(s))
    graphs = []
    for s in sets:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            call(s, ws)
        graphs.append(gr)
    for rep in range(4):
        for i in (0, 1, 1, 0):
            sets[i]["out"].zero_()
            graphs[i].replay()
            assert np.array_equal(result(sets[i]), want[i]), f"graph {i}, replay {rep}"
            call(sets[1 - i], ws)
            assert np.array_equal(result(sets[1 - i]), want[1 - i])


def test_a_draft_verified_and_given_back_is_as_if_it_had_not_been():
    """Tokens verified together attend what one token at a time does, and giving the places of those
    not accepted back leaves the pages as they were."""
    d = Decoder()
    d.begin()
    dev = device()
    set_want = lambda *a: d.want.copy_(torch.tensor(a, dtype=torch.int32, device=dev))
    set_want(30, 5, 60, 17)
    d.now.copy_(d.tokens[0])
    d.step()
    before = [x.clone() for x in (d.table, d.free[:int(d.count)], d.count)]
    set_want(*(x + DRAFT for x in (30, 5, 60, 17)))
    d.now.copy_(d.tokens[1])
    d.step()
    q = torch.randn(R * DRAFT, HQ, D, device=dev).bfloat16()
    together = api.paged_chunk_attn(q, d.kv[0][0], d.kv[0][1], d.table, d.len, d.off)
    for i in range(DRAFT):
        one = api.paged_attn(q.view(R, DRAFT, HQ, D)[:, i], d.kv[0][0], d.kv[0][1], d.table, d.len - (DRAFT - 1 - i))
        # each within half a step of bf16 and the fp32 sums
        err = (one.double() - together.view(R, DRAFT, HQ, D)[:, i].double()).abs()
        assert (err <= 2.0 ** -7 * one.double().abs() + 1e-4 * d.kv[0][1].abs().max()).all()
    set_want(30, 5, 60, 17)
    api.paged_resize(d.table, d.len, d.want, d.free, d.count, PAGE)
    torch.cuda.synchronize()
    assert torch.equal(d.table, before[0]) and torch.equal(d.free[:int(d.count)], before[1]) and torch.equal(d.count, before[2])
