"""Sampled generation as its parts are used together: prompts appended to a paged
cache, then per token every layer's attention with the token's own key and value
written in passing, the n-gram bans on the logits and the draw of a token.

The decoder is a toy of fixed random weights.  Its every operator is checked
against the fp64 forms on the inputs that the run has at that point, and the
whole run against its capture into a graph, its repetition and a run on another
stream, bit for bit."""
import numpy as np
import pytest
import torch

import oracle
from oracle import paged
from paper_2106_04718_amd import api

from _gpu import bits, device, say, to_f64

pytestmark = pytest.mark.gpu

R, LAYERS, HQ, HKV, D, PAGE, COLS, VOCAB, N_GRAM = 5, 2, 8, 2, 64, 16, 6, 613, 3
PROMPTS = [3, 16, 41, 1, 30]


class Decoder:
    def __init__(self, dtype=torch.bfloat16):
        dev = device()
        g = torch.Generator(device=dev).manual_seed(5)
        r = lambda *s, sd=1.0: (torch.randn(*s, device=dev, generator=g) * sd).to(dtype)
        dm = HQ * D
        self.embed = r(VOCAB, dm)
        self.qkv = [r(dm, (HQ + 2 * HKV) * D, sd=dm ** -0.5) for _ in range(LAYERS)]
        self.o = [r(dm, dm, sd=dm ** -0.5) for _ in range(LAYERS)]
        self.head = r(dm, VOCAB, sd=3 * dm ** -0.5)
        P = R * COLS + 4
        self.kv = [torch.zeros(2, P, HKV, PAGE, D, device=dev, dtype=dtype) for _ in range(LAYERS)]
        self.table = torch.randperm(P, device=dev, generator=g)[:R * COLS].view(R, COLS).int()
        self.len = torch.zeros(R, dtype=torch.int32, device=dev)
        self.prompt = torch.randint(0, VOCAB, (sum(PROMPTS),), device=dev, generator=g)
        self.u = torch.rand(64, R, device=dev, generator=g)
        self.cold = torch.tensor([0.7, 1.0, 0.0, 1.3, 0.9], device=dev)
        self.k = torch.tensor([20, 0, 0, 5, 0], dtype=torch.int32, device=dev)
        self.p = torch.tensor([1.0, 0.9, 1.0, 0.8, 1.0], device=dev)
        self.m = torch.tensor([0.0, 0.0, 0.0, 0.0, 0.05], device=dev)
        # buffers of a step
        self.tokens = torch.zeros(R, 64, dtype=torch.int32, device=dev)
        self.last = torch.zeros(R, dtype=torch.int32, device=dev)
        self.logprob = torch.zeros(R, device=dev)
        self.draws = torch.zeros(R, device=dev)
        self.out = torch.empty(R, HQ, D, device=dev, dtype=dtype)
        self.logits = torch.empty(R, VOCAB, device=dev)
        self.ws = api.new_workspace(api.paged_attn_workspace_bytes(R, HQ, HKV, PAGE, COLS, D, dtype), dev)
        self.ws2 = api.new_workspace(api.token_sample_workspace_bytes(R, VOCAB), dev)
        self.check = False

    def start(self):
        """The prompts' keys and values (of their embeddings alone) into every layer's cache."""
        x = self.embed[self.prompt]
        off = torch.tensor(np.concatenate([[0], np.cumsum(PROMPTS)]), dtype=torch.int32, device=x.device)
        for c, w in zip(self.kv, self.qkv):
            c.zero_()
            _, k, v = (x @ w).view(-1, HQ + 2 * HKV, D).split([HQ, HKV, HKV], 1)
            before = c.clone() if self.check else None
            api.paged_append(c[0], c[1], k, v, self.table, torch.zeros_like(self.len), off)
            if self.check:
                f = lambda t: t.float().cpu().numpy()
                want = paged.paged_append(f(before[0]), f(before[1]), f(k), f(v), self.table.cpu().numpy(),
                                          np.zeros(R, np.int32), off.cpu().numpy())
                assert np.array_equal(f(c[0]), want[0]) and np.array_equal(f(c[1]), want[1])
        self.len.copy_(torch.tensor(PROMPTS, dtype=torch.int32, device=x.device))
        self.last.copy_(self.prompt[(off[1:] - 1).long()].int())
        self.tokens.zero_()

    def step(self, t):
        self.len += 1
        x = self.embed[self.last.long()]
        for c, w, o in zip(self.kv, self.qkv, self.o):
            q, k, v = (x @ w).view(R, HQ + 2 * HKV, D).split([HQ, HKV, HKV], 1)
            before = c.clone() if self.check else None
            api.paged_attn(q, c[0], c[1], self.table, self.len, out=self.out, workspace=self.ws, k=k, v=v)
            if self.check:
                f = lambda t: t.float().cpu().numpy()
                want, K, V = paged.paged_attn(f(q), f(before[0]), f(before[1]), self.table.cpu().numpy(),
                                              self.len.cpu().numpy(), f(k), f(v))
                assert np.array_equal(f(c[0]), K) and np.array_equal(f(c[1]), V)
                # a half step of bf16 and fp32 sums of some hundred terms
                assert (np.abs(to_f64(self.out) - want) <= 2.0 ** -8 * np.abs(want) + 1e-4 * np.abs(V).max()).all()
            x = x + self.out.view(R, -1) @ o
        self.logits.copy_(x.float() @ self.head.float())
        before = self.logits.cpu().numpy() if self.check else None
        api.ngram_block(self.tokens, N_GRAM, self.logits, t=t)
        api.token_sample(self.logits, self.draws, temperature=self.cold, top_k=self.k, top_p=self.p, min_p=self.m,
                         out=(self.last, self.logprob), workspace=self.ws2)
        if self.check:
            want = oracle.ngram_block(self.tokens.cpu().numpy()[:, :t], N_GRAM, before) if t >= N_GRAM else before
            tok, lp = paged.token_sample(want, self.draws.cpu().numpy(), *(x.cpu().numpy() for x in (self.cold, self.k, self.p, self.m)))
            assert np.array_equal(self.last.cpu().numpy(), tok)
            assert (np.abs(self.logprob.cpu().numpy() - lp) <= 2.0 ** -24 * np.abs(lp) + 1e-11).all()
        self.tokens[:, t] = self.last

    def run(self, steps):
        self.start()
        for t in range(steps):
            self.draws.copy_(self.u[t])
            self.step(t)
        return self.state()

    def state(self):
        torch.cuda.synchronize()
        return [bits(x).copy() for x in (self.tokens, self.logprob, self.out, *self.kv)]


def same(a, b):
    return all(np.array_equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_every_operator_of_a_run_against_the_definitions(dtype):
    say(f"[generate] {dtype}")
    d = Decoder(dtype)
    d.check = True
    first = d.run(20)
    assert first[0].max() > 0
    d.check = False
    assert same(d.run(20), first), "the same run again"


def test_a_run_on_another_stream():
    d = Decoder()
    first = d.run(12)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        second = d.run(12)
    torch.cuda.current_stream().wait_stream(s)
    assert same(first, second)


def test_two_generations_on_two_streams_at_once():
    a, b = Decoder(), Decoder()
    want = a.run(12)
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    for s in (sa, sb):
        s.wait_stream(torch.cuda.current_stream())
    for d, s in ((a, sa), (b, sb)):
        with torch.cuda.stream(s):
            d.start()
    for t in range(12):
        for d, s in ((a, sa), (b, sb)):
            with torch.cuda.stream(s):
                d.draws.copy_(d.u[t])
                d.step(t)
    torch.cuda.synchronize()
    assert same(a.state(), want) and same(b.state(), want)


def test_a_captured_step_replayed_with_eager_work_between():
    d = Decoder()
    want = d.run(14)
    T = 5    # a step whose place in the history is fixed: capture one, replay it as the others run eagerly
    d.start()
    for t in range(T):
        d.draws.copy_(d.u[t])
        d.step(t)
    torch.cuda.synchronize()
    keep = [x.clone() for x in (d.len, d.last, d.tokens, *d.kv)]
    g = torch.cuda.CUDAGraph()
    d.draws.copy_(d.u[T])
    say("[generate] capture")
    with torch.cuda.graph(g):
        d.step(T)
    torch.cuda.synchronize()
    for rep in range(4):
        say(f"[generate] replay {rep}")
        for x, y in zip((d.len, d.last, d.tokens, *d.kv), keep):
            x.copy_(y)
        d.draws.copy_(d.u[T])
        g.replay()
        for t in range(T + 1, 14):   # the rest eagerly, in the same workspaces
            d.draws.copy_(d.u[t])
            d.step(t)
        assert same(d.state(), want), f"replay {rep}"


def test_two_graphs_of_different_sizes_share_the_workspaces():
    """The attention of two batches and two draws, captured apart, replayed in turn
    with eager calls between: workspaces hold nothing of a call after it."""
    dev = device()
    g = torch.Generator(device=dev).manual_seed(9)
    r = lambda *s: torch.randn(*s, device=dev, generator=g)
    sets = []
    for rows, length, V in ((3, 2500, 40000), (1, 4000, 9000)):
        cols = -(-length // PAGE)
        P = rows * cols
        sets.append(dict(q=r(rows, HQ, D).bfloat16(), K=r(P, HKV, PAGE, D).bfloat16(), V=r(P, HKV, PAGE, D).bfloat16(),
                         table=torch.randperm(P, device=dev, generator=g).view(rows, cols).int(),
                         n=torch.full((rows,), length, dtype=torch.int32, device=dev), x=r(rows, V) * 2,
                         u=torch.rand(rows, device=dev, generator=g), p=torch.full((rows,), 0.9, device=dev),
                         out=torch.empty(rows, HQ, D, device=dev, dtype=torch.bfloat16),
                         tok=torch.zeros(rows, dtype=torch.int32, device=dev), lp=torch.zeros(rows, device=dev)))
    wa = api.new_workspace(max(api.paged_attn_workspace_bytes(len(s["n"]), HQ, HKV, PAGE, s["table"].shape[1], D) for s in sets), dev)
    wb = api.new_workspace(max(api.token_sample_workspace_bytes(*s["x"].shape) for s in sets), dev)

    def call(s, wa, wb):
        api.paged_attn(s["q"], s["K"], s["V"], s["table"], s["n"], out=s["out"], workspace=wa)
        api.token_sample(s["x"], s["u"], top_p=s["p"], out=(s["tok"], s["lp"]), workspace=wb)

    def result(s):
        torch.cuda.synchronize()
        return [bits(s[x]).copy() for x in ("out", "tok", "lp")]

    want = []
    for s in sets:
        call(s, torch.zeros_like(wa), torch.zeros_like(wb))
        want.append(result(s))
    graphs = []
    for s in sets:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            call(s, wa, wb)
        graphs.append(gr)
    for rep in range(4):
        for i in (0, 1, 1, 0):
            for x in ("out", "tok", "lp"):
                sets[i][x].zero_()
            graphs[i].replay()
            assert same(result(sets[i]), want[i]), f"graph {i}, replay {rep}"
            call(sets[1 - i], wa, wb)
            assert same(result(sets[1 - i]), want[1 - i])
