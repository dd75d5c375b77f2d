"""The calls around the paged cache as a serving program makes them: planned, rotated, appended, attended to, verified, step after step, eager
and from a captured graph."""
import math

import numpy as np
import pytest
import torch

from oracle import serve_oracle as orc

pytestmark = pytest.mark.gpu
VOCAB, H, H_KV, D, PAGE, DRAFTS = 97, 4, 2, 64, 16, 3


@pytest.fixture(scope="module")
def esa():
    import paper_2502_14477_amd as lib
    return lib


class Server:
    """A model of one attention layer, a draft model that knows pairs of tokens, and a pool that its conversations share.  Everything a step needs
    is on the GPU; what changes from outside is written into buffers that keep their places."""

    def __init__(self, esa, n_seq, n_pages, in_place):
        g = torch.Generator("cuda").manual_seed(17)
        def normal(*shape, size=1.0):
            return torch.randn(shape, generator=g, device="cuda") * size
        self.esa, self.n_seq, self.in_place = esa, n_seq, in_place
        self.wq, self.wk, self.wv = (normal(VOCAB, n, D).bfloat16() for n in (H, H_KV, H_KV))
        self.head = normal(H * D, VOCAB, size=0.5)
        self.guess = torch.softmax(normal(VOCAB, VOCAB) * 2.0, 1)
        self.guess_sums = self.guess.double().cumsum(1)
        self.freq = esa.esa_rope_frequencies(1e4, D // 2, esa.ESA_SCALE_YARN, 4.0, 64.0)
        self.n_tok = n_seq * (DRAFTS + 1) + 2
        ints = lambda *n: torch.zeros(n, dtype=torch.int32, device="cuda")
        self.plan = esa.PagePlan.empty(n_seq, self.n_tok, "cuda")
        for t in self.plan:
            t.zero_()
        self.old = [ints(n_seq), ints(n_seq), torch.tensor([0, n_pages], dtype=torch.int32, device="cuda")]      # start, held, ring_at
        if in_place:
            self.plan = self.plan._replace(start=self.old[0], held=self.old[1], ring_at=self.old[2])
        self.pages, self.ring = ints(n_seq, 24), torch.arange(n_pages, dtype=torch.int32, device="cuda")
        self.caches = [torch.full((n_pages, H_KV, PAGE, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in "kv"]
        self.new, self.grow, self.extra = ints(n_seq), ints(n_seq), ints(n_seq)
        self.tokens = ints(self.n_tok)
        self.u = torch.zeros(self.n_tok, device="cuda")
        self.r = torch.zeros((n_seq, DRAFTS), device="cuda", dtype=torch.float64)
        self.of = torch.arange(n_seq, device="cuda")

    def step(self):
        esa, got = self.esa, {}
        got["grow"] = self.grow + self.extra
        plan = esa.esa_plan_paged(self.new, *self.old[:2], self.pages, self.ring, self.old[2], PAGE, self.n_tok, grow=got["grow"], out=self.plan)
        if not self.in_place:
            for a, b in zip(self.old, (plan.start, plan.held, plan.ring_at)):
                a.copy_(b)
        x = self.tokens.long()
        q, k, v = self.wq[x], self.wk[x], self.wv[x]
        got["q"], got["k"] = esa.esa_rope_at(q, plan.pos, self.freq, k=k, pairs=esa.ESA_PAIRS_NEIGHBOURS, gain=1.125, out_q=q, out_k=k)
        batch = (plan.cu, plan.start, self.pages, *self.caches)
        esa.esa_append_paged(got["k"], v, *batch)
        got["o"] = torch.zeros_like(q)
        esa.esa_attend_paged(got["q"], *batch, out=got["o"])
        got["target"] = torch.softmax(got["o"].flatten(1).float() @ self.head, 1)
        got["draft"] = self.guess[x.roll(1)]
        out = torch.full_like(self.tokens, -5)
        got["out"], got["count"] = esa.esa_verify_drafts(got["target"], self.tokens, plan.cu, self.u, draft=got["draft"], out=out)
        for name, t in zip(plan._fields, plan):
            got[name] = t.clone()
        got["tokens"] = self.tokens.clone()
        # the next step: the last new token and drafts behind it
        self.grow.copy_(got["count"])
        last = got["out"][(plan.cu[:-1] + got["count"] - 1).clamp(min=0).long()].clamp(min=0).long()
        rows = [last]
        for j in range(DRAFTS):
            rows.append((self.guess_sums[rows[-1]] <= self.r[:, j:j + 1]).sum(1).clamp(max=VOCAB - 1))
        self.tokens[:self.n_seq * (DRAFTS + 1)] = torch.stack(rows, 1).flatten().int()
        return got


def inputs(server, rng, step):
    """What comes from outside in front of a step: random numbers, a prompt's first rows, conversations that end and begin."""
    server.u.copy_(torch.from_numpy(rng.random(server.n_tok).astype(np.float32)))
    server.r.copy_(torch.from_numpy(rng.random((server.n_seq, DRAFTS))))
    server.new.fill_(DRAFTS + 1)
    server.extra.zero_()
    if step == 0:
        server.tokens.copy_(torch.from_numpy(rng.integers(0, VOCAB, server.n_tok)))
    if step in (5, 9):                                            # a conversation ends, another one takes its place
        server.extra[step % server.n_seq] = -10000


def check_step(server, got, pool, kept_slots, rng_half=2.0 ** -8):
    f64 = lambda t: t.double().cpu().numpy()
    whole = {n: got[n].cpu().numpy() for n in ("cu", "start", "held", "pos", "slot", "lack", "grow", "out", "count", "tokens")}
    fresh = [DRAFTS + 1] * server.n_seq
    cu, pos, slot, lack = pool.step(fresh, server.n_tok, whole["grow"])
    for name, want in (("cu", cu), ("pos", pos), ("slot", slot), ("start", pool.start), ("held", [len(r) for r in pool.rows])):
        assert np.array_equal(whole[name], want), name
    assert whole["lack"][0] == lack == 0
    x = whole["tokens"]
    there = pos >= 0
    for name, w in (("q", server.wq), ("k", server.wk)):
        rows = f64(w)[x]
        want = orc.rope(rows, pos, server.freq.cpu().numpy(), False, 1.125)
        assert np.all(np.abs(f64(got[name]) - want)[there] <= (rng_half * np.abs(want) * (1 + 1e-9) + 2.0 ** -40)[there])
        assert np.array_equal(f64(got[name])[~there], rows[~there])
    caches = [f64(c) for c in server.caches]
    for b in range(server.n_seq):
        del kept_slots[b][pool.start[b]:]                         # what the last step drafted in vain, or all of an ended one
        kept_slots[b] += slot[cu[b]:cu[b + 1]].tolist()
        at = np.array(kept_slots[b])
        assert len(at) == pool.start[b] + cu[b + 1] - cu[b]
        k, v = (c[at // PAGE, :, at % PAGE] for c in caches)
        new = f64(got["k"])[cu[b]:cu[b + 1]]
        assert np.array_equal(k[-len(new):], new)
        for i in range(cu[b], cu[b + 1]):
            n = pos[i] + 1
            for h in range(H):
                s = k[:n, h // 2] @ f64(got["q"])[i, h] / math.sqrt(D)
                p = np.exp(s - s.max())
                p /= p.sum()
                want = p @ v[:n, h // 2]
                spread = p @ np.abs(v[:n, h // 2])
                # probabilities keep 16 bits (two terms) in batches of up to 64 rows, 8 beyond; fp32 sums; one rounding to storage
                assert np.all(np.abs(f64(got["o"])[i, h] - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -7 + (n + 128) * 2.0 ** -22) * spread)
    want, margins = orc.verify(f64(got["target"]), x, cu, got["u"], f64(got["draft"]))
    assert min(margins) > 1e-12
    for b, w in enumerate(want):
        assert whole["out"][cu[b]:cu[b + 1]].tolist() == w + [-1] * (DRAFTS + 1 - len(w)) and whole["count"][b] == len(w)
    assert np.all(whole["out"][cu[-1]:] == -5)


@pytest.mark.parametrize("in_place", [True, False])
def test_steps_of_a_server(esa, in_place):
    rng = np.random.default_rng(6)
    server = Server(esa, 5, 40, in_place)
    pool, kept = orc.Pages(5, 24, 40, PAGE), [[] for _ in range(5)]
    for step in range(14):
        inputs(server, rng, step)
        got = server.step()
        got["u"] = server.u.cpu().numpy()
        check_step(server, got, pool, kept)


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("n_seq,n_pages", [(5, 40), (70, 700)])
def test_a_captured_step_goes_on_as_an_eager_one(esa, n_seq, n_pages, in_place):
    """Replays with the program's own work between them: every output of every step is the eager server's, bit for bit."""
    eager, captured = Server(esa, n_seq, n_pages, in_place), Server(esa, n_seq, n_pages, in_place)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                                 # warmed up on a server of its own
        warm = Server(esa, n_seq, n_pages, in_place)
        inputs(warm, np.random.default_rng(1), 0)
        warm.step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        replayed = captured.step()
    for s in (eager, captured):
        inputs(s, np.random.default_rng(7), 0)
    rng_a, rng_b = np.random.default_rng(8), np.random.default_rng(8)
    for step in range(1, 13):
        want = eager.step()
        graph.replay()
        torch.cuda.synchronize()
        for name in want:
            a, b = want[name], replayed[name]
            assert torch.equal(a.view(torch.uint8) if a.is_floating_point() else a, b.view(torch.uint8) if b.is_floating_point() else b), (step, name)
        for a, b in ((eager.pages, captured.pages), (eager.ring, captured.ring)):
            assert torch.equal(a, b)
        inputs(eager, rng_a, step)
        inputs(captured, rng_b, step)
        torch.randn(1000, device="cuda").sum().item()             # the program's own


def test_calls_on_two_streams_at_once(esa):
    """Workspaces belong to a call: two streams' calls do not meet."""
    streams = [torch.cuda.Stream() for _ in range(2)]
    g = torch.Generator("cuda").manual_seed(3)
    jobs = []
    for n_seq, vocab in ((40, 60001), (3, 120000)):
        cu = torch.arange(0, 4 * n_seq + 1, 4, dtype=torch.int32, device="cuda")
        p = torch.softmax(torch.randn((4 * n_seq, vocab), generator=g, device="cuda") * 2, 1)
        tokens = torch.randint(0, vocab, (4 * n_seq,), generator=g, device="cuda", dtype=torch.int32)
        u = torch.rand(4 * n_seq, generator=g, device="cuda")
        n = 3000 * n_seq
        state = [torch.full((n_seq,), 3000, dtype=torch.int32, device="cuda"), *(torch.zeros(n_seq, dtype=torch.int32, device="cuda") for _ in range(2)),
                 torch.zeros((n_seq, 200), dtype=torch.int32, device="cuda"), torch.arange(300 * n_seq, dtype=torch.int32, device="cuda"),
                 torch.tensor([5, 300 * n_seq], dtype=torch.int32, device="cuda")]
        jobs.append((lambda p=p, tokens=tokens, cu=cu, u=u: esa.esa_verify_drafts(p, tokens, cu, u, draft=p.roll(1, 0)),
                     lambda state=state, n=n: esa.esa_plan_paged(*state, 16, n)))
    want = [[call() for call in job] for job in jobs]
    torch.cuda.synchronize()
    got = [[], []]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(20):
        for i, (s, job) in enumerate(zip(streams, jobs)):
            with torch.cuda.stream(s):
                got[i].append([call() for call in job])
    torch.cuda.synchronize()
    for i in range(2):
        for one in got[i]:
            for x, y in zip(one, want[i]):
                assert all(torch.equal(a, b) for a, b in zip(x, y))


def test_two_graphs_of_one_pool(esa):
    """Two captured plans of the same state, replayed in turn: state goes from one to the other through its arrays alone."""
    n_seq, n_tok = 300, 900                                       # of two launches in place, with a workspace of each graph's own
    def fresh_state():
        ints = lambda *n: torch.zeros(n, dtype=torch.int32, device="cuda")
        return [ints(n_seq), ints(n_seq), ints(n_seq, 500), torch.arange(9000, dtype=torch.int32, device="cuda"), torch.tensor([0, 9000], dtype=torch.int32, device="cuda")]
    news = [torch.full((n_seq,), k, dtype=torch.int32, device="cuda") for k in (3, 2)]
    states = [fresh_state(), fresh_state()]
    outs = []
    for start, held, pages, ring, ring_at in states:
        outs.append([esa.PagePlan.empty(n_seq, n_tok, "cuda")._replace(start=start, held=held, ring_at=ring_at) for _ in range(2)])
    def plan(which, k):
        start, held, pages, ring, ring_at = states[which]
        return esa.esa_plan_paged(news[k], start, held, pages, ring, ring_at, 16, n_tok, grow=news[k], out=outs[which][k])
    torch.cuda.synchronize()
    graphs = []
    for k in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            plan(1, k)
        graphs.append(g)
    for step in range(40):
        plan(0, step % 2)
        graphs[step % 2].replay()
        torch.cuda.synchronize()
        for a, b in zip(outs[0][step % 2], outs[1][step % 2]):
            assert torch.equal(a, b)
        for a, b in zip(states[0], states[1]):
            assert torch.equal(a, b)
    assert states[0][0][0].item() == 100 and states[0][4][1].item() == 9000 - 300 * 7
