"""The loop around the paged cache with prompts among the drafts and a pool that is too small: what a program has to do of its own, and that its
conversations then have what they would have had alone."""
import math

import numpy as np
import pytest
import torch

from oracle import serve_oracle as orc

pytestmark = pytest.mark.gpu
VOCAB, H, H_KV, D, PAGE, DRAFTS, CHUNK = 31, 4, 2, 64, 16, 3, 20


@pytest.fixture(scope="module")
def esa():
    import paper_2502_14477_amd as lib
    return lib


def f64(t):
    return t.double().cpu().numpy()


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Talk:
    """A conversation as the host knows it: tokens in the cache, and those that its next step brings."""

    def __init__(self, rng):
        self.stored, self.prompt, self.rng = [], rng.integers(0, VOCAB, rng.integers(5, 60)).tolist(), rng
        self.rows = []

    def next(self):
        """The step's tokens, and how many of them, from the end, are verified."""
        if self.prompt:
            self.rows = self.prompt[:CHUNK]
            return self.rows, int(len(self.prompt) <= CHUNK)
        if len(self.rows) != DRAFTS + 1 or self.rows[0] != self.last:
            self.rows = [self.last] + self.rng.integers(0, VOCAB, DRAFTS).tolist()
        return self.rows, DRAFTS + 1

    def done(self, new):
        """The step has counted; new: the tokens behind its verified rows."""
        if self.prompt:
            self.stored, self.prompt = self.stored + self.rows, self.prompt[CHUNK:]
        else:
            self.stored = self.stored + self.rows[:len(new)]
        if new:
            self.last = new[-1]
        self.rows = []


@pytest.mark.parametrize("n_pages,lacking", [(60, False), (17, True)])
def test_prompts_and_lacking_pages(esa, n_pages, lacking):
    n_seq, n_tok, steps = 5, 5 * CHUNK + 2, 60
    rng = np.random.default_rng(3)
    g = torch.Generator("cuda").manual_seed(21)
    wq, wk, wv = (torch.randn((VOCAB, n, D), generator=g, device="cuda").bfloat16() for n in (H, H_KV, H_KV))
    head = torch.randn((H * D, VOCAB), generator=g, device="cuda") * 0.3
    caches = [torch.full((n_pages, H_KV, PAGE, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    start, held, ring_at = ints([0] * n_seq), ints([0] * n_seq), ints([0, n_pages])
    pages, ring = torch.full((n_seq, 12), -1, dtype=torch.int32, device="cuda"), torch.arange(n_pages, dtype=torch.int32, device="cuda")
    out = esa.PagePlan.empty(n_seq, n_tok, "cuda")._replace(start=start, held=held, ring_at=ring_at)
    talks, grow = [Talk(rng) for _ in range(n_seq)], ints([0] * n_seq)
    waited, prompts, drafted = 0, 0, 0
    for step in range(steps):
        steps_of = [t.next() for t in talks]
        new, checked = [len(r) for r, _ in steps_of], [n for _, n in steps_of]
        tokens = ints(sum((r for r, _ in steps_of), []) + [0] * (n_tok - sum(new)))
        plan = esa.esa_plan_paged(ints(new), start, held, pages, ring, ring_at, PAGE, n_tok, grow=grow, out=out)
        x = tokens.long()
        q, k, v = wq[x], wk[x], wv[x]
        batch = (plan.cu, plan.start, pages, *caches)
        esa.esa_append_paged(k, v, *batch)
        o = esa.esa_attend_paged(q, *batch)
        # the rows that a new token may follow, and their own offsets
        ends = np.cumsum(new)
        rows = np.concatenate([np.arange(e - n, e) for e, n in zip(ends, checked)]).astype(np.int64)
        own = np.concatenate(([0], np.cumsum(checked)))
        at = torch.from_numpy(rows).cuda()
        target = torch.softmax(o[at].flatten(1).float() @ head, 1)
        u = torch.from_numpy(rng.random(len(rows)).astype(np.float32)).cuda()
        got, count = esa.esa_verify_drafts(target, tokens[at], ints(own.tolist()), u)
        short = plan.held * PAGE < plan.start + plan.cu.diff()
        grow = torch.where(short, 0, count + plan.cu.diff() - ints(checked))
        # the host's side of it
        want, margins = orc.verify(f64(target), tokens[at].tolist(), own, u.cpu().numpy())
        missing = sum(-(-(s + n) // PAGE) - h for s, n, h in zip(start.tolist(), new, held.tolist()))
        assert plan.lack.item() == missing and plan.cu.tolist() == [0, *ends.tolist()]
        table, (k_cache, v_cache) = pages.cpu().numpy(), (f64(c) for c in caches)
        held_pages = [p for b in range(n_seq) for p in table[b, :held[b].item()]]
        assert len(set(held_pages)) == len(held_pages) and len(held_pages) + ring_at[1].item() == n_pages
        for b, t in enumerate(talks):
            assert plan.start[b].item() == len(t.stored)
            if short[b].item():
                waited += 1
                assert grow[b].item() == 0
                continue
            seen = np.array(t.stored + t.rows)
            place = np.arange(len(seen))
            keys, values = (c[table[b, place // PAGE], :, place % PAGE] for c in (k_cache, v_cache))
            assert np.array_equal(keys, f64(wk)[seen]) and np.array_equal(values, f64(wv)[seen])
            for i in range(len(t.rows)):
                n, row = len(t.stored) + i + 1, ends[b] - len(t.rows) + i
                for h in range(H):
                    s = keys[:n, h // 2] @ f64(q[row, h]) / math.sqrt(D)
                    p = np.exp(s - s.max())
                    p /= p.sum()
                    exact, spread = p @ values[:n, h // 2], p @ np.abs(values[:n, h // 2])
                    # probabilities keep 8 bits or more, sums are fp32, one rounding to storage
                    assert np.all(np.abs(f64(o[row, h]) - exact) <= 2.0 ** -8 * np.abs(exact) + (2.0 ** -7 + (n + 128) * 2.0 ** -22) * spread)
            assert margins[b] > 1e-12 and count[b].item() == len(want[b]) and got[own[b]:own[b] + len(want[b])].tolist() == want[b]
            prompts, drafted = prompts + bool(t.prompt), drafted + (len(want[b]) > 1)
            t.done(want[b])
        # conversations end, and where nobody can go on one is given up: another one takes its place
        for b, t in enumerate(talks):
            if len(t.stored) > 100 or (torch.all(short).item() and b == step % n_seq):
                grow[b] = -plan.start[b]
                talks[b] = Talk(rng)
    assert prompts > 10 and drafted > 0 and (waited > 0) == lacking      # what the steps were made of
