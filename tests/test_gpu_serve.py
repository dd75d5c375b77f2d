"""The calls around the paged cache against plain implementations in 64 bits and whole numbers."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import serve_oracle as orc

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
SMALLEST = {"bf16": 2.0 ** -134, "f32": 2.0 ** -150}      # half a step of subnormal numbers


@pytest.fixture(scope="module")
def esa():
    import paper_2502_14477_amd as lib
    return lib


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def ints(x, dtype=torch.int32):
    return torch.tensor(np.asarray(x), dtype=dtype, device="cuda")


# ---------------------------------------------------------------- rotation
def check_rope(x, got, pos, freq, halves, gain, transposed, dtype):
    """Rounding to storage: half a step.  The angle pos * freq is rounded to 2^-53 of itself, its reduction, sine, cosine and the products take a few
    roundings of 2^-53 more, of the pair's length."""
    want = orc.rope(f64(x), pos, freq, halves, gain, transposed)
    there = np.asarray(pos) >= 0
    angle = np.max(np.abs(np.asarray(pos, dtype=np.float64))) * np.max(np.abs(freq)) + 16
    pair = abs(gain) * 1.5 * np.max(np.abs(f64(x)), axis=-1, keepdims=True)
    tol = HALF_STEP[dtype] * np.abs(want) * (1 + 1e-9) + angle * 2.0 ** -53 * pair + SMALLEST[dtype]
    off = np.abs(f64(got) - want)
    assert np.all((off <= tol)[there]), float(np.max((off / tol)[there]))


def layout(rng, n, heads, d, dtype, kind):
    """A tensor [n, heads, d] of which tokens and heads lie in some order, and a place for outputs of the same kind."""
    def place():
        if kind == "contiguous":
            return torch.empty((n, heads, d), dtype=TYPES[dtype], device="cuda")
        if kind == "heads first":
            return torch.empty((heads, n, d), dtype=TYPES[dtype], device="cuda").transpose(0, 1)
        if kind == "one projection":
            return torch.empty((n, 2 * heads + 1, d), dtype=TYPES[dtype], device="cuda")[:, heads:2 * heads]
        if kind == "odd":
            return torch.empty((n, heads, d + 3), dtype=TYPES[dtype], device="cuda")[..., 1:d + 1]
        if kind == "half aligned":                               # 8-byte boundaries
            by = 4 if dtype == "bf16" else 2
            return torch.empty((n, heads, d + by), dtype=TYPES[dtype], device="cuda")[..., by:]
    x, out = place(), place()
    x.copy_(torch.from_numpy(rng.standard_normal((n, heads, d))))
    out.fill_(-7.0)
    return x, out


KINDS = ["contiguous", "heads first", "one projection", "odd", "half aligned"]
SHAPES = [  # tokens, heads, KV heads, head size, elements that turn
    (1, 1, 1, 2, 2), (1, 32, 8, 128, 128), (3, 5, 5, 40, 20), (130, 16, 2, 80, 32), (77, 4, 1, 256, 256), (16, 8, 8, 64, 64), (9, 3, 2, 1024, 256), (5, 7, 3, 96, 96), (300, 1, 1, 6, 4)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("halves", [True, False])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape", SHAPES, ids=["x".join(map(str, s)) for s in SHAPES])
def test_rope_at(esa, shape, kind, halves, dtype):
    n, h, h_kv, d, rot = shape
    rng = np.random.default_rng(n + d)
    pos = rng.integers(0, 300000, n)
    pos[0] = 0 if n > 1 else 123457
    if n > 2:
        pos[1], pos[2] = 2 ** 31 - 1, -1
    if n > 100:
        pos[-20:] = -rng.integers(1, 2 ** 31, 20)
    freq = esa.esa_rope_frequencies(1e4, rot, esa.ESA_SCALE_YARN, 4.0, 4096.0)
    q, oq = layout(rng, n, h, d, dtype, kind)
    k, ok = layout(rng, n, h_kv, d, dtype, kind)
    pairs = esa.ESA_PAIRS_HALVES if halves else esa.ESA_PAIRS_NEIGHBOURS
    for transposed, gain in ((False, 1.25), (True, 1.0)):
        got = esa.esa_rope_at(q, ints(pos), freq, k=k, pairs=pairs, gain=gain, transposed=transposed, out_q=oq, out_k=ok)
        assert got[0] is oq and got[1] is ok
        for x, y in ((q, oq), (k, ok)):
            check_rope(x, y, pos, freq.cpu().numpy(), halves, gain, transposed, dtype)
            assert torch.all(y[torch.from_numpy(pos < 0).cuda()] == -7.0)        # rows of nobody
    alone = esa.esa_rope_at(q, ints(pos), freq, pairs=pairs, transposed=True)    # one tensor, into a new one
    assert torch.equal(alone[torch.from_numpy(pos >= 0).cuda()], oq[torch.from_numpy(pos >= 0).cuda()])
    before = k.clone()
    esa.esa_rope_at(q, ints(pos), freq, k=k, pairs=pairs, transposed=True, out_q=q, out_k=k)      # in place
    assert torch.equal(q[torch.from_numpy(pos >= 0).cuda()], alone[torch.from_numpy(pos >= 0).cuda()]) and torch.equal(k[torch.from_numpy(pos >= 0).cuda()], ok[torch.from_numpy(pos >= 0).cuda()])
    there = torch.from_numpy(pos < 0).cuda()
    assert torch.equal(k[there], before[there])


def test_rope_at_leaves_what_lies_around(esa):
    """Rows in a wider buffer: nothing but the rows is written."""
    for d, rot, pad in ((40, 20, 3), (64, 64, 8), (80, 32, 16)):
        for dtype in ("bf16", "f32"):
            whole = torch.full((11, 5, d + pad), 3.0, dtype=TYPES[dtype], device="cuda")
            q = torch.ones((11, 5, d), dtype=TYPES[dtype], device="cuda")
            esa.esa_rope_at(q, ints(np.arange(11)), esa.esa_rope_frequencies(1e4, rot), out_q=whole[..., :d])
            assert torch.all(whole[..., d:] == 3.0) and not torch.any(whole[..., :d] == 3.0)


def test_rope_at_turns_as_the_framework_does(esa):
    """Unscaled halves of whole heads are what esa_rope and esa_append_paged turn, to a rounding of the same 64-bit numbers."""
    x = torch.randn((500, 8, 128), device="cuda", generator=torch.Generator("cuda").manual_seed(4)).bfloat16()
    a = esa.esa_rope(x, 1000.0, 1.0, 5e5)
    b = esa.esa_rope_at(x, torch.arange(1000, 1500, dtype=torch.int32, device="cuda"), esa.esa_rope_frequencies(5e5, 128))
    differ = a != b
    assert differ.sum() <= 2 and torch.all((a.float() - b.float()).abs() <= 2.0 ** -7 * a.float().abs())


@pytest.mark.parametrize("halves", [True, False])
def test_rope_at_gradients(esa, halves):
    """The transposed call against the formula's gradient and against differences: the map is linear, so these are exact but for roundings."""
    rng = np.random.default_rng(8)
    n, h, d, rot = 7, 3, 20, 12
    pos, gain = rng.integers(0, 1000, n), 1.375
    freq = esa.esa_rope_frequencies(1e4, rot, esa.ESA_SCALE_NTK, 4.0)
    kw = dict(pairs=esa.ESA_PAIRS_HALVES if halves else esa.ESA_PAIRS_NEIGHBOURS, gain=gain)
    x = torch.from_numpy(rng.standard_normal((n, h, d))).float().cuda()
    g = torch.from_numpy(rng.standard_normal((n, h, d))).float().cuda()
    back = f64(esa.esa_rope_at(g, ints(pos), freq, transposed=True, **kw))
    # d/dx sum(g * rope(x)) along a direction e, by a central difference of step 1
    for seed in range(4):
        e = torch.from_numpy(np.random.default_rng(seed).standard_normal((n, h, d))).float().cuda()
        up, down = (f64(esa.esa_rope_at(x + s * e, ints(pos), freq, **kw)) for s in (1.0, -1.0))
        by_difference = np.sum(f64(g) * (up - down))
        step = f64(x + e) - f64(x - e)
        tol = 2.0 ** -24 * (np.sum(np.abs(f64(g)) * (np.abs(up) + np.abs(down))) + np.sum(np.abs(back) * np.abs(step)))
        assert abs(by_difference - np.sum(back * step)) <= tol
    want = orc.rope(f64(g), pos, freq.cpu().numpy(), halves, gain, True)
    assert np.all(np.abs(back - want) <= 2.0 ** -24 * np.abs(want) * (1 + 1e-9) + 2.0 ** -40)


def test_rope_at_passes_infinities_and_nan(esa):
    x = torch.ones((2, 2, 8), device="cuda")
    x[0, 1, 2], x[1, 0, 3] = float("nan"), float("inf")
    for dtype in TYPES.values():
        y = esa.esa_rope_at(x.to(dtype), ints([5, 6]), esa.esa_rope_frequencies(1e4, 8))
        bad = ~torch.isfinite(y)
        want = torch.zeros_like(bad)
        want[0, 1, [2, 6]] = want[1, 0, [3, 7]] = True
        assert torch.equal(bad, want)


def test_rope_at_frequencies_of_any_content(esa):
    """Given ones: as they are; what is no number gives none in its own pair, and nothing else."""
    rng = np.random.default_rng(13)
    freq = np.array([64.0, -64.0, 1e-300, 0.0, 0.75, float("nan"), float("inf"), 1e300])
    x = torch.from_numpy(rng.standard_normal((40, 2, 16))).float().cuda()
    pos = rng.integers(1, 2 ** 31, 40)
    y = esa.esa_rope_at(x, ints(pos), ints(freq, torch.float64))
    want = orc.rope(f64(x)[..., [0, 1, 2, 3, 4, 8, 9, 10, 11, 12]], pos, freq[:5])
    # angles of up to 2^37, rounded to 2^-53 of themselves
    tol = 2.0 ** -24 * np.abs(want) + 64 * pos.max() * 2.0 ** -53 * 4
    assert np.all(np.abs(f64(y)[..., [0, 1, 2, 3, 4, 8, 9, 10, 11, 12]] - want) <= tol)
    assert torch.all(torch.isnan(y[..., [5, 6, 13, 14]]))


def test_rope_at_far_tokens(esa):
    """Offsets beyond 32 bits: tokens a gigabyte apart."""
    x = torch.empty((6, 1 << 29), dtype=torch.bfloat16, device="cuda")[:, :256].view(6, 2, 128)
    x.copy_(torch.randn((6, 2, 128), generator=torch.Generator().manual_seed(1)))
    pos = np.arange(6) * 1000
    freq = esa.esa_rope_frequencies(5e5, 128)
    check_rope(x, esa.esa_rope_at(x, ints(pos), freq), pos, freq.cpu().numpy(), True, 1.0, False, "bf16")
    want = esa.esa_rope_at(x.contiguous(), ints(pos), freq)
    assert torch.equal(esa.esa_rope_at(x, ints(pos), freq, out_q=x), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rope_at_in_one_buffer(esa, dtype):
    """Queries and keys of one projection turned where they lie: the values beside them stay; a row that all tokens share."""
    g = torch.Generator("cuda").manual_seed(6)
    x = torch.randn((50, 12, 64), generator=g, device="cuda").to(TYPES[dtype])
    before, pos, freq = x.clone(), torch.arange(50, dtype=torch.int32, device="cuda") * 7, esa.esa_rope_frequencies(1e4, 32)
    want = esa.esa_rope_at(before[:, :8], pos, freq, k=before[:, 8:10])
    esa.esa_rope_at(x[:, :8], pos, freq, k=x[:, 8:10], out_q=x[:, :8], out_k=x[:, 8:10])
    assert torch.equal(x[:, :8], want[0]) and torch.equal(x[:, 8:10], want[1]) and torch.equal(x[:, 10:], before[:, 10:])
    shared = before[:1].expand(50, 12, 64)
    assert torch.equal(esa.esa_rope_at(shared, pos, freq), esa.esa_rope_at(shared.contiguous(), pos, freq))


def test_rope_at_many_tokens(esa):
    """More workgroups than one dimension of a grid takes."""
    n, h, d = 18_000_000, 64, 8
    x = torch.ones((n, h, d), dtype=torch.bfloat16, device="cuda")
    pos = torch.arange(n, dtype=torch.int32, device="cuda") % 1000
    freq = esa.esa_rope_frequencies(1e4, d)
    esa.esa_rope_at(x, pos, freq, out_q=x)
    want = esa.esa_rope_at(torch.ones((1000, 1, d), dtype=torch.bfloat16, device="cuda"), pos[:1000], freq)
    for at in range(0, n, 1_000_000):
        assert torch.all(x[at:at + 1_000_000].view(1000, 1000, h, d) == want)


# ---------------------------------------------------------------- plans
class Guarded:
    """Arrays with numbers around them that nobody may change."""

    def __init__(self):
        self.all = []

    def __call__(self, x, dtype=torch.int32):
        x = np.asarray(x)
        whole = torch.full((x.size + 128,), 77, dtype=dtype, device="cuda")
        mine = whole[64:64 + x.size]
        mine.copy_(torch.from_numpy(x.reshape(-1)).to(dtype))
        self.all.append(whole)
        return mine

    def check(self):
        for w in self.all:
            assert torch.all(w[:64] == 77) and torch.all(w[-64:] == 77)


class Loop:
    """A pool on the GPU beside the oracle's, stepped together."""

    def __init__(self, esa, n_seq, max_pages, n_pages, page, n_tok, seed, pad=3):
        self.esa, self.page, self.n_tok, self.rng = esa, page, n_tok, np.random.default_rng(seed)
        self.keep = Guarded()
        self.oracle = orc.Pages(n_seq, max_pages, n_pages, page)
        self.table = np.full((n_seq, max_pages + pad), 99, dtype=np.int32)
        self.flat = self.keep(self.table)
        self.pages = self.flat.view(n_seq, max_pages + pad)[:, :max_pages]
        first = int(self.rng.integers(0, n_pages))
        self.oracle.free = self.rng.permutation(n_pages).tolist()
        self.ring = self.keep(np.roll(self.oracle.free, first))
        self.start, self.held, self.ring_at = self.keep(np.zeros(n_seq)), self.keep(np.zeros(n_seq)), self.keep([first, n_pages])
        k = self.keep
        self.out = esa.PagePlan(k(np.zeros(n_seq + 1)), self.start, self.held, self.ring_at, k(np.zeros(n_tok)), k(np.zeros(n_tok), torch.int64), k([0]))

    def step(self, fresh, grow):
        """In place, and into new tensors from copies: the same."""
        args = (ints(fresh), self.start, self.held, self.pages, self.ring, self.ring_at, self.page, self.n_tok)
        g = None if grow is None else ints(grow)
        copies = [self.start.clone(), self.held.clone(), self.pages.clone(), self.ring.clone(), self.ring_at.clone()]
        for _ in range(2):                                        # repeated on the same state
            aside = self.esa.esa_plan_paged(ints(fresh), *copies, self.page, self.n_tok, grow=g)
        got = self.esa.esa_plan_paged(*args, grow=g, out=self.out)
        assert got is self.out
        for x, y in zip(aside, got):
            assert torch.equal(x, y)
        assert torch.equal(copies[2], self.pages) and torch.equal(copies[3], self.ring)
        held = [len(r) for r in self.oracle.rows]
        cu, pos, slot, lack = self.oracle.step(fresh, self.n_tok, grow)
        o = self.oracle
        assert np.array_equal(got.cu.cpu().numpy(), cu) and np.array_equal(got.start.cpu().numpy(), o.start)
        assert np.array_equal(got.held.cpu().numpy(), [len(r) for r in o.rows]) and got.lack.item() == lack
        assert np.array_equal(got.pos.cpu().numpy(), pos) and np.array_equal(got.slot.cpu().numpy(), slot)
        first, count = got.ring_at.tolist()
        assert count == len(o.free) and np.array_equal(np.roll(self.ring.cpu().numpy(), -first)[:count], o.free)
        for b, row in enumerate(o.rows):
            if len(row) > held[b]:                                # what else the row holds stays
                self.table[b, held[b]:len(row)] = row[held[b]:]
            self.table[b, len(row):len(row) + o.missing[b]] = -1
        assert np.array_equal(self.flat.cpu().numpy().reshape(self.table.shape), self.table)
        self.keep.check()
        return cu

    def kept(self, cu, ended=0.15):
        n = np.diff(cu)
        grow = np.where(n > 0, self.rng.integers(0, 1 << 30, len(n)) % (n + 1), 0)
        return np.where(self.rng.random(len(n)) < ended, -np.array(self.oracle.start), grow)


PLANS = [  # sequences, entries of a row, pages, page size, rows, most new tokens
    (1, 1, 1, 16, 1, 1), (1, 40, 50, 128, 700, 600), (5, 7, 60, 16, 300, 60), (63, 9, 300, 32, 900, 12), (65, 12, 500, 16, 2000, 33), (1023, 4, 2500, 64, 3000, 5),
    (1025, 5, 3000, 16, 6000, 9), (2500, 3, 4000, 16, 3000, 3), (5000, 2, 7000, 16, 9000, 4), (7, 300, 900, 16, 20000, 4000)]


@pytest.mark.parametrize("shape", PLANS, ids=["x".join(map(str, s)) for s in PLANS])
def test_plans_of_many_steps(esa, shape):
    n_seq, max_pages, n_pages, page, n_tok, most = shape
    loop = Loop(esa, n_seq, max_pages, n_pages, page, n_tok, seed=n_seq + page)
    grow = None
    for step in range(8):
        fresh = loop.rng.integers(-1, most + 1, n_seq)            # some have nothing, some less than that
        if step == 3:
            fresh[:] = 0
        grow = loop.kept(loop.step(fresh, grow))


def test_plan_takes_pages_that_the_same_call_gives_back(esa):
    """Nothing is free: what ended sequences give back goes to those that grow, in order."""
    loop = Loop(esa, 6, 10, 30, 16, 500, seed=3)
    loop.step([80, 80, 80, 80, 80, 80], None)
    assert loop.out.ring_at.tolist()[1] == 0
    loop.step([0, 40, 0, 60, 10, 0], [-1000, 80, -1000, 80, 80, -1000])
    assert loop.out.lack.item() == 0
    loop.step([100, 100, 0, 0, 100, 0], [0, 40, 0, 60, 10, 0])
    assert loop.out.lack.item() > 0
    loop.step([100, 100, 0, 0, 100, 0], [0, 0, 0, -1000, 0, 0])   # again, as pages have come free


def test_plan_beyond_the_table(esa):
    """Positions that a row of the table has no entry for have no slot."""
    loop = Loop(esa, 3, 4, 40, 16, 300, seed=5)
    cu = loop.step([64, 100, 10], None)
    assert (loop.out.slot[64:164] >= 0).sum() == 64
    loop.step([5, 5, 100], [64, 100, 10])
    assert (loop.out.slot[:10] >= 0).sum() == 0


@pytest.mark.parametrize("n_seq", [70, 700, 3000, 5000])
def test_plan_of_more_rows_than_there_is_room_for(esa, n_seq):
    """Numbers whose sums leave 32 bits: rows are those that fit, in order."""
    loop = Loop(esa, n_seq, 3, 2 * n_seq, 16, 50, seed=8)
    loop.step([2 ** 31 - 1] * n_seq, None)
    loop.step([0] * (n_seq - 2) + [7, 2 ** 31 - 1], [2 ** 31 - 1] * n_seq)
    assert loop.out.cu[-1].item() == 50 and loop.out.lack.item() == n_seq


def test_plan_without_sequences_or_rows(esa):
    p = esa.esa_plan_paged(ints([]), ints([]), ints([]), torch.zeros((0, 3), dtype=torch.int32, device="cuda"), ints([4, 5, 6]), ints([2, 1]), 16, 5)
    assert p.cu.tolist() == [0] and p.pos.tolist() == [-1] * 5 and p.slot.tolist() == [-1] * 5 and p.ring_at.tolist() == [2, 1] and p.lack.item() == 0
    loop = Loop(esa, 4, 5, 30, 16, 0, seed=9)
    loop.step([3, 3, 3, 3], [0, 5, 40, 70])                       # no room for rows: the tokens that were kept have pages all the same


def test_plan_of_arrays_that_no_calls_lead_to(esa):
    """Nothing in the arrays leads out of a buffer."""
    rng = np.random.default_rng(12)
    wild = [-2 ** 31, -1, 0, 1, 2, 5, 100, 2 ** 20, 2 ** 31 - 1]
    for n_seq, max_pages, n_pages, n_tok in ((1, 1, 1, 3), (9, 5, 20, 40), (70, 3, 9, 300), (1500, 2, 50, 900)):
        for seed in range(4):
            keep = Guarded()
            fresh, start, held, grow = (keep(rng.choice(wild, n_seq)) for _ in range(4))
            pages = keep(rng.choice(wild, (n_seq, max_pages))).view(n_seq, max_pages)
            ring, ring_at = keep(rng.choice(wild, n_pages)), keep(rng.choice(wild, 2))
            k = keep
            out = esa.PagePlan(k(np.zeros(n_seq + 1)), k(np.zeros(n_seq)), k(np.zeros(n_seq)), k([0, 0]), k(np.zeros(n_tok)), k(np.zeros(n_tok), torch.int64), k([0]))
            esa.esa_plan_paged(fresh, start, held, pages, ring, ring_at, 16, n_tok, grow=grow, out=out)
            keep.check()
            cu, slot, first, count = out.cu.cpu().numpy(), out.slot.cpu().numpy(), *out.ring_at.tolist()
            assert cu[0] == 0 and np.all(np.diff(cu) >= 0) and cu[-1] <= n_tok and np.all((slot >= -1) & (slot < n_pages * 16))
            assert 0 <= first < n_pages and 0 <= count <= n_pages and torch.all((out.held >= 0) & (out.held <= max_pages))


def test_plan_of_a_long_table(esa):
    """Rows of the table beyond 32 bits of bytes."""
    n_seq, ld = 5, 1 << 28
    whole = torch.empty((n_seq, ld), dtype=torch.int32, device="cuda")
    pages = whole[:, :9]
    out = esa.esa_plan_paged(ints([40, 50, 60, 70, 80]), ints([0] * 5), ints([0] * 5), pages, ints(np.arange(40)), ints([0, 40]), 16, 320)
    want, at = [], 0
    for b, n in enumerate((40, 50, 60, 70, 80)):
        need = -(-n // 16)
        assert pages[b, :need].tolist() == list(range(at, at + need))
        want += [(at + i // 16) * 16 + i % 16 for i in range(n)]
        at += need
    assert out.slot.tolist() == want + [-1] * 20


# ---------------------------------------------------------------- drafts
def distributions(rng, n, vocab, peak=2.0):
    a = rng.standard_normal((n, vocab)) * peak
    p = np.exp(a - a.max(1, keepdims=True))
    b = np.exp(a + 0.7 * rng.standard_normal((n, vocab)))
    return p / p.sum(1, keepdims=True), b / b.sum(1, keepdims=True)


def held(x, dtype, pad=0):
    """Rows on the GPU, `pad` elements apart from each other, and what they hold."""
    whole = torch.full((x.shape[0], x.shape[1] + pad), float("nan"), dtype=TYPES[dtype], device="cuda")
    mine = whole[:, :x.shape[1]]
    mine.copy_(torch.from_numpy(x))
    return mine


def check_verify(esa, target, tokens, cu, u, draft, rows=None):
    n = len(tokens) if rows is None else rows
    out = torch.full((target.shape[0],), -9, dtype=torch.int32, device="cuda")
    got, count = esa.esa_verify_drafts(target, ints(tokens), ints(cu), ints(u, torch.float32), draft=draft, out=out)
    assert got is out
    want, margins = orc.verify(f64(target), tokens, cu, np.asarray(u, dtype=np.float32), None if draft is None else f64(draft))
    assert min(margins) > 1e-12                                   # the inputs', not the kernel's: no drawn number lies on a border
    got = got.cpu().numpy()
    assert count.tolist() == [len(w) for w in want]
    for b, w in enumerate(want):
        assert got[cu[b]:cu[b + 1]].tolist() == w + [-1] * (cu[b + 1] - cu[b] - len(w)), b
    assert np.all(got[cu[-1]:] == -9) and np.all(got[:cu[0]] == -9)
    fresh, again = esa.esa_verify_drafts(target, ints(tokens), ints(cu), ints(u, torch.float32), draft=draft)
    assert torch.equal(again, count) and np.array_equal(fresh.cpu().numpy()[cu[0]:cu[-1]], got[cu[0]:cu[-1]])
    return want


VERIFIES = [  # sequences, most drafts, vocabulary
    (1, 0, 1), (1, 4, 2), (3, 3, 63), (17, 5, 1000), (2, 2, 4096), (5, 4, 4097), (2, 150, 300), (4, 3, 50001), (3, 6, 131072), (40, 1, 777), (300, 1, 17001), (3, 2, 16384), (2, 2, 16385), (2, 3, 300007),
    (1, 2, 600001)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("shape", VERIFIES, ids=["x".join(map(str, s)) for s in VERIFIES])
def test_verify(esa, shape, drawn, dtype):
    n_seq, drafts, vocab = shape
    rng = np.random.default_rng(vocab + drafts)
    rows = [drafts + 1 if b == 0 else int(rng.integers(0, drafts + 2)) for b in range(n_seq)]
    cu = np.concatenate(([0], np.cumsum(rows)))
    n = int(cu[-1]) + 3                                           # rows of nobody
    p, q = distributions(rng, n, vocab)
    if drafts > 100:                                              # long runs that stand
        q = p.copy()
    tokens = np.array([rng.choice(vocab, p=x) for x in q])
    target = np.roll(p, -1, 0) if drawn else p                    # row i - 1's target stands behind row i's draft
    u = rng.random(n).astype(np.float32)
    if not drawn:
        tokens[1:] = np.where(rng.random(n - 1) < 0.8, p.argmax(1)[:-1], tokens[1:])
    t, d = held(target, dtype, pad=0 if vocab % 2 else 3), held(q, dtype) if drawn else None
    seen = check_verify(esa, t, tokens, cu, u, d)
    for special in (0.0, -1.0, 1.0, 2.0, float("nan")):           # drawing with the ends of the range and beyond
        v = u.copy()
        v[cu[:-1][np.diff(cu) > 0]] = special
        check_verify(esa, t, tokens, cu, v, d)
    if drafts > 100 and drawn:
        assert len(seen[0]) > 65


@pytest.mark.parametrize("vocab", [3, 5000, 17001, 50001])
def test_verify_counts_what_is_no_probability_as_nothing(esa, vocab):
    rng = np.random.default_rng(31)
    for dtype in ("f32", "bf16"):
        for drawn in (True, False):
            n = 1200 if vocab == 17001 else 60
            cu, tokens, u = np.arange(0, n + 1, 4), rng.integers(0, min(vocab, 50), n), rng.random(n).astype(np.float32)
            p, q = (x[:, rng.permutation(vocab)] for x in distributions(rng, n, vocab))
            for x in (p, q):
                x[rng.random(x.shape) < 0.2] = float("nan")
                x[rng.random(x.shape) < 0.1] = float("inf")
                x[rng.random(x.shape) < 0.1] = -0.5
                x[rng.random(x.shape) < 0.2] = 0.0
            check_verify(esa, held(p, dtype), tokens, cu, u, held(q, dtype) if drawn else None)


@pytest.mark.parametrize("vocab", [1000, 20001])
@pytest.mark.parametrize("power", [-140, -126, 120])
def test_verify_weights_of_any_size(esa, vocab, power):
    """Rows that sum to anything: subnormal numbers count, and sums leave fp32's range."""
    rng = np.random.default_rng(36)
    n, cu = 24, [0, 4, 8, 12, 16, 20, 24]
    p, q = (x * 2.0 ** power for x in distributions(rng, n, vocab))
    tokens = np.array([rng.choice(vocab, p=x / x.sum()) for x in q])
    for dtype in ("f32", "bf16"):
        for drawn in (True, False):
            check_verify(esa, held(np.roll(p, -1, 0), dtype), tokens, cu, rng.random(n).astype(np.float32), held(q, dtype) if drawn else None)


@pytest.mark.parametrize("vocab", [5, 9000, 50001, 300007])
def test_verify_where_nothing_is_left(esa, vocab):
    """Differences that are nowhere positive: the target's own row; a row without any probability: no token."""
    rng = np.random.default_rng(32)
    cu = [0, 3, 6, 7, 9]
    p = distributions(rng, 9, vocab)[0]
    q = np.ones_like(p)                                           # turns every draft down, and leaves nothing
    tokens, u = rng.integers(0, vocab, 9), np.full(9, 0.999, dtype=np.float32)
    check_verify(esa, held(p, "f32"), tokens, cu, u, held(q, "f32"))
    p[[3, 6]] = 0.0
    want = check_verify(esa, held(p, "f32"), tokens, cu, u, held(q, "f32"))
    assert want[1] == [-1] and want[2] == [-1]
    p[:] = 0.0
    p[:, vocab - 1] = 1.0                                              # a draft that was looked up and is sure to be right
    tokens[:] = vocab - 1
    want = check_verify(esa, held(p, "f32"), tokens, cu, u, None)
    assert want[0] == [vocab - 1] * 3
    u[:] = 1.0                                                    # turned down, and all of p with it: p itself
    assert check_verify(esa, held(p, "f32"), tokens, cu, u, None)[0] == [vocab - 1]


def test_verify_tokens_outside_the_vocabulary(esa):
    rng = np.random.default_rng(33)
    p, q = distributions(rng, 8, 300)
    for drawn in (True, False):
        for bad in (-1, 300, 2 ** 31 - 1, -2 ** 31):
            tokens = np.full(8, 5)
            tokens[2], tokens[5] = bad, bad
            check_verify(esa, held(p, "f32"), tokens, [0, 4, 8], np.linspace(0, 0.9, 8, dtype=np.float32), held(q, "f32") if drawn else None)


@pytest.mark.parametrize("vocab", [700, 20000])
def test_verify_offsets_of_any_content(esa, vocab):
    """cu that does not ascend or leads out of the rows is clamped; nothing outside the outputs is written."""
    rng = np.random.default_rng(34)
    p, q = (held(x, "f32") for x in distributions(rng, 6, vocab))
    for _ in range(20):
        keep = Guarded()
        cu = keep(rng.choice([-2 ** 31, -5, 0, 1, 2, 4, 6, 9, 2 ** 31 - 1], 9))
        out, count = keep(np.zeros(6)), keep(np.zeros(8))
        esa.esa_verify_drafts(p, keep(rng.integers(-2, vocab + 100, 6)), cu, torch.rand(6, device="cuda"), draft=q, out=out, count=count)
        keep.check()
        assert torch.all((out >= -1) & (out < vocab)) and torch.all((count >= 0) & (count <= 6))


def test_verify_without_rows(esa):
    p = torch.zeros((0, 50), device="cuda")
    out, count = esa.esa_verify_drafts(p, ints([]), ints([0, 0, 0]), ints([], torch.float32))
    assert out.numel() == 0 and count.tolist() == [0, 0]
    out, count = esa.esa_verify_drafts(torch.zeros((2, 50), device="cuda"), ints([0, 0]), ints([0]), ints([0, 0], torch.float32))
    assert count.numel() == 0


def test_verify_far_rows(esa):
    """Rows of probabilities beyond 32 bits, and a sequence's rows as views of a larger array."""
    rng = np.random.default_rng(35)
    p, q = distributions(rng, 6, 1001)
    whole = [torch.empty((6, 1 << 28), dtype=torch.float32, device="cuda")[:, 5:1006] for _ in "pq"]
    for w, x in zip(whole, (p, q)):
        w.copy_(torch.from_numpy(x))
    check_verify(esa, whole[0], rng.integers(0, 1001, 6), [0, 3, 6], rng.random(6).astype(np.float32), whole[1])


@pytest.mark.parametrize("vocab", [40, 16400])
def test_verify_many_sequences(esa, vocab):
    """More of them than a launch has workgroups in one dimension of its grid."""
    n = 70000
    g = torch.Generator("cuda").manual_seed(5)
    sure = torch.randint(0, vocab, (n,), generator=g, device="cuda")
    p = torch.zeros((n, vocab), dtype=torch.bfloat16, device="cuda").scatter_(1, sure[:, None], 1.0)
    # two rows a sequence: drafts that are sure to stand, or sure not to
    tokens = torch.where(torch.arange(n, device="cuda") % 4 < 2, sure.roll(1), (sure.roll(1) + 1) % vocab).int()
    cu = torch.arange(0, n + 1, 2, dtype=torch.int32, device="cuda")
    u = torch.rand(n, generator=g, device="cuda")
    out, count = esa.esa_verify_drafts(p, tokens, cu, u)
    stands = torch.arange(n // 2, device="cuda") % 2 == 0
    assert torch.equal(count, torch.where(stands, 2, 1).int())
    want = sure.int().view(-1, 2).clone()
    want[~stands, 1] = -1
    assert torch.equal(out.view(-1, 2), want)
    one = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    out, count = esa.esa_verify_drafts(p, tokens, one, u)
    assert torch.equal(out, sure.int()) and torch.all(count == 1)
