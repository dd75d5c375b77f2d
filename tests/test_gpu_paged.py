"""esa_append_paged and esa_attend_paged against their float64 definitions.  Everything in a pool that no sequence has is NaN."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import paged_oracle as orc
from paged_support import TYPES, Pool, check_attention, f64

pytestmark = pytest.mark.gpu
BASE = 5e5
# Probabilities are rounded to bf16 where a matrix-core kernel takes them as one term; the bound allows it for bf16 everywhere.
P_STEP = {"bf16": 2.0 ** -8, "f32": 0.0}


@pytest.fixture(scope="module")
def esa():
    import paper_2502_14477_amd as lib
    return lib


# ---------------------------------------------------------------- appending
RAGGED = [(0, 1), (63, 1), (64, 3), (5, 0), (17, 200), (0, 129), (1000, 31), (15, 1)]


def appended(esa, pool, k, v, q, base=BASE, **kw):
    return esa.esa_append_paged(k, v, *pool.batch(), q=q, rope_base=base, **kw)


def in_storage(x, dtype):
    """x rounded once: 8 (bf16) or 24 significant bits, ties to even."""
    _, e = np.frexp(x)
    step = np.exp2(e.astype(np.float64) - (8 if dtype == "bf16" else 24))
    return np.rint(x / step) * step


@pytest.mark.parametrize("dtype,held", [("bf16", "e4m3"), ("bf16", "same"), ("f32", "e4m3"), ("f32", "same")])
@pytest.mark.parametrize("h,h_kv,d,page,major", [(8, 2, 64, 16, False), (4, 1, 32, 64, True), (8, 4, 128, 128, False), (2, 2, 256, 32, True), (32, 8, 128, 64, False)])
def test_append(esa, dtype, held, h, h_kv, d, page, major):
    print("[case] append", dtype, held, h, h_kv, d, page, major, flush=True)
    pool = Pool(RAGGED, h_kv, d, page, dtype, held, seed=3, token_major=major).fill((0.3, 1.0))
    k, v, q = pool.rows(pool.n_tok, h_kv, 2.0), pool.rows(pool.n_tok, h_kv), pool.rows(pool.n_tok, h)
    before = pool.values()
    got_q = appended(esa, pool, k, v, q)
    pos = np.concatenate([t0 + np.arange(n) for t0, n in RAGGED])
    rows = {"q": in_storage(orc.turn(f64(q), pos, BASE), dtype), "k": in_storage(orc.turn(f64(k), pos, BASE), dtype), "v": f64(v)}
    assert np.array_equal(f64(got_q), rows["q"])
    want_k, want_v, want_ks, want_vs = before
    row0 = 0
    for b, (t0, n) in enumerate(RAGGED):
        for name, values, scale in (("k", want_k, want_ks), ("v", want_v, want_vs)):
            new = rows[name][row0:row0 + n]
            if held == "e4m3":
                orc.append_blocks(values, scale, new, t0, pool.table[b], page)
            else:
                for i in range(n):
                    values[pool.table[b, (t0 + i) // page], :, (t0 + i) % page] = new[i]
        row0 += n
    after = pool.values()
    for i, name in enumerate(("k", "v", "k_scale", "v_scale")):
        if after[i] is not None:
            assert np.array_equal(after[i], (want_k, want_v, want_ks, want_vs)[i], equal_nan=name in "kv"), name


def test_append_in_steps_gives_the_same_rows(esa):
    """A prompt at once, or token by token: the same numbers but for e4m3's subnormals, which a growing scale may round twice."""
    n, page = 100, 32
    whole, steps = (Pool([(0, n)], 2, 128, page, seed=5) for _ in range(2))
    k, v = whole.rows(n, 2, 1.0), whole.rows(n, 2, 1.0)
    k[40] *= 50
    appended(esa, whole, k, v, None)
    at = 0
    for m in (1, 1, 30, 9, 1, 20, 38):
        cu, start = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, m], [at]))
        esa.esa_append_paged(k[at:at + m], v[at:at + m], cu, start, *steps.batch()[2:], rope_base=BASE)
        at += m
    assert at == n
    for a, b in zip(whole.values(), steps.values()):
        used = whole.table[0, :4]
        if a.ndim == 2:
            assert np.array_equal(a[used], b[used])
        else:
            x, y = a[used][:, :, :page], b[used]
            assert np.array_equal(np.isnan(x), np.isnan(y))
            x, y = np.nan_to_num(x), np.nan_to_num(y)
            assert np.all((x == y) | ((np.abs(x) <= 2.0 ** -6) & (np.abs(x - y) <= 2.0 ** -9)))


def test_append_values_at_the_ends_of_the_range(esa):
    """Zeros, the smallest and largest numbers, infinities and NaN: a block holds what its scale can, NaN as NaN."""
    d, page = 64, 16
    sizes = [0.0, 1e-38, 1e-30, 2.0 ** -96, 1.0, 448.0, 449.0, 3e38, 2.0 ** 118]
    pool = Pool([(0, 1)] * len(sizes), 1, d, page, "bf16", "e4m3")
    v = torch.ones(len(sizes), 1, d) * torch.tensor(sizes)[:, None, None] * torch.linspace(-1, 1, d)
    v = v.to(torch.bfloat16).cuda()
    v[4, 0, 5], v[5, 0, 6] = float("nan"), float("inf")
    esa.esa_append_paged(v, v, *pool.batch())
    values, _, scale, _ = pool.values()
    for b in range(len(sizes)):
        page_of = pool.table[b, 0]
        x = f64(v[b, 0])
        finite = np.where(np.isnan(x), 0.0, x)
        byte = orc.scale_byte(float(np.max(np.abs(finite))))
        assert scale[page_of, 0] == byte
        assert np.array_equal(values[page_of, 0, 0], np.where(np.isnan(x), np.nan, orc.to_e4m3(finite * 2.0 ** (127 - byte))), equal_nan=True), b


@pytest.mark.parametrize("held", ["e4m3", "same"])
def test_append_leaves_out_what_has_no_page_and_what_belongs_to_nobody(esa, held):
    lengths = [(30, 40), (0, 5)]
    pool = Pool(lengths, 2, 64, 16, "bf16", held).fill()
    pool.pages[0, 3] = -1
    pool.pages[1, 0] = pool.n_pages
    k, v = pool.rows(60, 2), pool.rows(60, 2)                 # 15 rows behind the last sequence
    q = pool.rows(60, 4)
    out = torch.full_like(q, 7.0)
    before = pool.values()
    got = esa.esa_append_paged(k, v, *pool.batch(), q=q, rope_base=BASE, out_q=out)
    assert got is out and torch.all(out[45:] == 7.0) and not torch.any(out[:45] == 7.0)
    after = pool.values()
    written = {pool.table[0, p] for p in (1, 2, 4)}
    for x, y in zip(before, after):
        if x is not None:
            for p in range(pool.n_pages):
                same = np.array_equal(x[p], y[p], equal_nan=x.ndim == 4)
                assert same if p not in written else x.ndim == 2 or not same, p      # (a page may keep its scale)


def test_append_takes_slices_of_a_fused_projection_in_place(esa):
    lengths = [(3, 7), (100, 1)]
    h, h_kv, d = 4, 2, 64
    a, b = (Pool(lengths, h_kv, d, 16, "bf16", "same", seed=1) for _ in range(2))
    fused = a.rows(a.n_tok, h + 2 * h_kv)
    parts = fused[:, :h], fused[:, h:h + h_kv], fused[:, h + h_kv:]
    q = appended(esa, a, parts[1].contiguous(), parts[2].contiguous(), parts[0].contiguous())
    same = appended(esa, b, parts[1], parts[2], parts[0], out_q=parts[0])
    assert same is parts[0] and torch.equal(same, q)
    for x, y in zip(a.values()[:2], b.values()[:2]):
        assert np.array_equal(x, y, equal_nan=True)


def test_append_is_what_esa_rope_writes(esa):
    lengths = [(131000, 33)]
    pool = Pool([(0, 33)], 2, 128, 64, "bf16", "same")
    pool.pages = torch.full((1, 2048), 0, dtype=torch.int32, device="cuda")       # only the pages of the new rows matter
    pool.pages[0, 131000 // 64] = 1
    pool.pages[0, 131000 // 64 + 1] = 2
    k, v = pool.rows(33, 2), pool.rows(33, 2)
    esa.esa_append_paged(k, v, *pool.batch(first=[131000]), rope_base=BASE)
    want = esa.esa_rope(k, 131000.0, 1.0, BASE)
    t0 = lengths[0][0]
    got = torch.stack([pool.caches[0][1 if (t0 + i) // 64 == t0 // 64 else 2, :, (t0 + i) % 64] for i in range(33)])
    assert torch.equal(got, want)


# ---------------------------------------------------------------- attention
MIXED = [(0, 1), (31, 1), (32, 2), (7, 0), (300, 1), (63, 40), (0, 150), (513, 7)]


@pytest.mark.parametrize("dtype,held", [("bf16", "e4m3"), ("bf16", "same"), ("f32", "e4m3"), ("f32", "same")])
@pytest.mark.parametrize("h,h_kv,d,page,major", [(8, 2, 64, 16, False), (4, 1, 32, 64, True), (8, 4, 128, 128, False), (2, 2, 256, 32, True), (10, 2, 128, 64, True)])
@pytest.mark.parametrize("cap", [0.0, 2.0])
def test_attend(esa, dtype, held, h, h_kv, d, page, major, cap):
    print("[case] attend", dtype, held, h, h_kv, d, page, major, cap, flush=True)
    pool = Pool(MIXED, h_kv, d, page, dtype, held, seed=11, token_major=major).fill((1.5, 1.0))
    q = pool.rows(pool.n_tok, h)
    out, lse = esa.esa_attend_paged(q, *pool.batch(), cap=cap, return_lse=True)
    check_attention(pool, q, out, lse, cap=cap, p_half_step=P_STEP[dtype])


def selections(pool, l_i, l_l, n_sel, seed=2):
    rng = np.random.default_rng(seed)
    idx = np.full((len(pool.lengths), n_sel + 2), 2 ** 31 - 1, dtype=np.int32)
    idx[:, :n_sel] = -1
    for b, (t0, _) in enumerate(pool.lengths):
        i_end = min(l_i, t0)
        l_start = max(t0 - l_l, i_end)
        k = min(n_sel, l_start - i_end)
        idx[b, :k] = np.sort(rng.choice(l_start - i_end, k, replace=False)) + i_end if k else 0
        if k < n_sel:
            idx[b, k] = t0                                     # no middle token: not seen
    return torch.from_numpy(idx).to(pool.device)[:, :n_sel]    # rows further apart than they are long


@pytest.mark.parametrize("dtype,held", [("bf16", "e4m3"), ("bf16", "same"), ("f32", "e4m3"), ("f32", "same")])
@pytest.mark.parametrize("l_i,l_l,n_sel", [(16, 64, 100), (0, 0, 70), (5, 33, 0), (1000, 2, 3), (0, 2, 1)])
def test_attend_view(esa, dtype, held, l_i, l_l, n_sel):
    print("[case] view", dtype, held, l_i, l_l, n_sel, flush=True)
    pool = Pool(MIXED + [(900, 3)], 2, 128 if held == "e4m3" else 64, 32, dtype, held, seed=4).fill()
    q = pool.rows(pool.n_tok, 8)
    idx = selections(pool, l_i, l_l, n_sel) if n_sel else None
    out, lse = esa.esa_attend_paged(q, *pool.batch(), l_i=l_i, l_l=l_l, idx=idx, return_lse=True)
    check_attention(pool, q, out, lse, l_i=l_i, l_l=l_l, idx=idx, p_half_step=P_STEP[dtype])


@pytest.mark.parametrize("dtype,held,h,h_kv,d", [("bf16", "e4m3", 32, 8, 128), ("bf16", "same", 8, 8, 64), ("f32", "e4m3", 4, 1, 64), ("f32", "same", 4, 2, 128)])
@pytest.mark.parametrize("lengths", [[(5000, 1)], [(4095, 1), (77, 1), (2048, 1)], [(3500, 1), (0, 0), (1, 70), (0, 1)]], ids=["one", "three", "mixed"])
def test_attend_long(esa, dtype, held, h, h_kv, d, lengths):
    print("[case] long", dtype, held, h, h_kv, d, lengths, flush=True)
    pool = Pool(lengths, h_kv, d, 64, dtype, held, seed=6).fill((1.0, 1.0))
    q = pool.rows(pool.n_tok, h)
    out, lse = esa.esa_attend_paged(q, *pool.batch(), return_lse=True)
    check_attention(pool, q, out, lse, p_half_step=P_STEP[dtype])


@pytest.mark.parametrize("held", ["e4m3", "same"])
@pytest.mark.parametrize("l_c,h,h_kv,d", [(300, 32, 8, 128), (257, 4, 4, 64), (64, 16, 2, 128)])
def test_attend_chunk(esa, held, l_c, h, h_kv, d):
    print("[case] chunk", held, l_c, h, h_kv, d, flush=True)
    pool = Pool([(700, l_c), (1500, l_c // 2)], h_kv, d, 64, "bf16", held, seed=8).fill((1.0, 1.0))
    q = pool.rows(pool.n_tok, h)
    out, lse = esa.esa_attend_paged(q, *pool.batch(), return_lse=True)
    check_attention(pool, q, out, lse, p_half_step=P_STEP["bf16"])
    idx = selections(pool, 20, 100, 333)
    out, lse = esa.esa_attend_paged(q, *pool.batch(), l_i=20, l_l=100, idx=idx, cap=5.0, return_lse=True)
    check_attention(pool, q, out, lse, l_i=20, l_l=100, idx=idx, cap=5.0, p_half_step=P_STEP["bf16"])


@pytest.mark.parametrize("dtype,held", [("bf16", "e4m3"), ("bf16", "same"), ("f32", "e4m3"), ("f32", "same")])
@pytest.mark.parametrize("h,h_kv,d", [(8, 2, 32), (4, 1, 256)])
def test_attend_other_head_sizes(esa, dtype, held, h, h_kv, d):
    """Head sizes 32 and 256 with sequences that are cut, a chunk among them, and a view."""
    print("[case] head size", dtype, held, h, h_kv, d, flush=True)
    pool = Pool([(3500, 1), (0, 0), (700, 70), (40, 3)], h_kv, d, 32, dtype, held, seed=23).fill((1.0, 1.0))
    q = pool.rows(pool.n_tok, h)
    out, lse = esa.esa_attend_paged(q, *pool.batch(), return_lse=True)
    check_attention(pool, q, out, lse, p_half_step=P_STEP[dtype])
    idx = selections(pool, 20, 100, 333)
    out, lse = esa.esa_attend_paged(q, *pool.batch(), l_i=20, l_l=100, idx=idx, cap=5.0, return_lse=True)
    check_attention(pool, q, out, lse, l_i=20, l_l=100, idx=idx, cap=5.0, p_half_step=P_STEP[dtype])


# Chunks whose keys are shared out over the workgroups: blocks cut in many places or left whole, blocks of a few rows, groups of heads that
# do not divide a block, sequences that another kernel serves in between.
SHARED = {
    "one long": [(6000, 70)], "from the beginning": [(0, 1300)], "short ones": [(200, 65), (0, 80), (31, 100), (1, 64), (450, 90)],
    "ragged": [(3000, 300), (40, 600), (0, 33), (2500, 1), (700, 129)], "just over a block": [(1000, 129), (999, 257), (63, 65)],
}


@pytest.mark.parametrize("held", ["e4m3", "same"])
@pytest.mark.parametrize("h,h_kv,d,page", [(4, 1, 64, 32), (2, 2, 128, 64), (10, 2, 64, 128), (16, 1, 128, 16)])
@pytest.mark.parametrize("name", sorted(SHARED))
def test_attend_shares_blocks(esa, held, h, h_kv, d, page, name):
    print("[case] shares", held, h, h_kv, d, page, name, flush=True)
    lengths = [(t0, -(-n * 2 // (h // h_kv))) for t0, n in SHARED[name]]      # rows of a KV head: twice n, a block has 256
    pool = Pool(lengths, h_kv, d, page, "bf16", held, seed=20).fill((1.0, 1.0))
    q = pool.rows(pool.n_tok, h)
    out, lse = esa.esa_attend_paged(q, *pool.batch(), return_lse=True)
    check_attention(pool, q, out, lse, p_half_step=P_STEP["bf16"])


@pytest.mark.parametrize("held,cap", [("e4m3", 0.0), ("same", 3.0)])
def test_attend_of_random_batches(esa, held, cap):
    for seed in range(12):
        rng = np.random.default_rng(100 + seed)
        lengths = [(int(rng.integers(0, 10 ** rng.integers(1, 4))), int(rng.integers(0, 6 if rng.random() < 0.4 else 260))) for _ in range(rng.integers(1, 9))]
        if sum(n for _, n in lengths) == 0:
            continue
        print("[case] random", held, cap, seed, lengths, flush=True)
        pool = Pool(lengths, 1, 64, int(rng.choice([16, 32, 64, 128])), "bf16", held, seed=seed).fill((1.0, 1.0))
        q = pool.rows(pool.n_tok, 4)
        out, lse = esa.esa_attend_paged(q, *pool.batch(), cap=cap, return_lse=True)
        check_attention(pool, q, out, lse, cap=cap, p_half_step=P_STEP["bf16"])
        idx = selections(pool, 7, 50, 60, seed=seed)
        out, lse = esa.esa_attend_paged(q, *pool.batch(), l_i=7, l_l=50, idx=idx, cap=cap, return_lse=True)
        check_attention(pool, q, out, lse, l_i=7, l_l=50, idx=idx, cap=cap, p_half_step=P_STEP["bf16"])


@pytest.mark.parametrize("dtype,held", [("bf16", "e4m3"), ("bf16", "same"), ("f32", "same")])
def test_attend_with_large_and_far_apart_logits(esa, dtype, held):
    """Logits of some hundreds: the running maximum moves by more than an exponential's range, in both directions."""
    pool = Pool([(700, 1), (500, 90)], 2, 128, 64, dtype, held, seed=9).fill((12.0, 1.0))
    q = pool.rows(pool.n_tok, 8, 12.0)
    out, lse = esa.esa_attend_paged(q, *pool.batch(), return_lse=True)
    check_attention(pool, q, out, lse, p_half_step=P_STEP[dtype])
    out, lse = esa.esa_attend_paged(q, *pool.batch(), cap=30.0, return_lse=True)
    check_attention(pool, q, out, lse, cap=30.0, p_half_step=P_STEP[dtype])


@pytest.mark.parametrize("dtype,held", [("bf16", "e4m3"), ("bf16", "same"), ("f32", "same")])
def test_attend_with_large_values_and_caps(esa, dtype, held):
    """Values of some 2^87, and the largest cap."""
    pool = Pool([(700, 1), (500, 90)], 2, 128, 64, dtype, held, seed=24).fill((4.0, 2.0 ** 85))
    q = pool.rows(pool.n_tok, 8, 3.0)
    for cap in (0.0, 4096.0):
        out, lse = esa.esa_attend_paged(q, *pool.batch(), cap=cap, return_lse=True)
        check_attention(pool, q, out, lse, cap=cap, p_half_step=P_STEP[dtype])


@pytest.mark.parametrize("dtype,held", [("bf16", "e4m3"), ("bf16", "same"), ("f32", "e4m3")])
@pytest.mark.parametrize("new", [1, 100])
def test_attend_with_logits_that_rise_towards_the_end(esa, dtype, held, new):
    """Every key's logit is larger than those before it: the softmax's reference moves again and again, by more than its lag each time."""
    pool = Pool([(900, new)], 1, 64, 64, dtype, held, seed=23).fill((0.01, 1.0))
    direction = torch.zeros(64)
    direction[5] = 1.0
    at = torch.arange(900 + new)
    rise = (at.double() / 4).to(TYPES[dtype])                    # logits 0 .. 250 in steps
    host = pool.caches[0].cpu()
    if held == "e4m3":
        pool.scales[0].fill_(127)
        x = torch.zeros(pool.caches[0].shape)
        for p in range(-(-(900 + new) // 64)):
            rows = rise[p * 64:(p + 1) * 64].float()
            x[pool.table[0, p], 0, :len(rows), 5] = rows
        pool.caches[0].view(torch.uint8).copy_(x.to(torch.float8_e4m3fn).view(torch.uint8))
    else:
        for p in range(-(-(900 + new) // 64)):
            rows = rise[p * 64:(p + 1) * 64]
            host[pool.table[0, p], 0, :len(rows)] = 0
            host[pool.table[0, p], 0, :len(rows), 5] = rows
        pool.caches[0].copy_(host)
    q = (torch.ones(new, 4, 64) * direction).to(TYPES[dtype]).cuda()
    out, lse = esa.esa_attend_paged(q, *pool.batch(), scale=1.0, return_lse=True)
    check_attention(pool, q, out, lse, scale=1.0, p_half_step=P_STEP[dtype])


@pytest.mark.parametrize("held", ["e4m3", "same"])
@pytest.mark.parametrize("l_c", [1, 100])
def test_attend_with_missing_pages(esa, held, l_c):
    """Positions without a page are not seen; a token that sees nothing has 0 and -inf; rows that belong to nobody stay."""
    lengths = [(100, l_c), (40, l_c), (16 * 7, l_c)]
    pool = Pool(lengths, 2, 64, 16, "bf16", held, seed=10).fill()
    pool.pages[0, 2] = -1
    pool.pages[0, 0] = pool.n_pages
    pool.pages[1] = -5
    pool.pages = pool.pages[:, :7].contiguous()               # the third sequence's last positions lie behind the table
    q = pool.rows(pool.n_tok + 9, 4)
    out = torch.full_like(q, 3.0)
    got, lse = esa.esa_attend_paged(q, *pool.batch(), out=out, return_lse=True)
    assert got is out and torch.all(out[pool.n_tok:] == 3.0)
    second = slice(l_c, 2 * l_c)
    assert torch.all(out[second] == 0) and torch.all(lse[second] == float("-inf"))
    qf = f64(q)
    for b in (0, 2):
        t0 = lengths[b][0]
        at = [p for p in range(min(t0 + l_c, 7 * 16)) if b == 2 or p // 16 not in (0, 2)]
        k, v = pool.seen(b, at)
        rows = slice(b * l_c, (b + 1) * l_c)
        want, want_lse, spread, most = orc.attend(qf[rows], t0, k, v, at, 1 / 8)
        share = 2 * (2.0 ** -8 + (64 + 16 + 2 * most) * 2.0 ** -21 + 300 * 2.0 ** -24)
        assert np.all(np.abs(f64(out[rows]) - want) <= 2.0 ** -8 * np.abs(want) + share[..., None] * spread)
        assert np.all(np.abs(f64(lse[rows]) - want_lse) <= share)


def test_attend_of_positions_listed_twice_counts_them_twice(esa):
    pool = Pool([(200, 2)], 1, 128, 64, "bf16", "e4m3", seed=12).fill()
    q = pool.rows(2, 4)
    idx = torch.tensor([[50, 50, 51, 7, -1, 300]], dtype=torch.int32, device="cuda")
    out, lse = esa.esa_attend_paged(q, *pool.batch(), l_i=10, l_l=20, idx=idx, return_lse=True)
    check_attention(pool, q, out, lse, l_i=10, l_l=20, idx=idx, p_half_step=P_STEP["bf16"])


def test_offsets_beyond_32_bits(esa):
    """A pool of over 2^32 bytes, the sequences' pages at its end."""
    h_kv, d, page = 2, 128, 128
    n_pages = (1 << 32) // (h_kv * d * page) + 40
    k_cache, v_cache = (torch.empty((n_pages, h_kv, page, d), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in "kv")
    k_scale, v_scale = (torch.empty((n_pages, h_kv), dtype=torch.uint8, device="cuda") for _ in "kv")
    pool = Pool([(0, 300), (0, 200)], h_kv, d, page, "bf16", "e4m3", seed=13)
    far = torch.where(pool.pages < pool.n_pages, n_pages - 1 - pool.pages, pool.pages)
    k, v, q = pool.rows(500, h_kv), pool.rows(500, h_kv), pool.rows(500, 4)
    got = []
    for batch in (pool.batch(), (pool.cu, pool.start, far, k_cache, v_cache, k_scale, v_scale)):
        turned = esa.esa_append_paged(k, v, *batch, q=q, rope_base=BASE)
        got.append(esa.esa_attend_paged(turned, *batch))
        step = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
        got.append(esa.esa_attend_paged(turned[[299, 499]].contiguous(), step, torch.tensor([299, 199], dtype=torch.int32, device="cuda"), *batch[2:]))
    assert torch.equal(got[0], got[2]) and torch.equal(got[1], got[3])


@pytest.mark.parametrize("lengths", [[(2000, 1), (500, 3)], [(100, 90), (40, 70)]], ids=["few rows", "many"])
def test_attend_with_more_heads_than_workgroups_at_a_time(esa, lengths):
    pool = Pool(lengths, 600, 64, 64, "bf16", "same", seed=25).fill((1.0, 1.0))
    q = pool.rows(pool.n_tok, 600)
    out, lse = esa.esa_attend_paged(q, *pool.batch(), return_lse=True)
    check_attention(pool, q, out, lse, p_half_step=P_STEP["bf16"])


@pytest.mark.parametrize("dtype,held,d", [("bf16", "e4m3", 128), ("bf16", "same", 64), ("f32", "same", 256), ("f32", "e4m3", 32)])
def test_attend_takes_and_writes_parts_of_larger_tensors(esa, dtype, held, d):
    """Queries out of a fused projection, results into it, index list and table out of wider ones, another scale; the rest stays as it is."""
    pool = Pool([(900, 1), (300, 80), (0, 0)], 2, d, 32, dtype, held, seed=26).fill((1.0, 1.0))
    h, n = 8, pool.n_tok + 3                                      # rows behind the last sequence
    fused = pool.rows(n, 3 * h)
    q, out = fused[:, :h], fused[:, h:2 * h]
    before = fused.clone()
    idx = selections(pool, 20, 50, 60)
    wide = torch.full((3, 100), -1, dtype=torch.int32, device="cuda")
    wide[:, :60] = idx
    table = torch.full((3, pool.pages.shape[1] + 5), -1, dtype=torch.int32, device="cuda")
    table[:, :pool.pages.shape[1]] = pool.pages
    batch = list(pool.batch())
    batch[2] = table[:, :pool.pages.shape[1]]
    got, lse = esa.esa_attend_paged(q, *batch, l_i=20, l_l=50, idx=wide[:, :60], scale=0.03, out=out, return_lse=True)
    assert got is out
    check_attention(pool, q[:pool.n_tok], out[:pool.n_tok], lse[:pool.n_tok], l_i=20, l_l=50, idx=idx, scale=0.03, p_half_step=P_STEP[dtype])
    assert torch.equal(fused[:, :h], before[:, :h]) and torch.equal(fused[:, 2 * h:], before[:, 2 * h:]) and torch.equal(out[pool.n_tok:], before[pool.n_tok:, h:2 * h])


def test_many_sequences(esa):
    """More sequences than a wave has lanes, some of them idle."""
    rng = np.random.default_rng(14)
    lengths = [(int(rng.integers(0, 150)), int(rng.integers(0, 3))) for _ in range(203)]
    pool = Pool(lengths, 1, 64, 16, "bf16", "e4m3", seed=15).fill()
    k, v, q = pool.rows(pool.n_tok, 1), pool.rows(pool.n_tok, 1), pool.rows(pool.n_tok, 4)
    turned = appended(esa, pool, k, v, q)
    out, lse = esa.esa_attend_paged(turned, *pool.batch(), return_lse=True)
    check_attention(pool, turned, out, lse, p_half_step=P_STEP["bf16"])


@pytest.mark.parametrize("dtype,held", [("bf16", "e4m3"), ("f32", "same")])
@pytest.mark.parametrize("n_seq", [64, 65, 128, 1000, 4200])
def test_sequences_in_groups_of_64(esa, dtype, held, n_seq):
    """Single tokens, most of them with few keys or idle, some with so many that they are cut."""
    print("[case] groups", dtype, held, n_seq, flush=True)
    rng = np.random.default_rng(n_seq)
    lengths = [(int(rng.integers(0, 40)), int(rng.random() < 0.8)) for _ in range(n_seq)]
    for b in (0, 3, 62, 63, n_seq // 2, n_seq - 1):
        lengths[b] = (int(rng.integers(600, 4000)), 1)
    pool = Pool(lengths, 2, 64, 64, dtype, held, seed=21).fill((1.0, 1.0))
    q = pool.rows(pool.n_tok, 4)
    out, lse = esa.esa_attend_paged(q, *pool.batch(), return_lse=True)
    check_attention(pool, q, out, lse, p_half_step=P_STEP[dtype])


@pytest.mark.parametrize("held", ["e4m3", "same"])
@pytest.mark.parametrize("n_seq", [65, 150, 300])
def test_chunks_in_groups_of_64(esa, held, n_seq):
    print("[case] chunk groups", held, n_seq, flush=True)
    rng = np.random.default_rng(n_seq)
    lengths = [(int(rng.integers(0, 60)), int(rng.integers(0, 2 if b % 3 else 50))) for b in range(n_seq)]
    for b in (1, 63, 64, n_seq - 1):
        lengths[b] = (int(rng.integers(600, 2000)), int(rng.integers(1, 200)))
    pool = Pool(lengths, 1, 64, 32, "bf16", held, seed=22).fill((1.0, 1.0))
    q = pool.rows(pool.n_tok, 8)
    out, lse = esa.esa_attend_paged(q, *pool.batch(), return_lse=True)
    check_attention(pool, q, out, lse, p_half_step=P_STEP["bf16"])


# ---------------------------------------------------------------- as a program uses them
def test_results_are_the_same_every_time_and_on_every_stream(esa):
    pool = Pool([(3000, 1), (100, 64), (1, 1)], 8, 128, 64, "bf16", "e4m3", seed=16).fill()
    other = Pool([(2000, 9)], 2, 64, 32, "bf16", "same", seed=17).fill()
    q, q2 = pool.rows(pool.n_tok, 32), other.rows(9, 8)
    first, first2 = esa.esa_attend_paged(q, *pool.batch()), esa.esa_attend_paged(q2, *other.batch())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(5):
        with torch.cuda.stream(streams[0]):
            got.append((esa.esa_attend_paged(q, *pool.batch()), first))
        with torch.cuda.stream(streams[1]):
            got.append((esa.esa_attend_paged(q2, *other.batch()), first2))
    torch.cuda.synchronize()
    for a, b in got:
        assert torch.equal(a, b)


@pytest.mark.parametrize("held", ["e4m3", "same"])
def test_a_captured_step_follows_the_lengths_it_finds(esa, held):
    """One graph of append and attention, replayed as the sequences grow (and one of them pauses), against eager calls on another pool;
    a second graph on the same pool is replayed in between."""
    room, steps, h, h_kv, d = [(0, 90), (0, 400), (0, 33)], 12, 8, 2, 128
    pools = [Pool(room, h_kv, d, 16, "bf16", held, seed=18) for _ in range(2)]
    lengths = [70, 380, 16]
    k, v = pools[0].rows(sum(lengths), h_kv), pools[0].rows(sum(lengths), h_kv)
    cu = torch.tensor([0, 70, 450, 466], dtype=torch.int32, device="cuda")
    for p in pools:
        esa.esa_append_paged(k, v, cu, torch.zeros(3, dtype=torch.int32, device="cuda"), *p.batch()[2:], rope_base=BASE)
    kn, vn, qn = (torch.zeros(3, n, d, dtype=torch.bfloat16, device="cuda") for n in (h_kv, h_kv, h))
    cu, start = torch.tensor([0, 1, 2, 3], dtype=torch.int32, device="cuda"), torch.tensor(lengths, dtype=torch.int32, device="cuda")

    def step(pool, q, k, v):
        turned = esa.esa_append_paged(k, v, cu, start, *pool.batch()[2:], q=q, rope_base=BASE)
        return esa.esa_attend_paged(turned, cu, start, *pool.batch()[2:])

    def look(pool, q):
        return esa.esa_attend_paged(q, cu, start, *pool.batch()[2:], l_i=4, l_l=30)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        look(pools[0], qn)
    torch.cuda.current_stream().wait_stream(side)
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    with torch.cuda.graph(graphs[0]):
        captured = step(pools[0], qn, kn, vn)
    with torch.cuda.graph(graphs[1]):
        looked = look(pools[0], qn)
    for i in range(steps):
        counts = [1, 0 if i % 3 == 0 else 1, 1]
        cu.copy_(torch.tensor(np.concatenate(([0], np.cumsum(counts))), dtype=torch.int32))
        start.copy_(torch.tensor(lengths, dtype=torch.int32))
        for t, n in ((kn, h_kv), (vn, h_kv), (qn, h)):
            t.copy_(pools[0].rows(3, n))
        graphs[0].replay()
        graphs[1].replay()
        rows = sum(counts)
        assert torch.equal(captured[:rows], step(pools[1], qn, kn, vn)[:rows])
        assert torch.equal(looked[:rows], look(pools[1], qn)[:rows])
        lengths = [a + n for a, n in zip(lengths, counts)]


@pytest.mark.parametrize("held", ["e4m3", "same"])
def test_esa_steps_over_a_paged_cache(esa, held):
    """Chunks and decode steps of one sequence: append with rotation, compress, score and select, attend through the pages.  With pages in
    the storage type the attention is esa_attend_indexed's on a contiguous cache; with 8 bits it is the definition's on what the pages hold."""
    h, h_kv, d, d_c, l_i, l_l, k_sel = 8, 2, 128, 64, 16, 64, 100
    chunks = [128, 128, 128, 100, 1, 1, 1]
    total = sum(chunks)
    pool = Pool([(0, total)], h_kv, d, 32, "bf16", held, seed=19)
    Wk = esa.esa_pack_weights((torch.randn(h_kv * d, d_c, device="cuda") / 16).to(torch.bfloat16))
    Wq = esa.esa_pack_weights((torch.randn(h * d, d_c, device="cuda") / 32).to(torch.bfloat16))
    kc = torch.zeros(total, d_c, dtype=torch.bfloat16, device="cuda")
    flat_k, flat_v = (torch.zeros(total, h_kv, d, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    t0 = 0
    for n in chunks:
        q, k, v = pool.rows(n, h), pool.rows(n, h_kv), pool.rows(n, h_kv)
        cu, start = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, n], [t0]))
        batch = (cu, start, *pool.batch()[2:])
        q = esa.esa_append_paged(k, v, *batch, q=q, rope_base=BASE)
        flat_k[t0:t0 + n], flat_v[t0:t0 + n] = esa.esa_rope(k, float(t0), 1.0, BASE), v
        qc, _ = esa.esa_compress_qk(q, Wq, flat_k[t0:t0 + n], Wk, out_k=kc[t0:t0 + n])
        i_end, l_start = esa.esa_segments(t0, l_i, l_l)
        idx = None
        if l_start > i_end:
            _, idx, _, _ = esa.esa_score_select_gather(qc, kc, i_end, l_start, k_sel)
        rows = None if idx is None else idx[None]
        out, lse = esa.esa_attend_paged(q, *batch, l_i=l_i, l_l=l_l, idx=rows, return_lse=True)
        pool.lengths = [(t0, n)]
        check_attention(pool, q, out, lse, l_i=l_i, l_l=l_l, idx=rows, p_half_step=P_STEP["bf16"])
        if held == "same":
            want = esa.esa_attend_indexed(q, flat_k, flat_v, t0, l_i, l_l, idx)
            # two kernels, each within its own bound of the definition: outputs of unit-size values differ by a rounding of each and by
            # probabilities' roundings, 2 (2^-8 + 2^-8) of sum p|v| <= max|v|
            assert float((out.float() - want.float()).abs().max()) <= 2.0 ** -6 * float(flat_v.float().abs().max())
        t0 += n
