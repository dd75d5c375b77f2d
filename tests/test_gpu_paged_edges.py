"""Calls of the paged cache at the ends of what its header allows."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import paged_oracle as orc
from paged_support import TYPES, Pool, check_attention, f64

pytestmark = pytest.mark.gpu
BASE = 5e5
P_STEP = {"bf16": 2.0 ** -8, "f32": 0.0}      # probabilities of chunks of head size 128 are rounded to bf16


@pytest.fixture(scope="module")
def esa():
    import paper_2502_14477_amd as lib
    return lib


def step_and_look(esa, batch, k, v, q, lengths):
    """A chunk of every sequence, then a token of each: turned queries, the attention of both."""
    turned = esa.esa_append_paged(k, v, *batch, q=q, rope_base=BASE)
    out, lse = esa.esa_attend_paged(turned, *batch, return_lse=True)
    ends = torch.tensor(lengths).cumsum(0) - 1
    cu = torch.arange(len(lengths) + 1, dtype=torch.int32, device="cuda")
    start = torch.tensor([n - 1 for n in lengths], dtype=torch.int32, device="cuda")
    one, one_lse = esa.esa_attend_paged(turned[ends.tolist()].contiguous(), cu, start, *batch[2:], return_lse=True)
    return turned, out, lse, one, one_lse


@pytest.mark.parametrize("dtype,held,d", [("bf16", "e4m3", 128), ("bf16", "same", 64), ("f32", "e4m3", 64)])
@pytest.mark.parametrize("order", ["tokens", "heads"])
def test_rows_and_heads_beyond_32_bits(esa, dtype, held, d, order):
    """A pool whose outermost dimension is a page's positions, or its heads: rows of one page lie up to 12 GB apart."""
    print("[case] far rows", dtype, held, d, order, flush=True)
    lengths, page, h_kv = [300, 200], 64, 8
    pool = Pool([(0, n) for n in lengths], h_kv, d, page, dtype, held, seed=41)
    at = torch.uint8 if held == "e4m3" else TYPES[dtype]
    tok_bytes = 190 << 20                                        # 24 of them are more than 2^32
    n_pages = tok_bytes // (h_kv * d * torch.empty(0, dtype=at).element_size())
    shape, back = {"tokens": ((page, n_pages, h_kv, d), (1, 2, 0, 3)), "heads": ((h_kv, n_pages, page, d), (1, 0, 2, 3))}[order]
    caches = [torch.empty(shape, dtype=at, device="cuda").permute(back) for _ in "kv"]
    if held == "e4m3":
        caches = [c.view(torch.float8_e4m3fn) for c in caches]
    scales = [torch.empty((n_pages, h_kv), dtype=torch.uint8, device="cuda") if held == "e4m3" else None for _ in "kv"]
    far = torch.where(pool.pages < pool.n_pages, n_pages - 1 - pool.pages, pool.pages)
    k, v, q = pool.rows(pool.n_tok, h_kv), pool.rows(pool.n_tok, h_kv), pool.rows(pool.n_tok, 16)
    near = step_and_look(esa, pool.batch(), k, v, q, lengths)
    there = step_and_look(esa, (pool.cu, pool.start, far, *caches, *scales), k, v, q, lengths)
    # one order of summation, whichever way a tile's rows are found
    for a, b in zip(near, there):
        assert torch.equal(a, b)
    used = pool.table[0, :len(range(0, lengths[0], page)) - 1]   # whole pages of the first sequence: what the pools hold is the same
    for a, b in zip(pool.caches, caches):
        raw = [c.view(torch.uint8) if held == "e4m3" else c for c in (a, b)]
        rows = torch.from_numpy(used).long().cuda()
        assert torch.equal(raw[0][rows], raw[1][n_pages - 1 - rows])


def test_a_growing_scale_reaches_rows_beyond_32_bits(esa):
    """Earlier rows of a block are brought to a larger scale wherever they lie."""
    page, h_kv, d = 64, 8, 128
    pool = Pool([(0, 60)], h_kv, d, page, "bf16", "e4m3", seed=42)
    n_pages = (190 << 20) // (h_kv * d)
    caches = [torch.empty((page, n_pages, h_kv, d), dtype=torch.uint8, device="cuda").permute(1, 2, 0, 3).view(torch.float8_e4m3fn) for _ in "kv"]
    scales = [torch.empty((n_pages, h_kv), dtype=torch.uint8, device="cuda") for _ in "kv"]
    far = torch.where(pool.pages < pool.n_pages, n_pages - 1 - pool.pages, pool.pages)
    k, v = pool.rows(60, h_kv), pool.rows(60, h_kv)
    k[55:] *= 64
    for cu, start, rows in (([0, 50], [0], slice(0, 50)), ([0, 10], [50], slice(50, 60))):
        cu, start = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (cu, start))
        for batch in ((cu, start, *pool.batch()[2:]), (cu, start, far, *caches, *scales)):
            esa.esa_append_paged(k[rows], v[rows], *batch, rope_base=BASE)
    at = int(pool.table[0, 0])
    for a, b, sa, sb in zip(pool.caches, caches, pool.scales, scales):
        assert torch.equal(a.view(torch.uint8)[at, :, :60], b.view(torch.uint8)[n_pages - 1 - at, :, :60]) and torch.equal(sa[at], sb[n_pages - 1 - at])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_to_blocks_of_any_scale(esa, dtype):
    """Every exponent byte that a page may hold before a sequence goes on in it; 255 is a block that holds nothing."""
    bytes_held, first, new, page, h_kv, d = [0, 1, 26, 27, 120, 239, 240, 253, 254, 255], 7, 5, 16, 2, 64
    pool = Pool([(first, new)] * len(bytes_held), h_kv, d, page, dtype, "e4m3", seed=43)
    values, _, scale, _ = [None if x is None else x.copy() for x in pool.values()]
    rows, raw = [], pool.caches[0].view(torch.uint8).cpu()
    for b, byte in enumerate(bytes_held):
        at = pool.table[b, 0]
        # rows some of which the block's own scale can hold
        rows.append(torch.from_numpy(pool.rng.standard_normal((new, h_kv, d)) * 2.0 ** (min(max(byte, 40), 250) - 127)))
        if byte != 255:
            x = orc.to_e4m3(pool.rng.standard_normal((h_kv, first, d)) * 100)
            values[at, :, :first] = x
            raw[at, :, :first] = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8)
        scale[at] = byte
    for cache, s in zip(pool.caches, pool.scales):
        cache.view(torch.uint8).copy_(raw)
        s.copy_(torch.from_numpy(scale))
    k = torch.cat(rows).to(TYPES[dtype]).cuda()
    esa.esa_append_paged(k, k, *pool.batch())
    for b, byte in enumerate(bytes_held):
        at, mine = pool.table[b, 0], f64(k[b * new:(b + 1) * new])
        earlier = values[at, :, :first].copy()
        if byte == 255:
            scale[at], values[at, :, :first] = 0, 0.0
        orc.append_blocks(values, scale, mine, first, pool.table[b], page)
        if byte == 255:
            values[at, :, :first] = earlier
    for got, want in zip(pool.values(), (values, values, scale, scale)):
        assert np.array_equal(got, want, equal_nan=want.ndim == 4)


@pytest.mark.parametrize("dtype,d,new", [("bf16", 64, 1), ("bf16", 128, 100), ("f32", 64, 1), ("f32", 256, 1)])
def test_attend_reads_every_scale(esa, dtype, d, new):
    """Values of a block are its numbers times 2^(byte - 127) from the first byte to the last: outputs grow by that power of two."""
    pool = Pool([(300, new)], 1, d, 64, dtype, "e4m3", seed=44).fill()
    # numbers from 256 to 448 and probabilities of about one: no value or product is subnormal under byte 0 but for what a probability's second
    # term adds, so fp32 outputs are the same but for the power of two, bf16 ones within a rounding of each
    q = pool.rows(new, 4, 0.01)
    raw = pool.caches[1].view(torch.uint8)
    raw.copy_((raw & 0x7F).clamp(0x78, 0x7E))
    got = []
    for byte in (127, 0, 1, 200):
        pool.scales[1].fill_(byte)
        got.append(esa.esa_attend_paged(q, *pool.batch()).double() * 2.0 ** (127 - byte))
    for x in got[1:]:
        assert torch.equal(x, got[0]) if dtype == "f32" else torch.all((x - got[0]).abs() <= 2.0 ** -7 * got[0])


@pytest.mark.parametrize("dtype,held,d", [("bf16", "e4m3", 128), ("bf16", "same", 64), ("bf16", "same", 256), ("f32", "same", 64), ("f32", "e4m3", 128), ("f32", "same", 256)])
@pytest.mark.parametrize("cap", [0.0, 30.0])
@pytest.mark.parametrize("lengths", [[(100, 2), (20, 1)], [(5000, 2), (20, 1)], [(100, 90), (0, 40)], [(3000, 300), (20, 1)]], ids=["short", "cut", "chunk", "cut chunk"])
def test_a_query_that_is_nan_shows(esa, dtype, held, d, cap, lengths):
    """Its rows are NaN however their keys are shared out, and every other row is what it would be."""
    print("[case] NaN query", dtype, held, d, cap, lengths, flush=True)
    pool = Pool(lengths, 2, d, 64, dtype, held, seed=45).fill()
    q = pool.rows(pool.n_tok, 8)
    want, want_lse = esa.esa_attend_paged(q, *pool.batch(), cap=cap, return_lse=True)
    ill = torch.zeros(pool.n_tok, 8, dtype=torch.bool, device="cuda")
    for tok, head in ((0, 3), (lengths[0][1] - 1, 0), (pool.n_tok - 1, 7)):
        ill[tok, head] = True
        q[tok, head, 5 + head] = float("nan")
    out, lse = esa.esa_attend_paged(q, *pool.batch(), cap=cap, return_lse=True)
    assert torch.all(torch.isnan(out[ill])) and torch.all(torch.isnan(lse[ill]))
    assert torch.equal(out[~ill], want[~ill]) and torch.equal(lse[~ill], want_lse[~ill])


# ---------------------------------------------------------------- more workgroups than a dimension of a launch takes (2^24 of 256 threads)
@pytest.fixture
def memory():
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("held,n_tok,h_kv", [("same", (1 << 26) + 70, 1), ("e4m3", (1 << 24) + 70, 8)])
def test_append_of_millions_of_tokens(esa, memory, held, n_tok, h_kv):
    """A prompt all but whose last rows have no page; those are the rows that they are by themselves."""
    print("[case] long append", held, n_tok, h_kv, flush=True)
    d, page, last = 32, 16, 50
    pool = Pool([(0, last)], h_kv, d, page, "bf16", held, seed=46, spare=20)
    k = torch.empty((n_tok, h_kv, d), dtype=torch.bfloat16, device="cuda")
    k[-last:] = pool.rows(last, h_kv)
    first = n_tok - last
    table = torch.full((1, -(-n_tok // page)), -1, dtype=torch.int32, device="cuda")
    n = table.shape[1] - first // page
    got = []
    for at, cu, start, rows in ((0, [0, n_tok], [0], k), (8, [0, last], [first], k[-last:])):
        table[0, -n:] = torch.arange(at, at + n, dtype=torch.int32)
        # the page in which the last rows begin has earlier ones too where they belong to the call
        table[0, first // page] = -1
        cu, start = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (cu, start))
        esa.esa_append_paged(rows, rows, cu, start, table, *pool.batch()[3:], rope_base=BASE)
        got.append([c.view(torch.uint8)[at + 1:at + n].clone() if held == "e4m3" else c[at + 1:at + n].clone() for c in pool.caches]
                   + [s[at + 1:at + n].clone() for s in pool.scales if s is not None])
    for a, b in zip(*got):
        if a.dtype == torch.bfloat16:
            a, b = a.view(torch.int16), b.view(torch.int16)
        assert torch.equal(a, b)
    assert held == "e4m3" or not torch.all(torch.isnan(got[0][0]))


@pytest.mark.parametrize("dtype,h,h_kv,d,lengths", [("f32", 65535, 1, 256, [(0, 257)]), ("bf16", 65535, 65535, 32, [(b % 16, 1) for b in range(257)])],
                         ids=["plain", "few rows"])
def test_attend_with_millions_of_workgroups(esa, memory, dtype, h, h_kv, d, lengths):
    print("[case] workgroups", dtype, h, h_kv, d, flush=True)
    n_tok, n_seq, page = sum(n for _, n in lengths), len(lengths), 16
    width = -(-max(t0 + n for t0, n in lengths) // page)
    caches = [torch.randn((width, h_kv, page, d), device="cuda").to(TYPES[dtype]) for _ in "kv"]
    table = torch.arange(width, dtype=torch.int32, device="cuda").expand(n_seq, -1).contiguous()      # pages that all sequences read
    cu = torch.tensor([0] + [n for _, n in lengths], dtype=torch.int32).cumsum(0).to(torch.int32).cuda()
    start = torch.tensor([t0 for t0, _ in lengths], dtype=torch.int32, device="cuda")
    q = torch.zeros((n_tok, h, d), dtype=TYPES[dtype], device="cuda")
    q[-1] = torch.randn((h, d), device="cuda").to(q.dtype)
    out, lse = esa.esa_attend_paged(q, cu, start, table, *caches, return_lse=True)
    one = (torch.tensor([0, 1], dtype=torch.int32, device="cuda"), (start + cu[1:] - cu[:-1] - 1)[-1:].contiguous(), table[-1:], *caches)
    want, want_lse = esa.esa_attend_paged(q[-1:].contiguous(), *one, return_lse=True)
    assert torch.equal(out[-1:], want) and torch.equal(lse[-1:], want_lse)
    assert torch.all(lse[0] == torch.log(torch.tensor(1.0 + lengths[0][0])).item())       # one key, a query of zeros


def test_one_token_of_millions_beside_a_chunk(esa, memory):
    """More blocks times tiles than fp32 counts exactly: the kernels cut the long sequence alike.  Its table repeats eight pages, so its softmax is theirs."""
    page, d, h, chunk, repeats = 128, 32, 32, 2050, 8192
    caches = [torch.randn((8, 1, page, d), device="cuda") for _ in "kv"]
    width = 8 * repeats
    table = torch.arange(width, dtype=torch.int32, device="cuda").remainder(8).expand(2, -1).contiguous()
    total = [width * page, 1 << 18]
    cu = torch.tensor([0, 1, 1 + chunk], dtype=torch.int32, device="cuda")
    start = torch.tensor([total[0] - 1, total[1] - chunk], dtype=torch.int32, device="cuda")
    q = torch.randn((1 + chunk, h, d), device="cuda")
    out, lse = esa.esa_attend_paged(q, cu, start, table, *caches, return_lse=True)
    k, v = (f64(c)[:, 0].reshape(-1, d) for c in caches)
    for row, n in ((0, repeats), (-1, total[1] // (8 * page))):
        want, want_lse, spread, _ = orc.attend(f64(q[row])[None], 8 * page, k[:, None], v[:, None], range(8 * page), d ** -0.5)
        # sums of a wave run over up to 2^16 tiles, one rounding each, of the exponentials and of their products; 2^-20 for the rest
        tol = 2 * (2.0 ** -8 + 2.0 ** -20)
        assert np.all(np.abs(f64(out[row]) - want[0]) <= tol * spread[0])
        assert np.all(np.abs(f64(lse[row]) - want_lse[0] - np.log(n)) <= tol)


# ---------------------------------------------------------------- what the arrays on the device may hold
BAD = {
    "descending": ([0, 40, 10, 60, 20, 70], [0, 5, 0, 700, 3]), "behind the rows": ([0, 500, 3, 10 ** 9, 2 ** 31 - 1, 90], [0, 0, 100, 0, 0]),
    "negative": ([-5, 7, -2 ** 31, 30, 30, 69], [-1, -2 ** 31, 4, 50, 0]), "positions at the end": ([0, 1, 2, 40, 50, 70], [2 ** 31 - 1, 2 ** 31 - 2, 2 ** 31 - 30, 899, 10 ** 9]),
    "one sequence has all": ([0, 70, 70, 70, 70, 70], [900, -7, 5, 2 ** 30, 0]),
}


@pytest.mark.parametrize("dtype,held,d", [("bf16", "e4m3", 128), ("bf16", "same", 64), ("bf16", "e4m3", 32), ("f32", "same", 64), ("f32", "e4m3", 256)])
@pytest.mark.parametrize("name", sorted(BAD))
@pytest.mark.parametrize("times", [1, 20], ids=["5 sequences", "100"])
def test_nothing_in_the_arrays_leads_out_of_the_buffers(esa, dtype, held, d, name, times):
    """Offsets, positions, pages and selected entries of any content: what lies around the pool, the outputs and the workspace stays as it is."""
    print("[case] bad arrays", dtype, held, d, name, times, flush=True)
    rng = np.random.default_rng(47)
    h, h_kv, page, n_pages, width, n_tok, n_sel, edge = 8, 2, 16, 12, 64, 70, 33, 64
    t, at = TYPES[dtype], torch.uint8 if held == "e4m3" else TYPES[dtype]
    ints = lambda *shape: torch.from_numpy(rng.integers(-2 ** 31, 2 ** 31, shape, dtype=np.int64).astype(np.int32))
    cu = torch.tensor((BAD[name][0][:-1] * times + BAD[name][0][-1:]), dtype=torch.int64).to(torch.int32).cuda()
    start = torch.tensor(BAD[name][1] * times, dtype=torch.int64).to(torch.int32).cuda()
    n_seq = len(start)
    pages = torch.where(torch.from_numpy(rng.random((n_seq, width)) < 0.5), ints(n_seq, width), torch.from_numpy(rng.integers(0, n_pages, (n_seq, width)).astype(np.int32))).cuda()
    idx = torch.where(torch.from_numpy(rng.random((n_seq, n_sel)) < 0.5), ints(n_seq, n_sel), torch.from_numpy(rng.integers(0, 1000, (n_seq, n_sel)).astype(np.int32))).cuda()
    pool = [torch.full((n_pages + 2, h_kv, page, d), 1, dtype=at, device="cuda") for _ in "kv"]
    scales = [torch.full((n_pages + 2, h_kv), 127, dtype=torch.uint8, device="cuda") for _ in "kv"]
    inner = [p[1:-1].view(torch.float8_e4m3fn) if held == "e4m3" else p[1:-1] for p in pool] + [s[1:-1] if held == "e4m3" else None for s in scales]
    q, k, v = (torch.from_numpy(rng.standard_normal((n_tok, n, d))).to(t).cuda() for n in (h, h_kv, h_kv))
    out, turned = (torch.full((n_tok + 2, h, d), 3.0, dtype=t, device="cuda") for _ in range(2))
    esa.esa_append_paged(k, v, cu, start, pages, *inner, q=q, rope_base=BASE, out_q=turned[1:-1])
    for l_i, l_l, chosen in ((None, 0, None), (20, 100, idx)):
        esa.esa_attend_paged(q, cu, start, pages, *inner, l_i=l_i, l_l=l_l, idx=chosen, out=out[1:-1], return_lse=True)
    # the C entry, whose workspace is the caller's
    need = esa.lib.esa_attend_paged_workspace_bytes(n_tok, n_seq, h, h_kv, d, 0 if dtype == "f32" else 1)
    ws = torch.full((need + edge * 1024,), 0x5A, dtype=torch.uint8, device="cuda")
    lse = torch.full((n_tok + 2, h), 3.0, device="cuda")
    batch = esa.PagedBatch(cu=cu.data_ptr(), start=start.data_ptr(), pages=pages.data_ptr(), pages_ld=width, n_tok=n_tok, n_seq=n_seq, max_pages=width)
    e = {"e4m3": 2, "same": 0 if dtype == "f32" else 1}[held]
    cache = esa.PagedCache(k=inner[0].data_ptr(), v=inner[1].data_ptr(), k_scale=inner[2].data_ptr() if e == 2 else None, v_scale=inner[3].data_ptr() if e == 2 else None,
                           page_stride=h_kv * page * d, head_stride=page * d, tok_stride=d, n_pages=n_pages, page_size=page, h_kv=h_kv, d=d, dtype=e)
    assert esa.lib.esa_attend_paged(q.data_ptr(), h * d, h, ctypes.byref(batch), ctypes.byref(cache), 1 << 40, 0, None, 0, 0, 0.1, 0.0, out[1:].data_ptr(), h * d,
                                    lse[1:].data_ptr(), 0 if dtype == "f32" else 1, ws.data_ptr(), need, torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    for x, same in [(p, 1) for p in pool] + [(s, 127) for s in scales] + [(out, 3.0), (turned, 3.0), (lse, 3.0)]:
        assert torch.all(x[0] == same) and torch.all(x[-1] == same)
    assert torch.all(ws[need:] == 0x5A)


@pytest.mark.parametrize("dtype,held,d", [("bf16", "e4m3", 128), ("bf16", "same", 64), ("f32", "e4m3", 256)])
@pytest.mark.parametrize("new", [1, 80])
def test_pages_that_several_sequences_read(esa, dtype, held, d, new):
    """A common beginning lies in the pool once."""
    print("[case] shared pages", dtype, held, d, new, flush=True)
    page, shared = 32, 6
    pool = Pool([(300, new), (200, new), (shared * page, new)], 2, d, page, dtype, held, seed=48)
    pool.table[1:, :shared] = pool.table[0, :shared]
    pool.pages = torch.tensor(pool.table, device="cuda")
    pool.fill()
    k, v, q = pool.rows(pool.n_tok, 2), pool.rows(pool.n_tok, 2), pool.rows(pool.n_tok, 8)
    turned = esa.esa_append_paged(k, v, *pool.batch(), q=q, rope_base=BASE)
    out, lse = esa.esa_attend_paged(turned, *pool.batch(), return_lse=True)
    check_attention(pool, turned, out, lse, p_half_step=P_STEP[dtype])


WIDE = {"one short": [(301, 1)], "chunks": [(40, 90), (200, 33)], "mixed": [(0, 1), (63, 40), (513, 7), (7, 0), (31, 1)], "drafts": [(455, 5)] * 4}


@pytest.mark.parametrize("dtype,held,d", [("bf16", "e4m3", 128), ("bf16", "same", 64), ("f32", "same", 64), ("f32", "e4m3", 128), ("bf16", "same", 256)])
@pytest.mark.parametrize("name", sorted(WIDE))
def test_short_sequences_under_a_wide_table(esa, dtype, held, d, name):
    """A table with room for 131072 positions: sequences are cut and joined otherwise than under one of their own length."""
    print("[case] wide table", dtype, held, d, name, flush=True)
    pool = Pool(WIDE[name], 2, d, 64, dtype, held, seed=49).fill()
    wide = torch.full((len(WIDE[name]), 2048), -1, dtype=torch.int32, device="cuda")
    wide[:, :pool.pages.shape[1]] = pool.pages
    q = pool.rows(pool.n_tok, 8)
    for l_i, l_l in ((None, 0), (20, 100)):
        out, lse = esa.esa_attend_paged(q, *pool.batch()[:2], wide, *pool.batch()[3:], l_i=l_i, l_l=l_l, return_lse=True)
        check_attention(pool, q, out, lse, l_i=l_i, l_l=l_l, p_half_step=P_STEP[dtype])
