"""Calls around the paged cache that would write over what other workgroups read: refused on the host, before anything is enqueued."""
import ctypes

import pytest

import paper_2502_14477_amd as esa

SEQS, WIDTH, LD, PAGES, ROWS = 3, 8, 12, 20, 7


def places(**kw):
    """Arrays of a plan that is not in place, one behind the other (never dereferenced), and their sizes in bytes."""
    sizes = dict(start_in=4 * SEQS, held_in=4 * SEQS, ring_at_in=8, start=4 * SEQS, held=4 * SEQS, ring_at=8, pages=4 * (LD * (SEQS - 1) + WIDTH), ring=4 * PAGES, grow=4 * SEQS,
                 fresh=4 * SEQS, cu=4 * SEQS + 4, pos=4 * ROWS, slot=8 * ROWS, lack=4, ws=256)
    at, got = 1 << 20, {}
    for name, n in sizes.items():
        got[name] = at
        at += n + (-n) % 256
    got.update(kw)
    return got, sizes


def plan(p):
    """The call's code.  A call that passes would be enqueued: none here does."""
    fields = {f[0] for f in esa.PageState._fields_}
    s = esa.PageState(**{k: v for k, v in p.items() if k in fields}, pages_ld=LD, n_seq=SEQS, max_pages=WIDTH, n_pages=PAGES, page_size=64)
    return esa.lib.esa_plan_paged(ctypes.byref(s), p["grow"], p["fresh"], ROWS, p["cu"], p["pos"], p["slot"], p["lack"], p["ws"], 1 << 20, None)


READ = ["start_in", "held_in", "ring_at_in", "grow", "fresh", "pages"]
WRITTEN = ["start", "held", "ring_at", "ring", "cu", "lack", "pos", "slot"]
OWN = {("start", "start_in"), ("held", "held_in"), ("ring_at", "ring_at_in")}


@pytest.mark.parametrize("a,b", [(a, b) for a in WRITTEN for b in READ + WRITTEN if a != b])
def test_plan_refuses_arrays_over_one_another(a, b):
    p, sizes = places()
    if (a, b) not in OWN:
        p[a] = p[b]
        assert plan(p) == -1 and b"overlaps" in esa.lib.esa_last_error()
    by = 8 if a == "slot" else 4
    p, _ = places()
    p[a] = p[b] + (sizes[b] - 4) // by * by                       # its last element
    if (a, b) not in OWN or p[a] != p[b]:
        assert plan(p) == -1 and b"overlaps" in esa.lib.esa_last_error()
    p, _ = places()
    p[a] = p[b] - (sizes[a] - by)                                 # its first one
    if b != "slot" or p[a] % by == 0:
        assert plan(p) == -1


def test_plan_refuses_its_own_workspace():
    p, _ = places()
    in_place = dict(start=p["start_in"], held=p["held_in"], ring_at=p["ring_at_in"])
    for name in ("start_in", "ring", "pages", "cu"):
        q, _ = places(**in_place)
        q["ws"] = q[name] // 256 * 256
        assert plan(q) == -1 and b"overlaps" in esa.lib.esa_last_error()


def test_plan_refuses_the_table_it_reads():
    """An array inside the table's rows or over the end of what lies between them."""
    for name in ("grow", "fresh", "cu", "pos"):
        for element in (0, WIDTH - 1, LD, 2 * LD + WIDTH - 1, WIDTH + 2):
            p, _ = places()
            p[name] = p["pages"] + 4 * element
            assert plan(p) == -1 and b"overlaps" in esa.lib.esa_last_error(), (name, element)


# ---------------------------------------------------------------- drafts
VERIFY = dict(target=4 * (ROWS - 1) * 20010 + 80000, draft=4 * (ROWS - 1) * 20010 + 80000, tokens=4 * ROWS, u=4 * ROWS, cu=4 * SEQS + 4, out=4 * ROWS, count=4 * SEQS, ws=4096)


def verify(**kw):
    at, p = 1 << 20, {}
    for name, n in VERIFY.items():
        p[name] = at
        at += n + (-n) % 256
    for name, (other, by) in kw.items():
        p[name] = p[other] + by
    return esa.lib.esa_verify_drafts(p["target"], 20010, p["draft"], 20010, p["tokens"], p["u"], p["cu"], ROWS, SEQS, 20000, p["out"], p["count"], 0, p["ws"], 4096, None)


@pytest.mark.parametrize("a", ["out", "count"])
@pytest.mark.parametrize("b", list(VERIFY))
def test_verify_refuses_arrays_over_one_another(a, b):
    if a != b:
        for by in (0, 4 - VERIFY[a], (0 if b == "ws" else VERIFY[b]) - 4):
            assert verify(**{a: (b, by)}) == -1 and b"esa_verify_drafts" in esa.lib.esa_last_error()


def test_verify_refuses_what_lies_over_rows():
    for rows in ("target", "draft"):
        for element in (0, 19999, 20008, 6 * 20010 + 19999):      # the first, a row's last, in front of a row and into it, the last
            assert verify(out=(rows, 4 * element)) == -1 and b"overlaps" in esa.lib.esa_last_error()
    for name in ("target", "draft", "cu", "tokens", "u"):
        assert verify(ws=(name, 0)) == -1
