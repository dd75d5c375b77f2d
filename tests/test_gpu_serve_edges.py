"""The calls around the paged cache at the ends of what they take."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def esa():
    import paper_2502_14477_amd as lib
    return lib


@pytest.mark.parametrize("vocab", [3000, 5000, 16384, 16400])
def test_verify_millions_of_sequences(esa, vocab):
    """Nearly all of them without a row: workgroups of 512 and 1024 threads, more than a row of the grid has; the last sequences are in its third row
    (long rows by two launches, whose first one goes through the sequences in turn)."""
    n_seq = (1 << 22) + 5 if vocab <= 16384 else 70001
    with_rows = [0, 1, n_seq // 2 - 1, n_seq // 2, n_seq - 2, n_seq - 1]
    rows = torch.zeros(n_seq, dtype=torch.int32, device="cuda")
    rows[with_rows] = 1
    cu = torch.cat((torch.zeros(1, dtype=torch.int32, device="cuda"), rows.cumsum(0, dtype=torch.int32)))
    n = len(with_rows)
    sure = torch.arange(n, device="cuda") * (vocab // n) + 1
    p = torch.zeros((n, vocab), device="cuda").scatter_(1, sure[:, None], 1.0)
    out, count = esa.esa_verify_drafts(p, torch.zeros(n, dtype=torch.int32, device="cuda"), cu, torch.full((n,), 0.5, device="cuda"))
    assert torch.equal(out, sure.int())
    assert torch.equal(count, rows)


def test_plan_in_arrays_that_touch(esa):
    """One buffer holds everything: arrays one right behind the other, one of them between the table's rows."""
    n_seq, width, ld, n_pages, n_tok = 3, 5, 9, 20, 60
    buffer = torch.full((200,), 55, dtype=torch.int32, device="cuda")
    at = 0

    def take(values):
        nonlocal at
        x = buffer[at:at + len(values)]
        x.copy_(torch.tensor(values, dtype=torch.int32))
        at += len(values)
        return x

    pages = buffer[at:at + n_seq * ld].view(n_seq, ld)[:, :width]
    grow = buffer[at + width:at + width + n_seq]
    grow.copy_(torch.tensor([0, 2, 1], dtype=torch.int32))
    at += (n_seq - 1) * ld + width                                # right behind the table's last entry
    ring, start, held, ring_at, new = take(list(range(n_pages))), take([0, 0, 0]), take([0, 0, 0]), take([4, n_pages]), take([20, 17, 16])
    cu, pos, lack = take([7] * (n_seq + 1)), take([7] * n_tok), take([7])
    end = at
    slot = torch.empty(n_tok, dtype=torch.int64, device="cuda")
    esa.esa_plan_paged(new, start, held, pages, ring, ring_at, 16, n_tok, grow=grow, out=esa.PagePlan(cu, start, held, ring_at, pos, slot, lack))
    assert start.tolist() == [0, 2, 1] and held.tolist() == [2, 2, 2] and ring_at.tolist() == [10, 14] and lack.item() == 0
    assert cu.tolist() == [0, 20, 37, 53] and pages[:, :2].tolist() == [[4, 5], [6, 7], [8, 9]] and torch.all(pages[:, 2:] == 55)
    assert grow.tolist() == [0, 2, 1] and new.tolist() == [20, 17, 16] and torch.all(buffer[end:] == 55)
    assert pos[:53].tolist() == list(range(20)) + list(range(2, 19)) + list(range(1, 17)) and torch.all(pos[53:] == -1)


def test_new_tensors_are_made_where_torch_sees_them(esa):
    """A dispatch mode sees the outputs being made, and deterministic mode fills them: rows that a call leaves alone hold no number then."""
    from torch.utils._python_dispatch import TorchDispatchMode

    class Seen(TorchDispatchMode):
        def __init__(self):
            super().__init__()
            self.shapes = []

        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            if func is torch.ops.aten.empty.memory_format:
                self.shapes.append(tuple(args[0]))
            return func(*args, **(kwargs or {}))

    q, k = torch.ones((3, 2, 8), device="cuda"), torch.ones((3, 1, 8), device="cuda")
    pos, freq = torch.tensor([4, -1, 0], dtype=torch.int32, device="cuda"), esa.esa_rope_frequencies(1e4, 8)
    p, cu = torch.full((4, 10), 0.1, device="cuda"), torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    tokens, u = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.full((4,), 0.55, device="cuda")
    plain = esa.esa_rope_at(q, pos, freq, k=k), esa.esa_verify_drafts(p, tokens, cu, u)
    with Seen() as seen:
        watched = esa.esa_rope_at(q, pos, freq, k=k), esa.esa_verify_drafts(p, tokens, cu, u)
    assert seen.shapes == [(3, 2, 8), (3, 1, 8), (4,), (2,)]
    was = torch.are_deterministic_algorithms_enabled()
    torch.use_deterministic_algorithms(True)
    try:
        filled = esa.esa_rope_at(q, pos, freq, k=k), esa.esa_verify_drafts(p, tokens, cu, u)
    finally:
        torch.use_deterministic_algorithms(was)
    for got in (watched, filled):
        for x, y in zip(plain[0], got[0]):
            assert torch.equal(x[[0, 2]], y[[0, 2]]) and x.device == y.device and x.stride() == y.stride()
        assert got[1][0][:2].tolist() == plain[1][0][:2].tolist() == [5, 5] and got[1][1].tolist() == [1, 1]
    assert all(torch.all(torch.isnan(x[1])) for x in filled[0])
    assert torch.all(filled[1][0][2:] == torch.iinfo(torch.int32).max)
