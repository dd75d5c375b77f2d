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
