"""What rotation refuses where gradients are wanted, without a GPU."""
import pytest
import torch

import paper_2502_14477_amd as esa


def test_refusals_where_gradients_are_wanted():
    q, pos, freq = torch.zeros(5, 4, 64), torch.zeros(5, dtype=torch.int32), esa.esa_rope_frequencies(1e4, 64, device="cpu")
    asked = q.clone().requires_grad_()
    for args, kw in (((asked, pos, freq), dict(out_q=q)), ((q, pos, freq), dict(k=asked, out_k=q)), ((asked * 1, pos, freq), dict(out_q=q)),
                     ((q, pos, freq.clone().requires_grad_()), {})):
        with pytest.raises(esa.EsaError):
            esa.esa_rope_at(*args, **kw)
        with torch.no_grad(), pytest.raises(AssertionError):      # as before: no tensor on a GPU
            esa.esa_rope_at(*args, **kw)
    with pytest.raises(AssertionError):
        esa.esa_rope_at(asked, pos, freq)
