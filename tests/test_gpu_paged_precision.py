"""How near the paged attention's bf16 outputs are: probabilities keep sixteen bits wherever a kernel takes them as two bf16 terms."""
import pytest

from paged_support import Pool, check_attention

pytestmark = pytest.mark.gpu
# A first term is off by half a step, 2^-8 of the probability at most, and a second one by as much of what the first leaves.
TWO_TERMS = 2.0 ** -16


@pytest.fixture(scope="module")
def esa():
    import paper_2502_14477_amd as lib
    return lib


# Outputs smaller than the terms of their sums, so that a probability's rounding shows beside the output's own: hundreds of keys, values of both signs.
@pytest.mark.parametrize("held", ["e4m3", "same"])
@pytest.mark.parametrize("d", [32, 64, 128, 256])
@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("lengths", [[(700, 1)], [(3000, 2), (90, 1), (0, 3)]], ids=["one", "ragged"])
def test_few_rows_keep_sixteen_bits_of_a_probability(esa, held, d, cap, lengths):
    print("[case] precision, few rows", held, d, cap, lengths, flush=True)
    pool = Pool(lengths, 2, d, 32, "bf16", held, seed=31).fill((1.0, 1.0))
    q = pool.rows(pool.n_tok, 8)
    out, lse = esa.esa_attend_paged(q, *pool.batch(), cap=cap, return_lse=True)
    # (a capped bf16 score is off by up to 2^-21 of the cap, as the header says, eight times what the bound has for a cap's rounding)
    check_attention(pool, q, out, lse, cap=cap, p_half_step=TWO_TERMS + cap * 2.0 ** -21)


@pytest.mark.parametrize("held", ["e4m3", "same"])
@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("lengths", [[(700, 90)], [(3000, 65), (90, 129), (0, 33)], [(1000, 300), (2000, 1)]], ids=["one", "ragged", "mixed"])
def test_chunks_of_head_size_64_keep_sixteen_bits_of_a_probability(esa, held, cap, lengths):
    print("[case] precision, chunk", held, cap, lengths, flush=True)
    pool = Pool(lengths, 2, 64, 64, "bf16", held, seed=32).fill((1.0, 1.0))
    q = pool.rows(pool.n_tok, 8)
    out, lse = esa.esa_attend_paged(q, *pool.batch(), cap=cap, return_lse=True)
    check_attention(pool, q, out, lse, cap=cap, p_half_step=TWO_TERMS + cap * 2.0 ** -21)
