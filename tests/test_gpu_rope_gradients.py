"""Rotation in a graph of gradients: what autograd gives is the transposed call, rows without a position have no part in it."""
import numpy as np
import pytest
import torch

from oracle import serve_oracle as orc

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


@pytest.fixture(scope="module")
def esa():
    import paper_2502_14477_amd as lib
    return lib


def f64(t):
    return t.detach().double().cpu().numpy()


def rows(seed, n, heads, d, dtype):
    return torch.randn((n, heads, d), generator=torch.Generator("cuda").manual_seed(seed), device="cuda").to(TYPES[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("halves", [True, False])
@pytest.mark.parametrize("transposed", [True, False])
def test_gradients_are_the_transposed_call(esa, transposed, halves, dtype):
    n, h, h_kv, d, rot = 23, 6, 2, 40, 24
    pos = np.random.default_rng(1).integers(0, 5000, n)
    pos[[3, 22]] = -1
    there = torch.from_numpy(pos >= 0).cuda()
    at, freq = torch.tensor(pos, dtype=torch.int32, device="cuda"), esa.esa_rope_frequencies(1e4, rot)
    kw = dict(pairs=esa.ESA_PAIRS_HALVES if halves else esa.ESA_PAIRS_NEIGHBOURS, gain=1.25, transposed=transposed)
    q, k, gq, gk = rows(1, n, h, d, dtype), rows(2, n, h_kv, d, dtype), rows(3, n, h, d, dtype), rows(4, n, h_kv, d, dtype)
    for ask_q, ask_k in ((True, True), (True, False), (False, True)):
        a, b = q.clone().requires_grad_(ask_q), k.clone().requires_grad_(ask_k)
        y = esa.esa_rope_at(a, at, freq, k=b, **kw)
        with torch.no_grad():
            plain = esa.esa_rope_at(q, at, freq, k=k, **kw)
        assert torch.equal(y[0][there], plain[0][there]) and torch.equal(y[1][there], plain[1][there])
        assert (y[0].requires_grad, y[1].requires_grad) == (ask_q, ask_k)
        torch.autograd.backward([t for t in y if t.requires_grad], [g for t, g in zip(y, (gq, gk)) if t.requires_grad])
        for x, g, asked in ((a, gq, ask_q), (b, gk, ask_k)):
            assert (x.grad is not None) == asked
            if not asked:
                continue
            want = orc.rope(f64(g), pos, freq.cpu().numpy(), halves, 1.25, not transposed)
            got = f64(x.grad)
            # one rounding to storage, and the angles' 2^-53 of 5000 and some of the pair's length
            tol = HALF_STEP[dtype] * np.abs(want) * (1 + 1e-9) + 2.0 ** -36
            assert np.all((np.abs(got - want) <= tol)[pos >= 0]) and not np.any(got[pos < 0])


def test_gradients_of_queries_alone_of_views_and_of_shared_heads(esa):
    """Keys that heads share by broadcasting get their heads' sum; a loss whose gradient is one number for all elements; part of a projection."""
    n, d = 9, 16
    at, freq = torch.arange(n, dtype=torch.int32, device="cuda"), esa.esa_rope_frequencies(1e4, d)
    shared = rows(5, n, 1, d, "f32").requires_grad_()
    g = rows(6, n, 4, d, "f32")
    esa.esa_rope_at(shared.expand(n, 4, d), at, freq).backward(g)
    each = f64(esa.esa_rope_at(g, at, freq, transposed=True))
    assert np.all(np.abs(f64(shared.grad) - each.sum(1, keepdims=True)) <= 3 * 2.0 ** -24 * np.abs(each).sum(1, keepdims=True))
    x = rows(7, n, 7, d, "f32").requires_grad_()
    y = esa.esa_rope_at(x[:, :4], at, freq, k=x[:, 4:6])
    (y[0].sum() + y[1].sum()).backward()
    ones = esa.esa_rope_at(torch.ones((n, 6, d), device="cuda"), at, freq, transposed=True)
    assert torch.equal(x.grad[:, :6], ones) and not torch.any(x.grad[:, 6:])


def test_gradients_by_differences_and_of_gradients(esa):
    n, d = 5, 8
    at, freq = torch.tensor([0, 7, -1, 900, 3], dtype=torch.int32, device="cuda"), esa.esa_rope_frequencies(1e4, 6)
    x = rows(8, n, 2, d, "f32").requires_grad_()
    w = rows(9, n, 2, d, "f32").masked_fill((at < 0)[:, None, None], 0.0)

    def loss(v):      # quartic, so that second derivatives are no constants
        y = esa.esa_rope_at(v, at, freq, gain=0.5)
        return (torch.where(w != 0, y, 0.0) ** 4 * w).sum()

    first, = torch.autograd.grad(loss(x), x, create_graph=True)
    e = rows(10, n, 2, d, "f32")
    second, = torch.autograd.grad((first * e).sum(), x)
    y = orc.rope(f64(x), at.cpu().numpy(), freq.cpu().numpy(), True, 0.5)
    turned = orc.rope(f64(e), at.cpu().numpy(), freq.cpu().numpy(), True, 0.5)
    y, turned = np.nan_to_num(y), np.nan_to_num(turned)
    want1 = np.nan_to_num(orc.rope(4 * y ** 3 * f64(w), at.cpu().numpy(), freq.cpu().numpy(), True, 0.5, True))
    want2 = np.nan_to_num(orc.rope(12 * y ** 2 * turned * f64(w), at.cpu().numpy(), freq.cpu().numpy(), True, 0.5, True))
    # fp32 powers, products and roundings: some ten half steps of the largest term
    for got, want in ((first, want1), (second, want2)):
        assert np.all(np.abs(f64(got) - want) <= 16 * 2.0 ** -24 * np.abs(want).max())
    # along a direction: the fourth-order difference of a quartic is exact but for its roundings, here in 64 bits by the oracle
    def in_64(v):
        t = np.nan_to_num(orc.rope(v, at.cpu().numpy(), freq.cpu().numpy(), True, 0.5))
        return np.sum(t ** 4 * f64(w))
    v, s, h = f64(x), f64(e), 0.125
    by_difference = (8 * (in_64(v + h * s) - in_64(v - h * s)) - (in_64(v + 2 * h * s) - in_64(v - 2 * h * s))) / (12 * h)
    terms = np.sum(np.abs(want1 * s))
    assert abs(np.sum(f64(first) * s) - by_difference) <= 32 * 2.0 ** -24 * terms + 16 * 2.0 ** -24 * np.abs(want1).max() * np.sum(np.abs(s))


def test_a_graph_of_gradients_is_asked_for(esa):
    """Without gradients, or where nobody needs one, the call is what it was; outputs that are given have none to offer."""
    x, at, freq = rows(11, 3, 2, 8, "f32").requires_grad_(), torch.arange(3, dtype=torch.int32, device="cuda"), esa.esa_rope_frequencies(1e4, 8)
    with torch.no_grad():
        out = torch.empty_like(x)
        assert esa.esa_rope_at(x, at, freq, out_q=out) is out and not out.requires_grad
    assert not esa.esa_rope_at(x.detach(), at, freq).requires_grad
    with pytest.raises(esa.EsaError):
        esa.esa_rope_at(x, at, freq, out_q=torch.empty_like(x))
    with pytest.raises(esa.EsaError):
        esa.esa_rope_at(x.detach(), at, freq.clone().requires_grad_())
    y = esa.esa_rope_at(x, at, freq)
    y.backward(torch.ones_like(y))
    assert torch.equal(x.grad, esa.esa_rope_at(torch.ones_like(y), at, freq, transposed=True))
