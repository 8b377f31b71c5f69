"""The operators' arithmetic below the step of their outputs, and values that are not finite, against float64
(tests/ops_oracle.py)."""
import pytest
import torch

import paper_2512_21835_amd as P
from tests import ops_oracle as O
from tests.test_gpu_ops import _adapter_case, _check_adapter, _run_adapter, _run_window, _window_case

pytestmark = pytest.mark.gpu


# ([1] * 3 and two KV heads: the keys cut over wavefronts; two prompts and many heads: whole tiles of rows)
@pytest.mark.parametrize("rows,held,hq,hkv", [([1, 1, 1], [5, 300, 900], 8, 2), ([37, 70], [90, 200], 8, 1),
                                              ([37, 1, 70], [90, 0, 200], 72, 9), ([37, 70], [90, 200], 50, 50)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (64, 3)])
def test_probabilities_of_bf16_rows(rows, held, hq, hkv, d, window, sinks):
    """Two bf16 terms, each within half a step of what it stands for, hold a probability to (2^-8)^2 of its value: the
    output is off by no more than 2^-16 of its terms' sizes beyond what fp32 rows are, before its own rounding."""
    b, q, out = c = _window_case(rows, held, hq, hkv, d, "bf16", "bf16")
    got = _run_window(c, window, sinks)
    want, off32, off16 = O.window(b, q, out, b.pool, hq, window, sinks)
    O.assert_within(got, want, O.rounded(want, off32 + off16 * 2.0 ** -8, torch.bfloat16))


# heads that make these whole tiles of rows, and those that do not
F32_CACHE = [([1, 1, 1], [5, 300, 900], 8, 2), ([37, 1, 70], [90, 0, 200], 72, 9), ([37, 70, 60, 50], [90, 200, 0, 7], 50, 50)]


@pytest.mark.parametrize("rows,held,hq,hkv", F32_CACHE)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (64, 3)])
def test_probabilities_and_values_of_bf16_rows_over_an_fp32_cache(rows, held, hq, hkv, d, window, sinks):
    """As above, and V as two terms too: 2^-16 twice."""
    b, q, out = c = _window_case(rows, held, hq, hkv, d, "bf16", "fp32")
    got = _run_window(c, window, sinks)
    want, off32, off16 = O.window(b, q, out, b.pool, hq, window, sinks)
    O.assert_within(got, want, O.rounded(want, off32 + 2 * off16 * 2.0 ** -8, torch.bfloat16))


@pytest.mark.parametrize("rows,held,hq,hkv", F32_CACHE)
@pytest.mark.parametrize("d", [64, 128])
def test_scores_of_bf16_rows_over_an_fp32_cache(rows, held, hq, hkv, d):
    """Scores of 200 from one product each, q of one element: half the keys' K are 4 and half the next number below, with V of
    the other sign, so that the output is what the scores are off.  A score's error does not grow with d here: three
    exact products and their sums, the scale in base 2 and the product by it: 8 of the 8 + d steps that the oracle takes."""
    b, q, out = c = _window_case(rows, held, hq, hkv, d, "bf16", "fp32")
    q.zero_()
    q[..., 5] = 50
    places = torch.arange(16) % 2 == 0
    b.pool[:, 0] = torch.where(places[:, None], 4.0, torch.nextafter(torch.tensor(4.0), torch.tensor(0.0)))
    b.pool[:, 1] = torch.where(places[:, None], 1.0, -1.0) * (1 + torch.rand(hkv, 1, d, generator=b.gen))
    got = _run_window(c, 0, 0, scale=1.0)
    want, off32, off16 = O.window(b, q, out, b.pool, hq, 0, 0, 1.0)
    keys = torch.tensor([n - r + t + 1 for n, r in zip(b.lengths, b.rows) for t in range(r)]).view(-1, 1, 1).double()
    term = off16 / O.U16
    size = (off32 / (term * O.U32) - 2 * keys - 32) / (2 * (d + 8))
    off = term * O.U32 * (2 * 16 * size + 2 * keys + 32) + 2 * off16 * 2.0 ** -8
    O.assert_within(got, want, O.rounded(want, off, torch.bfloat16))


@pytest.mark.parametrize("cache", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows,held,hq,hkv", F32_CACHE)
def test_rows_that_see_one_value_give_it(rows, held, hq, hkv, d, cache):
    """A window of one token: p V / p, with V of as many ones as its terms can have.  Off by 2^-24 of V for the products of
    small terms that are left out, two steps of the sum, the reciprocal and the product by it: 5 half steps of fp32."""
    b, q, out = c = _window_case(rows, held, hq, hkv, d, "fp32", cache)
    sign = torch.randint(0, 2, b.pool[:, 1].shape, generator=b.gen) * 2.0 - 1
    b.pool[:, 1] = sign * (1 + 2.0 ** -7 - 2.0 ** -23) * 2.0 ** torch.randint(-3, 4, sign.shape, generator=b.gen)
    got = _run_window(c, 1, 0)
    want = O.window(b, q, out, b.pool, hq, 1, 0)[0]
    O.assert_within(got, want, 5 * O.U32 * want.abs())


def _same(a, b):
    return torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(torch.nan_to_num(a), torch.nan_to_num(b))


@pytest.mark.parametrize("act", ["fp32", "bf16"])
@pytest.mark.parametrize("cache", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,held,hq,hkv", F32_CACHE)
def test_window_in_place(rows, held, hq, hkv, cache, act):
    """out is q: the same bits, where a K and a V that some rows see are not finite as well."""
    b, q, out = c = _window_case(rows, held, hq, hkv, 64, act, cache)
    for poisoned in (False, True):
        if poisoned:
            for what, i, back in ((0, 0, 1), (1, len(rows) - 1, 3)):
                p = b.lengths[i] - back
                b.pool[int(b.table[i, p // 16]), what, 0, p % 16, 9] = float("inf")
        want = _run_window(c, 40, 2)
        x = q.cuda()
        P.stage_window_attention(x, x, b.pool.cuda(), b.stage_batch(P), window=40, sinks=2)
        assert _same(x, want), poisoned


def test_window_in_place_with_another_stride_is_refused():
    b, q, out = _window_case([2], [3], 4, 2, 64, "fp32", "bf16")
    wide = torch.zeros(4, 4, 64, device="cuda")
    with pytest.raises(P.StageError) as e:
        P.stage_window_attention(wide[:2], wide[::2], b.pool.cuda(), b.stage_batch(P))
    assert e.value.code == P.STAGE_EINVAL


def _poisoned(rows, held, hq, hkv, d, act, cache, what, at, value):
    """A case, one with |V|, and one in which token 1 of every sequence has `value` in element 9 (or those of `at`) of K or V of
    KV head 0: a page that prompts behind held tokens see all of."""
    b, q, out = _window_case(rows, held, hq, hkv, d, act, cache)
    clean = b.pool.clone()
    for i in range(len(rows)):
        if b.lengths[i] > 1:
            for e, x in zip(at, value):
                b.pool[int(b.table[i, 0]), what, 0, 1, e] = x
    return b, q, out, clean


def _check_poisoned(b, q, out, clean, window, sinks):
    got = _run_window((b, q, out), window, sinks).double().cpu()
    want = O.window(b, q, out, b.pool, q.shape[1], window, sinks)[0]
    # what the probabilities are off relative to their sums' sizes, as without the odd value; those sizes with it
    _, off32, off16 = O.window(b, q, out, clean, q.shape[1], window, sinks)
    sizes = O.window(b, q, out, torch.cat([b.pool[:, :1], b.pool[:, 1:].abs()], 1), q.shape[1], window, sinks)[0]
    off = sizes * (off32 / (off16 / O.U16) + (2 * 2.0 ** -16 if q.dtype == torch.bfloat16 else 0))
    odd = ~torch.isfinite(want)
    assert torch.equal(got[odd], want[odd])
    O.assert_within(got[~odd], want[~odd], O.rounded(want, off, q.dtype)[~odd])
    return odd


@pytest.mark.parametrize("act", ["fp32", "bf16"])
@pytest.mark.parametrize("cache", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,held,hq,hkv", F32_CACHE)
@pytest.mark.parametrize("d", [64, 128])
def test_infinities_that_rows_see(rows, held, hq, hkv, d, cache, act):
    """Those of V reach the rows' elements as they are; a key of score -inf drops out."""
    inf = float("inf")
    for window, sinks in ((0, 0), (40, 2)):
        b, q, out, clean = _poisoned(rows, held, hq, hkv, d, act, cache, 1, (9, 10), (inf, -inf))
        assert bool(_check_poisoned(b, q, out, clean, window, sinks).any())
        b, q, out, clean = _poisoned(rows, held, hq, hkv, d, act, cache, 0, (9,), (-inf,))
        q[..., 9] = q[..., 9].abs() + 0.1
        assert not bool(_check_poisoned(b, q, out, clean, window, sinks).any())


@pytest.mark.parametrize("cache", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,held,hq,hkv", F32_CACHE)
@pytest.mark.parametrize("d", [64, 128])
def test_numbers_too_large_for_bf16(rows, held, hq, hkv, d, cache):
    """fp32 q and K between the largest bf16 and the largest fp32."""
    large = 3.4e38
    b, q, out = c = _window_case(rows, held, hq, hkv, d, "fp32", cache)
    q[..., 7] = large
    b.pool[:, 0, :, :, 7] = 2.0 ** -126 * torch.sign(b.pool[:, 0, :, :, 7])
    got = _run_window(c, 40, 2)
    want, off32, _ = O.window(b, q, out, b.pool, hq, 40, 2)
    O.assert_within(got, want, O.rounded(want, off32, torch.float32))
    if cache == "bf16":
        return
    q[..., 7] = 2.0 ** -126
    b.pool[:, 0, :, :, 7] = large * torch.sign(b.pool[:, 0, :, :, 7])
    got = _run_window(c, 40, 2)
    want, off32, _ = O.window(b, q, out, b.pool, hq, 40, 2)
    O.assert_within(got, want, O.rounded(want, off32, torch.float32))


@pytest.mark.parametrize("cache", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,held,hq,hkv", F32_CACHE)
@pytest.mark.parametrize("d", [64, 128])
def test_values_near_the_largest_number(rows, held, hq, hkv, d, cache):
    """Their mean is one too, though their sum is not."""
    large = 3.4e38 if cache == "fp32" else 3.3e38
    b, q, out = c = _window_case(rows, held, hq, hkv, d, "fp32", cache)
    q[..., 7] = 2.0 ** -126
    b.pool[:, 0, :, :, 7] = large * torch.sign(b.pool[:, 0, :, :, 7])
    b.pool[:, 1, :, :, 9] = large
    for window, sinks in ((40, 2), (0, 0)):
        got = _run_window(c, window, sinks)
        want, off32, _ = O.window(b, q, out, b.pool, hq, window, sinks)
        O.assert_within(got, want, O.rounded(want, off32, torch.float32))


# few rows of many adapters (shared out among wavefronts), many rows; ranks of one, some and many MFMA steps; more than eight
# slices of k
ADAPTERS = [(16, 520, 200, 5, 12), (5, 264, 1000, 4, 72), (100, 256, 136, 3, 16), (40, 96, 72, 6, 256), (3, 5000, 72, 4, 4)]


@pytest.mark.parametrize("act", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,k,n,adapters,rank", ADAPTERS)
@pytest.mark.parametrize("in_place", [False, True])
def test_adapters_of_infinities(rows, k, n, adapters, rank, act, in_place):
    """One in x, in A or in B, of an adapter of rank 1 and one of all ranks, reaches what it reaches in the formula."""
    inf = float("inf")
    for what in range(3):
        c = _adapter_case(rows, k, n, adapters, rank, act, [i % adapters for i in range(rows)],
                          [1 if i == 1 else rank for i in range(adapters)])
        x, base, a, b = c[:4]
        for i in (1, 2):
            if what == 0:
                x[i, 7] = inf if i == 1 else -inf
            elif what == 1:
                a[i, 0, k - 3] = inf
            else:
                b[i, 9, 0] = -inf
        want, off = O.adapter(*c)
        dev = [t.cuda() for t in c]
        out = dev[1] if in_place else torch.empty_like(dev[1])
        got = P.stage_adapter_add(dev[0], dev[1], out, *dev[2:]).double().cpu()
        odd = ~torch.isfinite(want)
        assert bool(odd.any()) and torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(got[odd]), torch.nan_to_num(want.to(x.dtype)[odd].double()))
        O.assert_within(got[~odd], want[~odd], O.rounded(want, off, x.dtype)[~odd])


@pytest.mark.parametrize("rows,k,n,adapters,rank", ADAPTERS)
def test_adapters_of_numbers_too_large_for_bf16(rows, k, n, adapters, rank):
    """fp32 x and A x between the largest bf16 and the largest fp32."""
    c = _adapter_case(rows, k, n, adapters, rank, "fp32", [i % adapters for i in range(rows)])
    c[0][:, 3] = 3.4e38
    c[2][..., 3] = 2.0 ** -126 * torch.sign(c[2][..., 3])
    want, off = O.adapter(*c)
    O.assert_within(_run_adapter(c), want, O.rounded(want, off, torch.float32))
    c[2].zero_()
    c[2][:, 0, 3] = 1.0                    # t 3.4e38
    c[3][..., 0] = 2.0 ** -126 * torch.sign(c[3][..., 0])
    want, off = O.adapter(*c[:6], torch.ones(adapters))
    O.assert_within(_run_adapter((*c[:6], None)), want, O.rounded(want, off, torch.float32))


@pytest.mark.parametrize("act", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,k,n,adapters,rank", ADAPTERS + [(16, 8200, 4096, 8, 128), (33, 9000, 264, 16, 200), (1, 4104, 8, 4, 68)])
def test_adapters_of_many_ranks_and_slices(rows, k, n, adapters, rank, act):
    ids = [i * 7 % (adapters + 1) - 1 for i in range(rows)]
    ranks = [max(1, rank - 13 * i) for i in range(adapters)]
    _check_adapter(_adapter_case(rows, k, n, adapters, rank, act, ids), _run_adapter(_adapter_case(rows, k, n, adapters, rank, act, ids)))
    c = _adapter_case(rows, k, n, adapters, rank, act, ids, ranks)
    _check_adapter(c, _run_adapter(c))


@pytest.mark.parametrize("act,cache", [("fp32", "bf16"), ("bf16", "bf16"), ("fp32", "fp32"), ("bf16", "fp32")])
@pytest.mark.parametrize("rows,held,hq,hkv", F32_CACHE + [([20, 1, 5], [3000, 90, 1000], 8, 2)])
def test_a_query_that_is_nan_stays_with_its_row(rows, held, hq, hkv, cache, act):
    b, q, out = c = _window_case(rows, held, hq, hkv, 64, act, cache)
    for window, sinks in ((0, 0), (1500, 2)):
        want = _run_window(c, window, sinks)
        at = len(q) - 2
        old = q[at].clone()
        q[at, :, 3::9] = float("nan")
        got = _run_window(c, window, sinks)
        assert bool(torch.isnan(got[at]).all())
        q[at] = old
        got[at] = want[at]
        assert torch.equal(got, want)


@pytest.mark.parametrize("act", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,k,n,adapters,rank", ADAPTERS)
def test_an_input_that_is_nan_stays_with_its_row(rows, k, n, adapters, rank, act):
    c = _adapter_case(rows, k, n, adapters, rank, act, [i % adapters for i in range(rows)])
    want = _run_adapter(c)
    for at in (slice(None), slice(k - 1, None)):
        bad = c[0].clone()
        bad[1, at] = float("nan")
        got = _run_adapter((bad, *c[1:]))
        assert bool(torch.isnan(got[1]).all())
        got[1] = want[1]
        assert torch.equal(got, want)


@pytest.mark.parametrize("act", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,k,n,adapters,rank", ADAPTERS)
def test_adapters_hold_anything_past_their_ranks(rows, k, n, adapters, rank, act):
    ranks = [max(1, rank // 2 - 3 * i) for i in range(adapters)]
    c = _adapter_case(rows, k, n, adapters, rank, act, [i % adapters for i in range(rows)], ranks)
    want = _run_adapter(c)
    for i, r in enumerate(ranks):
        c[2][i, r:], c[3][i, :, r:] = float("nan"), float("inf")
    assert torch.equal(_run_adapter(c), want)


@pytest.mark.parametrize("act,cache", [("fp32", "bf16"), ("bf16", "bf16"), ("fp32", "fp32"), ("bf16", "fp32")])
@pytest.mark.parametrize("rows,held,hq,hkv", F32_CACHE)
def test_a_row_of_scores_of_minus_infinity_becomes_0(rows, held, hq, hkv, cache, act):
    b, q, out = c = _window_case(rows, held, hq, hkv, 64, act, cache)
    q[..., 9] = q[..., 9].abs() + 0.1
    block = b.table[0, :(b.lengths[0] + 15) // 16].long()
    b.pool[block, 0, :, :, 9] = -float("inf")
    got = _run_window(c, 40, 2)
    assert not bool(got[:rows[0]].any()) and bool(torch.isfinite(got).all()) and bool(got[rows[0]:].any(-1).all())
