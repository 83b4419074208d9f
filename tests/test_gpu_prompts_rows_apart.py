"""mcsd_accumulate_weights where the queries of neighbouring rows lie far apart, or are no numbers: what a row gives to the keys does not
depend on the rows beside it, whichever kernel has them (few rows, and blocks of many)."""
import numpy as np
import pytest
import torch

import prompts_reference as ref
from paper_2401_06706_b200 import binding
from prompts_util import DTYPES, attend, attention, check_attention, host, plain_lse, problem, slots_of, within

pytestmark = pytest.mark.gpu

COUNTS = {"few": [3, 2], "many": [90, 70]}


def _weights(p):
    return torch.exp(torch.randn((p.cache.n_pages, p.kv, p.ps), generator=torch.Generator().manual_seed(5))).cuda()


def _run(p, lse, weights):
    got = attention(p).mcsd_accumulate_weights(p.q, lse, p.cache, p.table, p.start, p.cu, weights.clone(), decay=0.5)
    torch.cuda.synchronize()
    return host(got).astype(np.float64)


def _statement(p, lse, weights):
    return ref.accumulate(host(p.q), host(lse), p.cache.pages.cpu().numpy(), host(weights), host(p.table), host(p.start), host(p.cu), p.max_new, p.D, p.ps,
                          p.scale, 0.5, 0)


def _problem(rows, D, dtype, seed=31):
    """Two sequences; the odd row is a token of the first one with others before and behind it."""
    p = problem(seed, [37, 140], COUNTS[rows], 8, 2, D, 16, dtype)
    return p, COUNTS[rows][0] // 2


@pytest.mark.parametrize("rows", sorted(COUNTS))
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("power", [13, 28, 34, 40, 100])
def test_a_loud_row_of_no_weight_leaves_the_others_exact(rows, D, power):
    """(lse of +inf: the loud row itself gives nothing, so that the tolerance is that of the others.)"""
    p, token = _problem(rows, D, torch.bfloat16)
    lse, w = plain_lse(p), _weights(p)
    p.q[token, 1] *= 2.0 ** power
    lse[token, 1] = float("inf")
    want, tol = _statement(p, lse, w)
    within(_run(p, lse, w), want, tol, "weights")


@pytest.mark.parametrize("rows", sorted(COUNTS))
@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("factor", [2.0 ** 12, 2.0 ** 13, 2.0 ** -13, 0.0])
def test_a_row_far_from_the_others_counts_by_its_own_lse(rows, dtype, D, factor):
    """(Queries below the smallest half are zeros in fp16, which the statement sees as well. The scores' slack is about 1 at 2^13.)"""
    p, token = _problem(rows, D, DTYPES[dtype])
    p.q[token, 1] *= factor
    lse, w = plain_lse(p), _weights(p)
    want, tol = _statement(p, lse, w)
    within(_run(p, lse, w), want, tol, "weights")


@pytest.mark.parametrize("rows", sorted(COUNTS))
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_a_row_that_is_no_number_spoils_what_it_sees_only(rows, D, dtype, value):
    """Keys that the row sees become NaN with the lse that the attention gives it; those behind it, and those of the other key head, are exact."""
    p, token = _problem(rows, D, DTYPES[dtype])
    p.q[token, 1, 7] = value
    lse = attention(p).mcsd_chunk_attention(p.q, p.cache, p.table, p.start, p.cu).lse.clone()
    w = _weights(p)
    assert torch.isnan(lse[token, 1]) and int(torch.isnan(lse).sum()) == 1
    got = _run(p, lse, w)
    p.q[token, 1], lse[token, 1] = 0.0, float("-inf")
    want, tol = _statement(p, lse, w)
    seen = slots_of(p, 0, range(int(p.start[0]) + token + 1)).cpu().numpy()
    want[seen // 16, 0, seen % 16] = np.nan
    within(got, want, tol, "weights")


@pytest.mark.parametrize("rows", sorted(COUNTS))
@pytest.mark.parametrize("value", [1.0, 2.0 ** 60, float("inf"), float("nan")])
def test_rows_without_an_lse_count_nothing_whatever_their_queries(rows, value):
    p, token = _problem(rows, 128, torch.bfloat16)
    lse, w = plain_lse(p), _weights(p)
    p.q[token, 1, 5], lse[token, 1] = value, float("-inf")
    got = _run(p, lse, w)
    p.q[token, 1] = 0.0
    want, tol = _statement(p, lse, w)
    within(got, want, tol, "weights")


@pytest.mark.parametrize("rows", sorted(COUNTS))
def test_rows_without_an_lse_count_nothing_whatever_the_keys(rows):
    """The last token alone sees the last key, which is NaN, and counts nothing: that key starts at 0."""
    p, _ = _problem(rows, 64, torch.bfloat16)
    lse, w = plain_lse(p), _weights(p)
    n = COUNTS[rows][0]
    last = slots_of(p, 0, [int(p.start[0]) + n - 1])
    bad = torch.full((1, 2, 64), float("nan"), device="cuda")
    binding.mcsd_append_kv(p.cache, bad, bad, last)
    lse[n - 1] = float("-inf")
    got = _run(p, lse, w)
    want, tol = _statement(p, lse, w)
    at = int(last)
    assert (want[at // 16, :, at % 16] == 0).all()
    within(got, want, tol, "weights")


@pytest.mark.parametrize("rows", sorted(COUNTS))
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_attention_of_the_rows_beside_one_that_is_no_number(rows, D, value):
    p, token = _problem(rows, D, torch.bfloat16)
    p.q[token, 1, 7] = value
    r = attend(p)
    check_attention(p, r)
    odd = torch.isnan(r.out).any(-1)
    assert bool(odd[token, 1]) and int(odd.sum()) == 1
