"""Chunks of the same sequences in batches of another make-up: alone, in another order, among others, with a larger bound on the tokens (which
changes the kernels that a call takes and how the work is cut). Every result is held to the statement, and the results to one another."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch

import prompts_reference as ref
from prompts_util import DTYPES, attend, attention, check_attention, host, problem, within

pytestmark = pytest.mark.gpu


def _of(p, order):
    """The sequences `order` of a problem, in that order, and where their tokens lie in it."""
    cu = p.cu.tolist()
    rows = [r for b in order for r in range(cu[b], cu[b + 1])]
    counts = [cu[b + 1] - cu[b] for b in order]
    new = SimpleNamespace(**vars(p))
    new.B, new.q, new.table, new.start = len(order), p.q[rows].contiguous(), p.table[order].contiguous(), p.start[order].contiguous()
    new.cu = torch.tensor([0] + np.cumsum(counts).tolist(), dtype=torch.int32, device="cuda")
    new.max_new = max(counts)
    return new, rows


def _runs(p):
    """(sequences, bound on the tokens) of the calls that are compared."""
    n = p.B
    top = p.max_new
    yield list(range(n)), top
    yield list(range(n))[::-1], top
    yield list(range(n)), 3 * top + 200              # (few tokens for so large a bound: both kernels)
    for b in range(n):
        count = int(p.cu[b + 1] - p.cu[b])
        yield [b], count
        yield [b], count + 300                       # (alone, in the kernel of many rows or in both)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("heads,kv,D", [(4, 1, 128), (8, 2, 64), (3, 3, 128)])
@pytest.mark.parametrize("counts", [[2, 1, 2, 5], [200, 1, 90, 33]])
def test_attention_of_a_sequence_in_any_batch(dtype, heads, kv, D, counts):
    """Out and lse of a token in any two calls differ by what the statement allows both of them."""
    p = problem(41, [900, 30, 2000, 0], counts, heads, kv, D, 16, DTYPES[dtype])
    want, want_lse, tol, tol_lse = ref.chunk_attention(host(p.q), p.cache.pages.cpu().numpy(), host(p.table), host(p.start), host(p.cu), p.max_new, D, 16, p.scale,
                                                       torch.finfo(p.q.dtype).eps)
    low, high = np.full(want.shape, np.inf), np.full(want.shape, -np.inf)
    low_lse, high_lse = np.full(want_lse.shape, np.inf), np.full(want_lse.shape, -np.inf)
    for order, bound in _runs(p):
        part, rows = _of(p, order)
        r = attend(part, bound)
        out, lse = host(r.out).astype(np.float64), host(r.lse).astype(np.float64)
        within(out, want[rows], tol[rows], ("out", order, bound))
        within(lse, want_lse[rows], tol_lse[rows], ("lse", order, bound))
        low[rows], high[rows] = np.minimum(low[rows], out), np.maximum(high[rows], out)
        low_lse[rows], high_lse[rows] = np.minimum(low_lse[rows], lse), np.maximum(high_lse[rows], lse)
    assert np.isfinite(low).all() and (high - low <= 2 * tol).all() and (high_lse - low_lse <= 2 * tol_lse).all()


@pytest.mark.parametrize("counts", [[2, 1, 2, 5], [200, 1, 90, 33]])
def test_weights_of_a_sequence_in_any_batch(counts):
    p = problem(42, [900, 30, 2000, 0], counts, 8, 2, 128, 16, torch.bfloat16)
    lse = torch.tensor(ref.chunk_attention(host(p.q), p.cache.pages.cpu().numpy(), host(p.table), host(p.start), host(p.cu), p.max_new, 128, 16, p.scale,
                                           2.0 ** -8)[1], dtype=torch.float32).cuda()
    w = torch.exp(torch.randn((p.cache.n_pages, 2, 16), generator=torch.Generator().manual_seed(5))).cuda()
    for order, bound in _runs(p):
        part, rows = _of(p, order)
        got = attention(part, bound).mcsd_accumulate_weights(part.q, lse[rows], p.cache, part.table, part.start, part.cu, w.clone(), decay=0.5)
        torch.cuda.synchronize()
        want, tol = ref.accumulate(host(part.q), host(lse[rows]), p.cache.pages.cpu().numpy(), host(w), host(part.table), host(part.start), host(part.cu), bound, 128,
                                   16, p.scale, 0.5, 0)
        within(host(got).astype(np.float64), want, tol, ("weights", order, bound))


def test_a_repeated_call_gives_the_same_bits():
    p = problem(43, [900, 30, 2000], [200, 1, 90], 4, 1, 128, 16, torch.bfloat16)
    r, again = attend(p), attend(p)
    check_attention(p, r)
    assert torch.equal(r.out, again.out) and torch.equal(r.lse, again.lse)
