"""mcsd_accumulate_weights and mcsd_evict_rows against plain statements."""
import numpy as np
import pytest
import torch

import prompts_reference as ref
from paper_2401_06706_b200 import binding
from prompts_util import DTYPES, attention, host, plain_lse, problem, slots_of, within

pytestmark = pytest.mark.gpu


def _weights(p, seed=5):
    return torch.exp(torch.randn((p.cache.n_pages, p.kv, p.ps), generator=torch.Generator().manual_seed(seed))).cuda()


def _run(p, lse, weights, *, decay=1.0, last=0, scale=None, max_new=None):
    a = attention(p, max_new)
    got = a.mcsd_accumulate_weights(p.q, lse, p.cache, p.table, p.start, p.cu, weights.clone(), scale=scale, decay=decay, last_tokens=last)
    torch.cuda.synchronize()
    return got


def _check(p, lse, weights, got, *, decay=1.0, last=0, scale=None, max_new=None):
    want, tol = ref.accumulate(host(p.q), host(lse), p.cache.pages.cpu().numpy(), host(weights), host(p.table), host(p.start), host(p.cu),
                               max_new or p.max_new, p.D, p.ps, p.scale if scale is None else scale, decay, last)
    within(host(got).astype(np.float64), want, tol, "weights")


RAGGED = [([0, 1, 37, 130], [1, 1, 1, 1]), ([0, 5, 40, 127], [3, 1, 5, 2]), ([0, 0, 131, 20], [1, 70, 129, 0]), ([250, -1, 0], [40, 0, 33])]


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("D,ps", [(128, 16), (64, 16), (128, 64), (64, 128)])
@pytest.mark.parametrize("heads,kv", [(1, 1), (4, 1), (7, 1), (6, 2), (40, 1)])
@pytest.mark.parametrize("lengths", range(len(RAGGED)))
def test_against_reference(dtype, D, ps, heads, kv, lengths):
    starts, counts = RAGGED[lengths]
    p = problem(heads + lengths, starts, counts, heads, kv, D, ps, DTYPES[dtype])
    lse, w = plain_lse(p), _weights(p)
    for last, decay in ((0, 1.0), (2, 0.5), (32, 0.0)):
        _check(p, lse, w, _run(p, lse, w, decay=decay, last=last), decay=decay, last=last)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("last", [0, 1, 31, 32, 33, 300])
def test_lengths_around_every_border(D, last):
    starts = [0, 0, 0, 127, 128, 129, 1, 1000, 255, 256]
    counts = [1, 127, 300, 1, 2, 64, 257, 65, 63, 1]
    p = problem(3, starts, counts, 4, 1, D, 16, torch.float16)
    lse, w = plain_lse(p), _weights(p)
    _check(p, lse, w, _run(p, lse, w, last=last, decay=0.9), last=last, decay=0.9)


@pytest.mark.parametrize("counts", [[2, 0, 3, 1], [70, 0, 90, 140]])
def test_unused_entries_missing_pages_and_odd_lse(counts):
    p = problem(14, [100, -1, 60, 20], counts, 3, 1, 64, 16, torch.float16)
    lse, w = plain_lse(p), _weights(p)
    p.table[0, 2] = -1
    p.table[3, 1] = p.cache.n_pages
    lse[0, 0], lse[1, 1] = -np.inf, np.inf           # a row that saw nothing; one of no weight
    _check(p, lse, w, _run(p, lse, w), max_new=None)
    used = torch.unique(p.table[(p.table >= 0) & (p.table < p.cache.n_pages)])
    others = torch.tensor(sorted(set(range(p.cache.n_pages)) - set(used.tolist())), device="cuda")
    assert torch.equal(_run(p, lse, w)[others], w[others])
    lse[2, 0] = float("nan")                         # what such a row sees becomes NaN, nothing else
    _check(p, lse, w, _run(p, lse, w))


@pytest.mark.parametrize("count", [3, 150])
def test_new_rows_start_at_zero_and_hidden_rows_do_not_leak(count):
    """Weights and rows behind the sequence may be anything; rows of new tokens do not read what the page held."""
    p = problem(15, [50, 0], [count, count], 4, 2, 128, 16, torch.bfloat16)
    lse, w = plain_lse(p), _weights(p)
    for b in range(2):
        n, end = int(p.start[b]) + count, p.table.shape[1] * 16
        new = slots_of(p, b, range(int(p.start[b]), n))
        w[new // 16, :, new % 16] = float("nan")
        room = [x for x in range(n, end) if int(p.table[b, x // 16]) >= 0]
        if room:
            behind = slots_of(p, b, room)
            bad = torch.full((len(room), 2, 128), float("nan"), device="cuda")
            binding.mcsd_append_kv(p.cache, bad, bad, behind)
    got = _run(p, lse, w, decay=0.5)
    _check(p, lse, w, got, decay=0.5)
    for b in range(2):
        own = slots_of(p, b, range(int(p.start[b]) + count))
        assert torch.isfinite(got[own // 16, :, own % 16]).all()
    w[:] = float("nan")                              # decay 0 reads nothing
    got = _run(p, lse, w, decay=0.0)
    for b in range(2):
        own = slots_of(p, b, range(int(p.start[b]) + count))
        assert torch.isfinite(got[own // 16, :, own % 16]).all()


def test_other_scales_and_large_queries():
    for factor, scale in ((1.0, -0.3), (1.0, 0.0), (1e4, None), (1e-6, None)):
        p = problem(16, [200, 13], [90, 2], 4, 1, 128, 16, torch.bfloat16)
        p.q *= factor
        s = float(np.float32(0.09 / factor)) if scale is None else scale
        lse, w = plain_lse(p, s), _weights(p)
        _check(p, lse, w, _run(p, lse, w, scale=s), scale=s)


@pytest.mark.parametrize("count", [3, 75])
@pytest.mark.parametrize("pad", [0, 8, 3])
def test_strided_queries(count, pad):
    p = problem(17, [33, 64, 5], [count, 1, count + 4], 6, 2, 64, 16, torch.bfloat16)
    lse, w = plain_lse(p), _weights(p)
    T, H, D = p.q.shape
    fused = torch.randn((T, H * D + pad), device="cuda").to(torch.bfloat16)
    fused[:, pad:] = p.q.flatten(1)
    want = _run(p, lse, w)
    p.q = fused[:, pad:].unflatten(1, (H, D))
    assert torch.equal(_run(p, lse, w), want)
    _check(p, lse, w, want)


def test_counts_that_do_not_fit():
    p = problem(18, [20, 0, 33], [80, 40, 1], 4, 2, 128, 16, torch.bfloat16)
    lse, w = plain_lse(p), _weights(p)
    for max_new in (2, 50):
        _check(p, lse, w, _run(p, lse, w, max_new=max_new), max_new=max_new)


def test_weights_of_an_attention_sum_to_its_rows():
    """With the attention's own lse the weights of a sequence add up to the rows that saw them; whatever the batch, the same bits again."""
    p = problem(19, [900, 30, 2000, 0], [200, 1, 40, 700], 8, 2, 128, 16, torch.bfloat16)
    a = attention(p)
    r = a.mcsd_chunk_attention(p.q, p.cache, p.table, p.start, p.cu)
    w = torch.zeros((p.cache.n_pages, 2, 16), device="cuda")
    a.mcsd_accumulate_weights(p.q, r.lse, p.cache, p.table, p.start, p.cu, w, decay=0.0)
    for b in range(p.B):
        own = slots_of(p, b, range(int(p.start[b]) + int(p.cu[b + 1] - p.cu[b])))
        rows = 4 * int(p.cu[b + 1] - p.cu[b])
        assert (w[own // 16, :, own % 16].double().sum(0) - rows).abs().max() < 2e-5 * rows
    again = torch.zeros_like(w)
    a.mcsd_accumulate_weights(p.q, r.lse, p.cache, p.table, p.start, p.cu, again, decay=0.0)
    assert torch.equal(w, again)


def test_capture_and_replay():
    p = problem(20, [70, 300, 0], [100, 1, 30], 4, 2, 128, 16, torch.bfloat16)
    lse, w = plain_lse(p), _weights(p)
    want = _run(p, lse, w, decay=0.5)
    a, start, mine = attention(p), torch.zeros_like(p.start), w.clone()
    a.mcsd_accumulate_weights(p.q, lse, p.cache, p.table, start, p.cu, mine.clone(), decay=0.5)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.mcsd_accumulate_weights(p.q, lse, p.cache, p.table, start, p.cu, mine, decay=0.5)
    start.copy_(p.start)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(mine, want)


# ---------------------------------------------------------------- eviction
def _evict_problem(seed, lengths, layers, heads, D, ps, *, zeros=0.2):
    g = torch.Generator().manual_seed(seed)
    need = [-(-max(n, 0) // ps) for n in lengths]
    n_pages = sum(need) + 2
    ids = torch.randperm(n_pages, generator=g).to(torch.int32)
    table = torch.full((len(lengths), max(max(need), 1)), -1, dtype=torch.int32)
    at = 0
    for b, k in enumerate(need):
        table[b, :k] = ids[at:at + k]
        at += k
    pages = torch.randint(0, 256, (layers, n_pages, heads, ps * (D + 8)), generator=g, dtype=torch.uint8)
    w = torch.exp(2 * torch.randn((layers, n_pages, heads, ps), generator=g))
    w[torch.rand(w.shape, generator=g) < zeros] = 0.0
    w[torch.rand(w.shape, generator=g) < 0.05] = -0.0
    return pages, w, table, torch.tensor(lengths, dtype=torch.int32)


def _evict(pages, w, table, length, keep, sink, recent, D, ps, **kw):
    cache = binding.KvCache(pages.cuda(), D, ps)
    weights = w.cuda()
    out = binding.mcsd_evict_rows(cache, weights, table.cuda(), length.cuda(), keep.cuda() if isinstance(keep, torch.Tensor) else keep, sink=sink, recent=recent, **kw)
    torch.cuda.synchronize()
    return cache.pages.cpu().numpy(), weights.cpu().numpy(), out.cpu().numpy()


def _same(got, want):
    assert np.array_equal(got[2], want[2])
    assert np.array_equal(got[1].view(np.uint32), want[1].astype(np.float32).view(np.uint32))
    assert np.array_equal(got[0], want[0])


@pytest.mark.parametrize("D,ps", [(128, 16), (64, 16), (128, 64), (64, 128)])
@pytest.mark.parametrize("keep,sink,recent", [(40, 4, 8), (100, 0, 0), (1, 0, 0), (0, 3, 3), (64, 64, 5), (64, 70, 70), (50, 0, 50), (33, 1, 31), (10**6, 1, 1)])
def test_evict_against_reference(D, ps, keep, sink, recent):
    pages, w, table, length = _evict_problem(keep + ps, [130, 0, 1, 41, 300, 64, -1], 2, 2, D, ps)
    got = _evict(pages, w, table, length, keep, sink, recent, D, ps)
    _same(got, ref.evict(pages.numpy(), w.numpy(), table.numpy(), length.numpy(), [keep] * 7, sink, recent, D, ps))


@pytest.mark.parametrize("length", [255, 256, 257, 1023, 1025, 2600, 7200, 9000])
@pytest.mark.parametrize("share", [0.02, 0.5, 0.97])
def test_evict_long_sequences(length, share):
    pages, w, table, n = _evict_problem(length, [length], 1, 2, 64, 16)
    keep = int(length * share) + 1
    got = _evict(pages, w, table, n, keep, 3, min(20, keep // 2), 64, 16)
    _same(got, ref.evict(pages.numpy(), w.numpy(), table.numpy(), n.numpy(), [keep], 3, min(20, keep // 2), 64, 16))


def test_evict_keep_per_sequence_ties_and_odd_weights():
    """A budget for each sequence; all weights equal; NaN, infinities and both zeros; negative ones; pages that are not there."""
    pages, w, table, length = _evict_problem(7, [200, 150, 170, 90, 300], 2, 1, 64, 16)
    w[:, table[0, :13].long()] = 1.5
    own = w[:, table[2, :11].long()]
    own[..., ::3], own[..., 1::5], own[..., 2::7] = float("nan"), float("inf"), -float("inf")
    w[:, table[2, :11].long()] = own
    w[:, table[4, :19].long()] *= -1
    table[3, 1] = -1
    table[3, 4] = 10**6
    keep = torch.tensor([77, -1, 60, 50, 299], dtype=torch.int32)
    got = _evict(pages, w, table, length, keep, 2, 9, 64, 16)
    _same(got, ref.evict(pages.numpy(), w.numpy(), table.numpy(), length.numpy(), keep.tolist(), 2, 9, 64, 16))


def test_evict_rows_beyond_the_table_and_a_single_layer():
    pages, w, table, _ = _evict_problem(9, [100, 100], 1, 3, 64, 16)
    length = torch.tensor([10**9, 60], dtype=torch.int32)
    got = _evict(pages[0], w[0], table, length, 30, 2, 5, 64, 16)
    want = ref.evict(pages.numpy(), w.numpy(), table.numpy(), length.numpy(), [30, 30], 2, 5, 64, 16)
    _same((got[0][None], got[1][None], got[2]), want)


def test_evict_random_shapes():
    g = np.random.default_rng(3)
    for i in range(25):
        lengths = g.integers(-1, 400, size=g.integers(1, 5)).tolist()
        D, ps = int(g.choice([64, 128])), int(g.choice([16, 32, 64, 128]))
        pages, w, table, length = _evict_problem(100 + i, lengths, int(g.integers(1, 4)), int(g.integers(1, 4)), D, ps, zeros=float(g.choice([0.0, 0.3, 0.9])))
        keep, sink, recent = int(g.integers(0, 300)), int(g.integers(0, 40)), int(g.integers(0, 100))
        got = _evict(pages, w, table, length, keep, sink, recent, D, ps)
        _same(got, ref.evict(pages.numpy(), w.numpy(), table.numpy(), length.numpy(), [keep] * len(lengths), sink, recent, D, ps))


def test_evict_captured_and_repeated():
    """A captured call follows what it finds, and a second one over the first one's result does nothing."""
    pages, w, table, length = _evict_problem(11, [180, 333], 2, 2, 64, 16)
    want = ref.evict(pages.numpy(), w.numpy(), table.numpy(), length.numpy(), [90, 90], 4, 16, 64, 16)
    cache, weights, table, length = binding.KvCache(pages.cuda(), 64, 16), w.cuda(), table.cuda(), length.cuda()
    now, out = torch.zeros_like(length), torch.zeros_like(length)
    binding.mcsd_evict_rows(cache, weights, table, now, 90, sink=4, recent=16, len_out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.mcsd_evict_rows(cache, weights, table, now, 90, sink=4, recent=16, len_out=out)
    now.copy_(length)
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        _same((cache.pages.cpu().numpy(), weights.cpu().numpy(), out.cpu().numpy()), want)
        now.copy_(out)


def test_evict_beyond_four_gigabytes():
    """Layers whose offsets pass 32 bits; weights whose index does."""
    D, ps, heads = 64, 16, 1
    pages, w, table, length = _evict_problem(12, [100], 2, heads, D, ps)
    want = ref.evict(pages.numpy(), w.numpy(), table.numpy(), length.numpy(), [40], 2, 5, D, ps)
    n_pages = 5 * 2**30 // (ps * (D + 8))
    big = torch.zeros((2, n_pages, heads, ps * (D + 8)), dtype=torch.uint8, device="cuda")
    weights = torch.zeros((2, n_pages, heads, ps), device="cuda")
    n = pages.shape[1]
    big[:, -n:], weights[:, -n:] = pages.cuda(), w.cuda()
    cache = binding.KvCache(big, D, ps)
    out = binding.mcsd_evict_rows(cache, weights, torch.where(table >= 0, table + n_pages - n, -1).cuda(), length.cuda(), 40, sink=2, recent=5)
    _same((big[:, -n:].cpu().numpy(), weights[:, -n:].cpu().numpy(), out.cpu().numpy()), want)
