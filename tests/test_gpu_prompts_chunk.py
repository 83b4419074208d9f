"""mcsd_chunk_attention against a plain statement in 64 bits, at the sizes and masks where it can go wrong."""
import numpy as np
import pytest
import torch

from paper_2401_06706_b200 import binding
from prompts_util import DTYPES, attend, attention, check_attention, host, problem, slots_of

pytestmark = pytest.mark.gpu

HEADS = [(1, 1), (4, 1), (7, 1), (6, 2), (40, 1)]
RAGGED = [([0, 1, 37, 130], [1, 1, 1, 1]), ([0, 5, 40, 127], [3, 1, 5, 2]), ([0, 0, 131, 20], [1, 70, 129, 0]), ([250, -1, 0], [40, 0, 33])]


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("D,ps", [(128, 16), (64, 16), (128, 64), (64, 128)])
@pytest.mark.parametrize("heads,kv", HEADS)
@pytest.mark.parametrize("lengths", range(len(RAGGED)))
def test_against_reference(dtype, D, ps, heads, kv, lengths):
    starts, counts = RAGGED[lengths]
    p = problem(heads + lengths, starts, counts, heads, kv, D, ps, DTYPES[dtype])
    check_attention(p, attend(p))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("heads", [1, 4])
def test_lengths_around_every_border(D, heads):
    """Chunks and prefixes on both sides of the tiles' borders, long ones among them, in one batch."""
    starts = [0, 0, 0, 0, 0, 127, 128, 129, 1, 1000, 255, 256, 63, 64]
    counts = [1, 127, 128, 129, 300, 1, 2, 64, 257, 65, 63, 1, 512, 31]
    p = problem(3, starts, counts, heads, 1, D, 16, torch.bfloat16)
    check_attention(p, attend(p))


@pytest.mark.parametrize("heads,count", [(1, 24), (1, 25), (1, 48), (1, 49), (1, 72), (1, 73), (4, 6), (4, 12), (4, 18), (4, 19), (7, 10), (7, 11), (13, 5), (24, 3), (25, 2)])
def test_rows_around_the_blocks_borders(heads, count):
    """One block of few rows, two and three, and the first chunk that is too long for them; queries of one key head."""
    p = problem(5, [700, 0, 1300], [count, count, 1], heads, 1, 128, 16, torch.bfloat16)
    check_attention(p, attend(p, max_new=count))


@pytest.mark.parametrize("heads", [4, 32])
def test_one_long_sequence(heads):
    """Few rows over a long prefix: the work of a block is divided and joined."""
    p = problem(4, [5000], [9], heads, 1, 128, 32, torch.float16)
    check_attention(p, attend(p))
    check_attention(p, attend(p, max_new=400))       # (as a call would choose for longer chunks)


@pytest.mark.parametrize("loud", [12.0, 60.0])
@pytest.mark.parametrize("count", [2, 90])
def test_loud_keys(loud, count):
    """Scores far apart: the running maximum moves often and by much; a weight of one next to zeros."""
    p = problem(8, [300, 0], [count, count], 4, 1, 128, 16, torch.float16, loud=loud)
    check_attention(p, attend(p))


@pytest.mark.parametrize("count", [2, 90])
def test_rising_and_falling_scores(count):
    p = problem(9, [600, 600], [count, count], 4, 1, 64, 16, torch.bfloat16)
    ramp = torch.linspace(0.1, 40.0, 600).view(600, 1, 1)
    base = torch.randn((1, 1, 64), generator=torch.Generator().manual_seed(1))
    for b, r in enumerate((ramp, ramp.flip(0))):
        binding.mcsd_append_kv(p.cache, (r * base).cuda(), torch.randn((600, 1, 64), device="cuda"), slots_of(p, b, range(600)))
    p.q[:] = (base * 2).to(p.q.dtype).cuda()
    check_attention(p, attend(p))


@pytest.mark.parametrize("size", [1e-3, 1e-6, 3e4, 6.5e4])
@pytest.mark.parametrize("count", [2, 90])
def test_small_and_large_values(size, count):
    """Values far from one, tokens of very different size side by side, and values up to the end of half's range."""
    p = problem(10, [400], [count], 4, 1, 128, 16, torch.bfloat16 if size > 1 else torch.float16)
    n = 400 + count
    v = torch.randn((n, 1, 128), generator=torch.Generator().manual_seed(2)) * size / 4
    v[100:110] *= 0.01
    v[7] = size                                      # (a row without a range)
    v[8, :, :64], v[8, :, 64:] = size, -size
    k = torch.randn((n, 1, 128), generator=torch.Generator().manual_seed(3))
    binding.mcsd_append_kv(p.cache, k.cuda(), v.cuda(), slots_of(p, 0, range(n)))
    check_attention(p, attend(p))


@pytest.mark.parametrize("count", [2, 90])
@pytest.mark.parametrize("loud", [1e3, 3e4])
def test_a_loud_value_of_small_weight_takes_no_bits(count, loud):
    """One value is loud and hardly weighed: the others keep their precision (its share is of their size)."""
    p = problem(11, [200], [count], 2, 1, 64, 16, torch.float16)
    n = 200 + count
    k = 0.05 * torch.randn((n, 1, 64), generator=torch.Generator().manual_seed(2))
    v = torch.randn((n, 1, 64), generator=torch.Generator().manual_seed(3))
    p.q[:] = 1.0
    k[77], v[77] = -np.log(loud) * 8 / 64, v[77] * loud                   # its weight is 1 / loud
    binding.mcsd_append_kv(p.cache, k.cuda(), v.cuda(), slots_of(p, 0, range(n)))
    r = attend(p)
    check_attention(p, r)
    rest = host(r.out)
    assert np.abs(rest).max() < 4


@pytest.mark.parametrize("scale", [0.0, -0.3, 1.7, 1e-4])
@pytest.mark.parametrize("count", [2, 90])
def test_other_scales(scale, count):
    p = problem(11, [200, 13], [count, 1], 2, 1, 64, 32, torch.bfloat16)
    check_attention(p, attend(p, scale=scale), scale=scale)


@pytest.mark.parametrize("factor", [1e-6, 1e4])
@pytest.mark.parametrize("count", [2, 90])
def test_small_and_large_queries(factor, count):
    """bf16 queries outside the range of half precision, rows of zeros among them."""
    p = problem(12, [200, 13], [count, 1], 4, 1, 128, 16, torch.bfloat16)
    p.q *= factor
    p.q[0, 0] = 0
    p.q[-1, -1, :64] = 0
    scale = float(np.float32(0.09 / factor))
    check_attention(p, attend(p, scale=scale), scale=scale)


@pytest.mark.parametrize("count", [5, 140])
@pytest.mark.parametrize("D", [64, 128])
def test_hidden_positions_do_not_leak(count, D):
    """NaN rows behind a sequence, in its last page and in others: nothing of them is seen. One in the chunk: the tokens from there on."""
    p = problem(13, [40, 0, 131], [count, count - 2, 1], 4, 2, D, 16, torch.bfloat16)
    used = set()
    for b in range(3):
        used |= set(slots_of(p, b, range(int(p.start[b]) + int(p.cu[b + 1] - p.cu[b]))).tolist())
    free = torch.tensor(sorted(set(range(p.cache.n_pages * 16)) - used), device="cuda")
    bad = torch.full((max(free.numel(), 3), 2, D), float("nan"), device="cuda")
    binding.mcsd_append_kv(p.cache, bad[:free.numel()], bad[:free.numel()], free)
    r = attend(p)
    assert torch.isfinite(r.out).all() and torch.isfinite(r.lse).all()
    check_attention(p, r)
    for values_only in (True, False):                # a NaN value, then a NaN key as well, at token 2 of the first two sequences
        for b in range(2):
            keys = torch.randn((1, 2, D), device="cuda") if values_only else bad[:1]
            binding.mcsd_append_kv(p.cache, keys, bad[:1], slots_of(p, b, [int(p.start[b]) + 2]))
        r = attend(p)
        hit = torch.zeros(p.q.shape[0], dtype=torch.bool, device="cuda")
        for b in range(2):
            hit[int(p.cu[b]) + 2:int(p.cu[b + 1])] = True
        assert torch.isnan(r.out[hit]).all() and torch.isfinite(r.out[~hit]).all()
        assert torch.isfinite(r.lse[hit]).all() == values_only and torch.isfinite(r.lse[~hit]).all()
        check_attention(p, r)


@pytest.mark.parametrize("counts", [[2, 0, 3, 1, 4], [70, 0, 90, 1, 40]])
def test_unused_entries_missing_pages_and_empty_rows(counts):
    p = problem(14, [100, -1, 60, 20, 300], counts, 3, 1, 64, 16, torch.float16, pad_tokens=3)
    p.table[0, 2] = -1                               # a hole in the prefix
    p.table[2, :] = p.cache.n_pages + 3              # no page at all: rows of 0 with lse -inf
    p.start[3] = 2**31 - 10                          # longer than the table: what is there counts
    p.table[4, 300 // 16:] = -1                      # the chunk's own positions are missing
    a = attention(p)
    a.out.fill_(3.0)
    a.lse.fill_(4.0)
    r = a.mcsd_chunk_attention(p.q, p.cache, p.table, p.start, p.cu)
    torch.cuda.synchronize()
    mine = check_attention(p, r)
    assert (r.out[~torch.tensor(mine)] == 3).all() and (r.lse[~torch.tensor(mine)] == 4).all() and (~mine).sum() == 3
    at = slice(int(p.cu[2]), int(p.cu[3]))
    assert (r.out[at] == 0).all() and torch.isneginf(r.lse[at]).all()


@pytest.mark.parametrize("counts", [[3, 4, 2], [80, 40, 1]])
def test_counts_that_do_not_fit(counts):
    """max_new below a count, and fewer rows of q than cu_tokens says: the rest is left as it was."""
    p = problem(15, [20, 0, 33], counts, 4, 2, 128, 16, torch.bfloat16)
    for max_new, rows in ((2, sum(counts)), (max(counts), sum(counts) - 2), (max(counts), counts[0] - 1)):
        a = attention(p, max_new)
        a.out.fill_(3.0)
        a.lse.fill_(4.0)
        full, p.q = p.q, p.q[:rows]
        r = a.mcsd_chunk_attention(p.q, p.cache, p.table, p.start, p.cu)
        torch.cuda.synchronize()
        mine = torch.tensor(check_attention(p, r, max_new))
        assert (r.out[~mine] == 3).all() and (r.lse[~mine] == 4).all() and (a.out[rows:] == 3).all()
        p.q = full


@pytest.mark.parametrize("count", [3, 75])
@pytest.mark.parametrize("pad", [0, 8, 3])
def test_strided_queries_outputs_and_tables(count, pad):
    """q as a slice of a fused projection at an odd offset, out inside a larger tensor, a table with padding, out in place of q."""
    p = problem(15, [33, 64, 5], [count, 1, count + 4], 6, 2, 64, 16, torch.bfloat16)
    T, H, D = p.q.shape
    fused = torch.randn((T, H * D + 2 * 2 * D + pad), device="cuda").to(torch.bfloat16)
    fused[:, pad:pad + H * D] = p.q.flatten(1)
    qs = fused[:, pad:pad + H * D].unflatten(1, (H, D))
    wide = torch.full((p.B, p.table.shape[1] + 3), 10**6, dtype=torch.int32, device="cuda")
    wide[:, :p.table.shape[1]] = p.table
    big = torch.full((T, H, D + pad), 2.0, device="cuda").to(torch.bfloat16)
    a = attention(p)
    r = a.mcsd_chunk_attention(qs, p.cache, wide[:, :p.table.shape[1]], p.start, p.cu, out=big[..., :D])
    torch.cuda.synchronize()
    check_attention(p, r)
    assert (big[..., D:] == 2).all()
    inplace = p.q.clone()
    r2 = a.mcsd_chunk_attention(inplace, p.cache, p.table, p.start, p.cu, out=inplace)
    assert torch.equal(inplace, big[..., :D])
    no_lse = attention(p, want_lse=False).mcsd_chunk_attention(p.q, p.cache, p.table, p.start, p.cu)
    assert no_lse.lse is None and torch.equal(no_lse.out, inplace)


def test_the_widest_group():
    """128 query heads on one key head."""
    for counts in ([1, 1], [3, 2], [9, 1]):
        p = problem(16, [140, 3], counts, 128, 1, 64, 16, torch.float16)
        check_attention(p, attend(p))


def test_many_sequences():
    """More sequences than lanes and CTAs, decoding ones among chunks and unused ones."""
    g = torch.Generator().manual_seed(17)
    starts = torch.randint(0, 90, (210,), generator=g).tolist()
    counts = [(1, 1, 40, 0, 3)[i % 5] for i in range(210)]
    starts = [-1 if i % 35 == 3 else s for i, s in enumerate(starts)]
    p = problem(17, starts, counts, 2, 1, 64, 16, torch.bfloat16)
    check_attention(p, attend(p))


def _exact(p, b, rows):
    """Outputs and lse of tokens `rows` of sequence b in 64 bits on the GPU."""
    at, n = int(p.cu[b]), int(p.start[b]) + int(p.cu[b + 1] - p.cu[b])
    k, v = (torch.empty((n, p.kv, p.D), dtype=torch.float32, device="cuda") for _ in range(2))
    binding.mcsd_read_kv(p.cache, slots_of(p, b, range(n)), keys=k, values=v)
    rows = torch.as_tensor(rows, device="cuda")
    group = p.heads // p.kv
    s = torch.einsum("thd,nhd->thn", p.q[at + rows].double(), k.double().repeat_interleave(group, 1)) * p.scale
    s.masked_fill_((torch.arange(n, device="cuda") > int(p.start[b]) + rows[:, None])[:, None], float("-inf"))
    w = torch.softmax(s, -1)
    return torch.einsum("thn,nhd->thd", w, v.double().repeat_interleave(group, 1)), torch.logsumexp(s, -1)


@pytest.mark.parametrize("heads,kv,D", [(8, 2, 128), (6, 2, 64), (4, 4, 128)])
def test_busy_batches(heads, kv, D):
    """Prompts of unequal lengths that fill the device, with and without a prefix, checked row by row in 64 bits: outputs to half a
    step of their type and 2^-10 of the values' size, lse to 2^-17 (D 2^-24 of a score's parts, which are below 100 here)."""
    p = problem(18, [0, 2500, 333, 0, 4000, 64], [1800, 700, 1, 515, 96, 1200], heads, kv, D, 32, torch.float16)
    r = attend(p)
    for b in range(p.B):
        n = int(p.cu[b + 1] - p.cu[b])
        rows = sorted({0, n // 2, n - 1} | set(range(0, n, 37)))
        out, lse = _exact(p, b, rows)
        at = int(p.cu[b]) + torch.tensor(rows, device="cuda")
        assert ((r.out[at].double() - out).abs() <= 2.0 ** -11 * out.abs() + 2.0 ** -9).all()
        assert ((r.lse[at].double() - lse).abs() <= 100 * D * 2.0 ** -24).all()
        off = (r.out[at].double() - out).norm() / out.norm()
        assert off < 2.0 ** -11                      # (a half step is an upper bound of the mean error, which is smaller by sqrt 3 at least)


@pytest.mark.parametrize("count", [2, 200])
def test_a_sequence_is_right_in_any_batch(count):
    """The division of the work depends on the batch; the result only by the joining's roundings: both are checked, and a repeated call
    gives the same bits."""
    whole = problem(19, [900, 30, 2000], [count, 1, count], 4, 1, 128, 16, torch.bfloat16)
    r = attend(whole)
    check_attention(whole, r)
    again = attend(whole)
    assert torch.equal(r.out, again.out) and torch.equal(r.lse, again.lse)


@pytest.mark.parametrize("count", [3, 100])
def test_capture_replay_and_streams(count):
    """A captured call follows the lengths, tables and rows that it finds; two graphs with an object each, replayed at once."""
    p = problem(20, [70, 300, 0], [count, 1, count], 4, 2, 128, 16, torch.bfloat16)
    want = attend(p)
    calls, graphs, streams = [attention(p), attention(p)], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    start = torch.zeros_like(p.start)
    for a, s in zip(calls, streams):
        a.mcsd_chunk_attention(p.q, p.cache, p.table, start, p.cu)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            a.mcsd_chunk_attention(p.q, p.cache, p.table, start, p.cu)
        graphs.append(graph)
    start.copy_(p.start)
    torch.cuda.synchronize()
    for _ in range(3):
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    for a in calls:
        assert torch.equal(a.out, want.out) and torch.equal(a.lse, want.lse)


@pytest.mark.parametrize("count", [2, 64])
def test_a_cache_beyond_four_gigabytes(count):
    D, ps, kv = 128, 128, 8
    block = binding.mcsd_kv_block_bytes(D, ps)
    n_pages = 5 * 2**30 // (block * kv)
    pages = torch.zeros((n_pages, kv, block), dtype=torch.uint8, device="cuda")
    small = problem(21, [500], [count], 8, kv, D, ps, torch.bfloat16)
    want = attend(small)
    need = small.table.shape[1]
    for j in range(need):
        pages[n_pages - 1 - j] = small.cache.pages[int(small.table[0, j])]
    big = binding.KvCache(pages, D, ps)
    table = (n_pages - 1 - torch.arange(need, device="cuda", dtype=torch.int32)).view(1, -1)
    a = binding.ChunkAttention(1, count, 8, small.q.dtype, big, need)
    r = a.mcsd_chunk_attention(small.q, big, table, small.start, small.cu)
    assert torch.equal(r.out, want.out) and torch.equal(r.lse, want.lse)


def test_python_refusals():
    p = problem(22, [4], [3], 4, 2, 64, 16, torch.bfloat16)
    a = attention(p)
    for bad in (dict(q=p.q.half()), dict(q=p.q[:, :2]), dict(q=torch.cat([p.q, p.q])), dict(page_table=p.table.long()), dict(start=p.start.long()),
                dict(cu_tokens=p.cu[:-1]), dict(out=p.q[:1])):
        args = dict(q=p.q, cache=p.cache, page_table=p.table, start=p.start, cu_tokens=p.cu)
        args.update(bad)
        with pytest.raises(AssertionError):
            a.mcsd_chunk_attention(**args)
    with pytest.raises(binding.McsdError):
        binding.ChunkAttention(1, 3, 3, torch.bfloat16, p.cache, 4)
