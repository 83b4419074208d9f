"""mcsd_tree_attention against a plain statement in 64 bits, at the sizes and masks where it can go wrong."""
import numpy as np
import pytest
import torch

import ops_reference as ref
from paper_2401_06706_b200 import binding, synth

pytestmark = pytest.mark.gpu
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _tree(kconfig):
    return synth.tree_from_kconfig(synth.parse_kconfig(kconfig)) if isinstance(kconfig, str) else np.asarray(kconfig, dtype=np.int32)


def _pages(g, n_pages, heads, D, ps, loud=1.0):
    """Cache pages of quantised normal rows with an offset per channel."""
    T = n_pages * ps
    cache = binding.KvCache.empty(n_pages, heads, D, ps)
    k = torch.randn((T, heads, D), generator=g) * loud + 0.5 * torch.randn((1, heads, D), generator=g)
    v = torch.randn((T, heads, D), generator=g)
    binding.mcsd_append_kv(cache, k.cuda(), v.cuda(), torch.arange(T, device="cuda"))
    return cache


def _problem(seed, B, kconfig, heads, kv, D, ps, prefixes, dtype, *, spare=2, loud=1.0):
    g = torch.Generator().manual_seed(seed)
    parent = _tree(kconfig)
    N = len(parent)
    prefix = torch.tensor(prefixes, dtype=torch.int32)
    need = [max(-(-(p + N) // ps), 0) if p >= 0 else 0 for p in prefixes]
    W = max(max(need), 1)
    n_pages = sum(need) + spare
    ids = torch.randperm(n_pages, generator=g).to(torch.int32)
    table = torch.full((B, W), -1, dtype=torch.int32)
    at = 0
    for b in range(B):
        table[b, :need[b]] = ids[at:at + need[b]]
        at += need[b]
    cache = _pages(g, n_pages, kv, D, ps, loud)
    q = (1.2 * torch.randn((B, N, heads, D), generator=g)).to(dtype).cuda()
    return parent, q, cache, table.cuda(), prefix.cuda()


def _check(q, cache, table, prefix, parent, out, lse, scale=None, seen_nan=False):
    f = lambda t: t.float().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()
    scale = q.shape[-1] ** -0.5 if scale is None else scale
    want, want_lse, tol, tol_lse = ref.attention(f(q), cache.pages.cpu().numpy(), f(table), f(prefix), parent, cache.head_dim,
                                                 cache.page_size, scale, torch.finfo(q.dtype).eps)
    got, got_lse = f(out).astype(np.float64), f(lse).astype(np.float64)
    used = f(prefix) >= 0
    for g, w, t, name in ((got, want, tol, "out"), (got_lse, want_lse, tol_lse, "lse")):
        g, w, t = g[used], w[used], t[used]
        with np.errstate(invalid="ignore"):
            ok = (np.abs(g - w) <= t) | (g == w) | (np.isnan(g) & np.isnan(w))
        assert ok.all(), (name, np.argwhere(~ok)[:4], g[~ok][:4], w[~ok][:4], t[~ok][:4])


def _run(q, cache, table, prefix, parent, scale=None):
    att = binding.TreeAttention(q.shape[0], parent, q.shape[2], q.dtype, cache, table.shape[1])
    r = att.mcsd_tree_attention(q, cache, table, prefix, scale=scale)
    torch.cuda.synchronize()
    return r


SHAPES = [  # kconfig, query heads, key heads
    ("", 1, 1), ("", 4, 1), ("", 7, 1), ("", 16, 2), ("2", 2, 2), ("2", 24, 2), ("4x2x2x1", 2, 2), ("4x2x2x1", 6, 2), ("1x1x1x1x1x1x1", 8, 2),
    ("4x4x2x2x1", 1, 1), ("4x4x2x2x1", 4, 1), ("32", 1, 1), ("8x8x6", 1, 1)]


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("D,ps", [(128, 16), (64, 16), (128, 64), (64, 128)])
@pytest.mark.parametrize("kconfig,heads,kv", SHAPES)
def test_against_reference(dtype, D, ps, kconfig, heads, kv):
    prefixes = [0, 1, 37, 130]
    parent, q, cache, table, prefix = _problem(len(kconfig) + heads, 4, kconfig, heads, kv, D, ps, prefixes, DTYPES[dtype])
    r = _run(q, cache, table, prefix, parent)
    _check(q, cache, table, prefix, parent, r.out, r.lse)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kconfig,heads,kv", [("", 2, 1), ("", 8, 1), ("2", 8, 2), ("4x2x2x1", 2, 1), ("4x2x2x1", 4, 1)])
def test_long_and_ragged(dtype, D, kconfig, heads, kv):
    """Lengths on both sides of every tile and split border, some long, in one batch."""
    prefixes = [3000, 0, 127, 128, 129, 255, 256, 15, 16, 17, 31, 1000, 2047]
    parent, q, cache, table, prefix = _problem(7, len(prefixes), kconfig, heads, kv, D, 16, prefixes, DTYPES[dtype])
    r = _run(q, cache, table, prefix, parent)
    _check(q, cache, table, prefix, parent, r.out, r.lse)


@pytest.mark.parametrize("kconfig,heads", [("", 4), ("4x2x2x1", 3)])
@pytest.mark.parametrize("loud", [12.0, 60.0])
def test_loud_keys(kconfig, heads, loud):
    """Scores far apart: the running maximum moves often and by much; a weight of one next to zeros."""
    parent, q, cache, table, prefix = _problem(8, 2, kconfig, heads, 1, 128, 16, [700, 301], torch.float16, loud=loud)
    r = _run(q, cache, table, prefix, parent)
    _check(q, cache, table, prefix, parent, r.out, r.lse)


@pytest.mark.parametrize("kconfig,heads", [("", 4), ("4x2x2x1", 3)])
def test_rising_and_falling_scores(kconfig, heads):
    """Keys whose scores rise (or fall) steadily with the position, by thousands over the prefix."""
    parent, q, cache, table, prefix = _problem(9, 2, kconfig, heads, 1, 64, 16, [600, 600], torch.bfloat16)
    ramp = torch.linspace(0.1, 40.0, 600).view(600, 1, 1)
    base = torch.randn((1, 1, 64), generator=torch.Generator().manual_seed(1))
    for b, r in enumerate((ramp, ramp.flip(0))):
        pos = torch.arange(600, device="cuda")
        slots = table[b, pos // 16].long() * 16 + pos % 16
        binding.mcsd_append_kv(cache, (r * base).cuda(), torch.randn((600, 1, 64), device="cuda"), slots)
    q[:] = (base * 2).to(q.dtype).cuda()
    r = _run(q, cache, table, prefix, parent)
    _check(q, cache, table, prefix, parent, r.out, r.lse)


@pytest.mark.parametrize("small", [1e-3, 1e-6, 3e4])
@pytest.mark.parametrize("kconfig,heads", [("", 4), ("4x2x2x1", 3)])
def test_small_and_large_values(small, kconfig, heads):
    """Values far from one: weights are relative to the value scales; tokens of very different size side by side."""
    parent, q, cache, table, prefix = _problem(10, 1, kconfig, heads, 1, 128, 16, [500], torch.bfloat16 if small > 1 else torch.float16)
    g = torch.Generator().manual_seed(2)
    v = torch.randn((500, 1, 128), generator=g) * small / 4
    v[100:110] *= 0.01
    pos = torch.arange(500, device="cuda")
    binding.mcsd_append_kv(cache, torch.randn((500, 1, 128), generator=g).cuda(), v.cuda(), table[0, pos // 16].long() * 16 + pos % 16)
    r = _run(q, cache, table, prefix, parent)
    _check(q, cache, table, prefix, parent, r.out, r.lse)


@pytest.mark.parametrize("scale", [0.0, -0.3, 1.7, 1e-4])
@pytest.mark.parametrize("kconfig,heads", [("2", 2), ("4x2x2x1", 3)])
def test_other_scales(scale, kconfig, heads):
    parent, q, cache, table, prefix = _problem(11, 2, kconfig, heads, 1, 64, 32, [200, 13], torch.bfloat16)
    r = _run(q, cache, table, prefix, parent, scale)
    _check(q, cache, table, prefix, parent, r.out, r.lse, scale)


@pytest.mark.parametrize("factor", [1e-6, 1e4])
@pytest.mark.parametrize("kconfig,heads", [("2", 2), ("4x2x2x1", 3)])
def test_small_and_large_queries(factor, kconfig, heads):
    """bf16 queries outside the range of half precision, rows of zeros among them."""
    parent, q, cache, table, prefix = _problem(12, 2, kconfig, heads, 1, 128, 16, [200, 13], torch.bfloat16)
    q *= factor
    q[:, 0, 0] = 0
    q[0, -1, -1, :64] = 0
    r = _run(q, cache, table, prefix, parent, 0.09 / factor)
    _check(q, cache, table, prefix, parent, r.out, r.lse, float(np.float32(0.09 / factor)))


@pytest.mark.parametrize("kconfig,heads,kv", [("", 4, 2), ("4x2x2x1", 4, 2), ("4x4x2x2x1", 4, 1)])
def test_hidden_positions_do_not_leak(kconfig, heads, kv):
    """NaN rows where a node must not look (other branches, behind the tree, other pages): only the rows that
    see one are NaN."""
    parent, q, cache, table, prefix = _problem(13, 3, kconfig, heads, kv, 128, 16, [40, 0, 131], torch.bfloat16)
    N = len(parent)
    W = table.shape[1]
    used = set()
    for b in range(3):
        used |= {int(table[b, t // 16]) * 16 + t % 16 for t in range(int(prefix[b]) + N)}
    free = torch.tensor(sorted(set(range(cache.n_pages * 16)) - used), device="cuda")
    bad = torch.full((free.numel(), kv, 128), float("nan"), device="cuda")
    binding.mcsd_append_kv(cache, bad, bad, free)
    r = _run(q, cache, table, prefix, parent)
    assert torch.isfinite(r.out).all() and torch.isfinite(r.lse).all()
    _check(q, cache, table, prefix, parent, r.out, r.lse)
    # a NaN row at one node: exactly its descendants' rows are NaN
    if N > 1:
        node = 2
        slot = torch.tensor([int(table[b, (int(prefix[b]) + node) // 16]) * 16 + (int(prefix[b]) + node) % 16 for b in range(3)], device="cuda")
        binding.mcsd_append_kv(cache, bad[:3], bad[:3], slot)
        r = _run(q, cache, table, prefix, parent)
        below = torch.tensor([node in ref.path(parent, n) for n in range(N)], device="cuda")
        assert torch.isnan(r.out[:, below]).all() and torch.isfinite(r.out[:, ~below]).all()
        _check(q, cache, table, prefix, parent, r.out, r.lse)


@pytest.mark.parametrize("kconfig,heads", [("", 2), ("2", 3), ("4x2x2x1", 3), ("4x4x2x2x1", 1)])
def test_unused_entries_missing_pages_and_empty_rows(kconfig, heads):
    parent, q, cache, table, prefix = _problem(14, 5, kconfig, heads, 1, 64, 16, [100, -1, 60, 20, 300], torch.float16)
    table[0, 2] = -1                                 # a hole in the prefix
    table[2, :] = cache.n_pages + 3                  # no page at all: rows of 0 with lse -inf
    prefix[3] = 100000                               # longer than the table: what is there counts
    table[4, int(prefix[4]) // 16:] = -1             # the tree's own positions are missing
    att = binding.TreeAttention(5, parent, heads, q.dtype, cache, table.shape[1])
    att.out.fill_(3.0)
    att.lse.fill_(4.0)
    r = att.mcsd_tree_attention(q, cache, table, prefix)
    torch.cuda.synchronize()
    assert (r.out[1] == 3).all() and (r.lse[1] == 4).all()
    assert (r.out[2] == 0).all() and torch.isneginf(r.lse[2]).all()
    want_table = table.clone()
    _check(q, cache, want_table, torch.where(prefix > 10000, table.shape[1] * 16, prefix), parent, r.out, r.lse)


def test_strided_queries_outputs_and_tables():
    """q as a slice of a fused projection at an odd offset, out inside a larger tensor, a table with padding."""
    for pad in (0, 8, 3):
        parent, q, cache, table, prefix = _problem(15, 3, "3x2", 6, 2, 64, 16, [33, 64, 5], torch.bfloat16)
        B, N, H, D = q.shape
        fused = torch.randn((B, N, H * D + 2 * 2 * D + pad), device="cuda").to(torch.bfloat16)
        fused[:, :, pad:pad + H * D] = q.flatten(2)
        qs = fused[:, :, pad:pad + H * D].unflatten(2, (H, D))
        wide = torch.full((B, table.shape[1] + 3), 10**6, dtype=torch.int32, device="cuda")
        wide[:, :table.shape[1]] = table
        big = torch.full((B, N, H, D + pad), 2.0, device="cuda").to(torch.bfloat16)
        att = binding.TreeAttention(B, parent, H, q.dtype, cache, table.shape[1])
        r = att.mcsd_tree_attention(qs, cache, wide[:, :table.shape[1]], prefix, out=big[..., :D])
        torch.cuda.synchronize()
        _check(q, cache, table, prefix, parent, r.out, r.lse)
        assert (big[..., D:] == 2).all()


@pytest.mark.parametrize("parents", ["7x8x8", list(range(-1, 511))], ids=["wide", "chain"])
def test_the_largest_trees(parents):
    """512 nodes: three levels, and a chain (every mask word is used, tree positions fill several units)."""
    parent, q, cache, table, prefix = _problem(23, 3, parents, 1, 1, 64, 16, [0, 100, 259], torch.float16)
    assert len(parent) == 512
    r = _run(q, cache, table, prefix, parent)
    _check(q, cache, table, prefix, parent, r.out, r.lse)


@pytest.mark.parametrize("kconfig,heads", [("", 2), ("4x2x2x1", 8)])
def test_output_in_place_of_the_queries(kconfig, heads):
    """out may be q: a row of queries is read before its result is written, in whole and in divided items."""
    parent, q, cache, table, prefix = _problem(19, 5, kconfig, heads, 2, 128, 16, [1000, 31, 2500, 130, 7], torch.bfloat16)
    want = _run(q, cache, table, prefix, parent)
    att = binding.TreeAttention(5, parent, heads, q.dtype, cache, table.shape[1])
    got = att.mcsd_tree_attention(q, cache, table, prefix, out=q)
    torch.cuda.synchronize()
    assert got.out is q and torch.equal(q, want.out) and torch.equal(got.lse, want.lse)


def test_capture_replay_streams_and_a_shared_workspace():
    """A captured call replayed with new lengths, tables and queries; the same object used eagerly in between (its
    workspace is rewritten by every call); a second object on another stream at the same time."""
    parent, q, cache, table, prefix = _problem(16, 6, "4x2x2x1", 4, 2, 128, 16, [900, 700, 50, 1200, 3, 400], torch.bfloat16)
    att = binding.TreeAttention(6, parent, 4, q.dtype, cache, table.shape[1])
    other = binding.TreeAttention(6, parent, 4, q.dtype, cache, table.shape[1])
    att.mcsd_tree_attention(q, cache, table, prefix)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        att.mcsd_tree_attention(q, cache, table, prefix)
    before = prefix.clone()
    for step in range(4):
        prefix.copy_(torch.clamp(before - 37 * step, min=0))
        q.mul_(-1)
        att.out.fill_(float("nan"))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            r2 = other.mcsd_tree_attention(q, cache, table, prefix)
        graph.replay()
        torch.cuda.synchronize()
        _check(q, cache, table, prefix, parent, att.out, att.lse)
        assert torch.equal(att.out, r2.out) and torch.equal(att.lse, r2.lse)


def test_results_do_not_depend_on_what_else_is_in_the_batch_order():
    """Twice the same call gives the same bits."""
    parent, q, cache, table, prefix = _problem(17, 9, "2x2x2x2", 8, 2, 128, 16, [1500, 2, 90, 800, 1, 300, 77, 2000, 16], torch.bfloat16)
    a, b = _run(q, cache, table, prefix, parent), _run(q, cache, table, prefix, parent)
    assert torch.equal(a.out, b.out) and torch.equal(a.lse, b.lse)


def test_a_cache_beyond_four_gigabytes():
    D, ps, H = 128, 16, 8
    n_pages = (5 << 30) // (H * binding.mcsd_kv_block_bytes(D, ps))
    big = binding.KvCache.empty(n_pages, H, D, ps)
    for kconfig in ("", "4x2x2x1"):
        parent, q, cache, table, prefix = _problem(18, 2, kconfig, 8, H, D, ps, [300, 170], torch.bfloat16)
        far = torch.randperm(n_pages, generator=torch.Generator().manual_seed(1))[:cache.n_pages].cuda()
        far[0], far[-1] = n_pages - 1, n_pages - 2
        big.pages[far] = cache.pages
        r = _run(q, cache, table, prefix, parent)
        moved = torch.where(table >= 0, far[table.long().clamp(min=0)].to(torch.int32), table)
        s = _run(q, big, moved, prefix, parent)
        assert torch.equal(r.out, s.out) and torch.equal(r.lse, s.lse)


def test_many_sequences_and_an_empty_batch():
    """More sequences than one pass of a warp over the lengths holds."""
    B = 1100
    rng = np.random.default_rng(3)
    parent, q, cache, table, prefix = _problem(19, B, "2", 2, 1, 64, 16, [int(x) for x in rng.integers(-1, 60, B)], torch.float16)
    r = _run(q, cache, table, prefix, parent)
    _check(q, cache, table, prefix, parent, r.out, r.lse)
    e = _run(q[:0], cache, table[:0], prefix[:0], parent)
    assert e.out.shape[0] == 0


@pytest.mark.parametrize("kconfig,heads,kv", [("", 32, 8), ("2", 32, 8), ("4x2x2x1", 32, 32), ("4x2x2x1", 64, 32), ("2x2x2x2", 64, 8), ("4x4x2x2x1", 16, 8)])
@pytest.mark.parametrize("D", [64, 128])
def test_busy_batches(kconfig, heads, kv, D):
    """Enough items that every SM works through several, of unequal lengths, with idle rows in the last block: against
    products in 64 bits on the device, several times over."""
    prefixes = [1400, 1, 700, 300, 129, 1023, 64, 900]
    parent, q, cache, table, prefix = _problem(20, 8, kconfig, heads, kv, D, 16, prefixes, torch.bfloat16)
    N, G = len(parent), heads // kv
    att = binding.TreeAttention(8, parent, heads, q.dtype, cache, table.shape[1])
    runs = []
    for _ in range(4):
        r = att.mcsd_tree_attention(q, cache, table, prefix)
        runs.append((r.out.clone(), r.lse.clone()))
    torch.cuda.synchronize()
    assert all(torch.equal(a, runs[0][0]) and torch.equal(b, runs[0][1]) for a, b in runs)
    seen = torch.tensor([[m in ref.path(parent, n) for m in range(N)] for n in range(N)], device="cuda")
    for b, length in enumerate(prefixes):
        pos = torch.arange(length + N, device="cuda")
        slots = table[b, pos // 16].long() * 16 + pos % 16
        k, v = (t.double().transpose(0, 1) for t in binding.mcsd_read_kv(cache, slots))            # [kv, keys, D]
        x = q[b].double().view(N, kv, G, D).permute(1, 0, 2, 3).reshape(kv, N * G, D)
        s = torch.matmul(x, k.transpose(1, 2)) * D ** -0.5
        mask = torch.cat([torch.ones((N, length), dtype=torch.bool, device="cuda"), seen], 1).repeat_interleave(G, 0)
        s = s.masked_fill(~mask, float("-inf"))
        lse = torch.logsumexp(s, -1)
        p = torch.exp(s - lse[..., None])
        want = torch.matmul(p, v)
        # weights rounded to half (2^-12) and scores that are sums of D products in float32, of numbers up to |q| (|mid| + 15 scale)
        ds = D * 2.0 ** -24 * (D ** -0.5 * x.abs().sum(-1) * 3 * k.abs().amax()) + 2.0 ** -19
        tol = 2.0 ** -8 * want.abs() + torch.matmul(p, v.abs() + v.abs().amax(-1, keepdim=True)) * (2.0 ** -12 + 2 * ds)[..., None]
        back = lambda t: t.view(kv, N, G, -1).permute(1, 0, 2, 3).reshape(N, heads, -1)
        assert ((runs[0][0][b].double() - back(want)).abs() <= back(tol)).all()
        assert ((runs[0][1][b].double() - back(lse)[..., 0]).abs() <= back(ds + 2.0 ** -21 * lse.abs())[..., 0]).all()


# ---------------------------------------------------------------- value scales far apart
def _exact_rows(q, cache, table, prefix, parent, b, scale):
    """(out, lse, tolerance of out, of lse) of one sequence in 64 bits on the device, [N, heads, ..].

    Counted: the final rounding (half a step); a weight p vscale rounded to half (2^-11 of it, times the distance of its code
    from the middle) or, where it is a subnormal half, 2^-25 of the reference, which lies at most two octaves above the largest
    weight of the row (the scales of the keys but the loud ones lie within a factor of four: asserted), times a code of 8; the
    float32 scores (D 2^-24 of their parts, and 2^-19 for the exponential), which count twice in a quotient, and sums of n terms
    (n 2^-24)."""
    D, ps, N, heads, kv = cache.head_dim, cache.page_size, q.shape[1], q.shape[2], cache.n_heads
    n = int(prefix[b]) + N
    pos = torch.arange(n, device="cuda")
    page, row, half = table[b, pos // ps].long(), pos % ps, ps * D // 2
    par = cache.pages[:, :, 2 * half:].contiguous().view(torch.float16).view(-1, kv, 2, ps, 2)[page, :, :, row].double()   # [n, kv, which, (scale, mid)]
    k, v = (t.double().transpose(0, 1) for t in binding.mcsd_read_kv(cache, page * ps + row))           # [kv, n, D]
    ks, km, vs, vm = (par[:, :, w, c].T for w in (0, 1) for c in (0, 1))                                # [kv, n]
    quiet = vs[vs < 10]
    assert quiet.max() <= 4 * quiet.min()
    seen = torch.ones((N, n), dtype=torch.bool, device="cuda")
    seen[:, int(prefix[b]):] = torch.tensor([[m in ref.path(parent, i) for m in range(N)] for i in range(N)], device="cuda")
    g = torch.arange(heads, device="cuda") // (heads // kv)
    s = torch.einsum("nhd,hkd->nhk", q[b].double(), k[g]) * scale
    s = s.masked_fill(~seen[:, None], float("-inf"))
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - lse[..., None])
    out = torch.einsum("nhk,hkd->nhd", p, v[g])
    # (the parts of a score: of the keys that the row sees)
    part = torch.where(seen[:, None], (km.abs() + 15 * ks)[g][None], 0.0).amax(-1) * q[b].double().abs().sum(-1) * abs(scale)
    ds = D * 2.0 ** -24 * part + 2.0 ** -19
    tol = (torch.finfo(q.dtype).eps / 2 * out.abs() + 2.0 ** -11 * torch.einsum("nhk,hkd->nhd", p, (v - vm[..., None]).abs()[g])
           + (8 * n * 2.0 ** -23 * (p * vs[g][None]).amax(-1) + (p * (vm.abs() + 8 * vs)[g][None]).sum(-1) * (2 * ds + n * 2.0 ** -24))[..., None])
    return out, lse, tol, ds + 2.0 ** -21 * lse.abs() + n * 2.0 ** -24


BLOCKS = [("2", 2, 1), ("2", 5, 1), ("2", 8, 1), ("4x2x2x1", 1, 1), ("4x2x2x1", 8, 2), ("4x4x2x2x1", 1, 1)]     # blocks of 8, 16, 24, 24, 128, 128 rows


def _even_weights(seed, kconfig, heads, kv, D, prefixes):
    """A problem in which an error of the small weights adds up: every position has the same value row, one position in 32 a score
    some 5.5 above all others, which have the same key row. (The queries lean the way of the keys.)"""
    parent, q, cache, table, prefix = _problem(seed, len(prefixes), kconfig, heads, kv, D, 16, prefixes, torch.float16)
    g = torch.Generator().manual_seed(seed)
    way = torch.randn((D,), generator=g)
    way *= D ** 0.5 / way.norm()
    q.copy_((way + 0.1 * torch.randn(q.shape, generator=g)).to(q))
    value = torch.randn((1, kv, D), generator=g)
    for b, n in enumerate(prefixes):
        pos = torch.arange(n + len(parent))
        keys = torch.where(pos[:, None, None] % 32 == 7, 5.5 * D ** -0.5 * way, 0.0 * way).expand(-1, kv, D)
        binding.mcsd_append_kv(cache, keys.contiguous().cuda(), value.expand(len(pos), kv, D).contiguous().cuda(), _slots(table, b, pos))
    return parent, q, cache, table, prefix, way


def _slots(table, b, pos):
    return table[b, pos.cuda() // 16].long() * 16 + pos.cuda() % 16


@pytest.mark.parametrize("loud", [8e3, 5e4])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kconfig,heads,kv", BLOCKS)
def test_a_loud_value_on_another_branch_takes_no_bits(kconfig, heads, kv, D, loud):
    """One node's value row is thousands of times larger than all others: the rows that do not see it are as exact as without it."""
    parent, q, cache, table, prefix, _ = _even_weights(31, kconfig, heads, kv, D, [200, 20, 333])
    node = 2
    row = torch.rand((1, kv, D), generator=torch.Generator().manual_seed(5)).cuda() * loud
    for b in range(3):
        binding.mcsd_append_kv(cache, torch.zeros((1, kv, D), device="cuda"), row, _slots(table, b, prefix[b:b + 1] + node))
    r = _run(q, cache, table, prefix, parent)
    blind = torch.tensor([node not in ref.path(parent, n) for n in range(len(parent))], device="cuda")
    for b in range(3):
        out, lse, tol, tol_lse = _exact_rows(q, cache, table, prefix, parent, b, D ** -0.5)
        assert ((r.out[b].double() - out).abs() <= tol)[blind].all(), ((r.out[b].double() - out).abs() / tol)[blind].max()
        assert ((r.lse[b].double() - lse).abs() <= tol_lse).all()


@pytest.mark.parametrize("loud", [8e3, 5e4])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kconfig,heads,kv", [("", 4, 1)] + BLOCKS)
def test_a_loud_value_of_small_weight_takes_no_bits(kconfig, heads, kv, D, loud):
    """Some rows of the prefix have values thousands of times larger than the others' and scores so low that they do not
    count: the output is as exact as without them."""
    parent, q, cache, table, prefix, way = _even_weights(32, kconfig, heads, kv, D, [900, 130])
    g = torch.Generator().manual_seed(6)
    for b, at in ((0, [3, 64, 500, 501, 899]), (1, [0, 129])):
        keys = (-40 * D ** -0.5 * way).expand(len(at), kv, D).contiguous()
        binding.mcsd_append_kv(cache, keys.cuda(), loud * torch.rand((len(at), kv, D), generator=g).cuda(), _slots(table, b, torch.tensor(at)))
    r = _run(q, cache, table, prefix, parent)
    for b in range(2):
        out, lse, tol, tol_lse = _exact_rows(q, cache, table, prefix, parent, b, D ** -0.5)
        assert ((r.out[b].double() - out).abs() <= tol).all(), ((r.out[b].double() - out).abs() / tol).max()
        assert ((r.lse[b].double() - lse).abs() <= tol_lse).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("pad", [0, 8, 3])
@pytest.mark.parametrize("prefixes", [[33, 64, 5], [2300, 900, 1500]])
def test_strided_queries_and_outputs_of_many_rows(D, pad, prefixes):
    """The same for the kernel of many rows: by vectors and by elements, items in one piece and divided ones."""
    parent, q, cache, table, prefix = _problem(33, 3, "4x4x2x2x1", 2, 1, D, 16, prefixes, torch.bfloat16)
    B, N, H, _ = q.shape
    fused = torch.randn((B, N, H * D + 4 * D + pad), device="cuda").to(torch.bfloat16)
    fused[:, :, pad:pad + H * D] = q.flatten(2)
    qs = fused[:, :, pad:pad + H * D].unflatten(2, (H, D))
    big = torch.full((B, N, H, D + pad), 2.0, device="cuda").to(torch.bfloat16)
    want = _run(q, cache, table, prefix, parent)
    att = binding.TreeAttention(B, parent, H, q.dtype, cache, table.shape[1])
    r = att.mcsd_tree_attention(qs, cache, table, prefix, out=big[..., :D])
    torch.cuda.synchronize()
    assert torch.equal(r.out, want.out) and torch.equal(r.lse, want.lse) and (big[..., D:] == 2).all()
    if max(prefixes) < 100:                          # (the statement goes position by position)
        _check(q, cache, table, prefix, parent, r.out, r.lse)
    else:
        for b in range(B):
            out, lse, tol, tol_lse = _exact_rows(q, cache, table, prefix, parent, b, D ** -0.5)
            assert ((r.out[b].double() - out).abs() <= tol).all() and ((r.lse[b].double() - lse).abs() <= tol_lse).all()


@pytest.mark.parametrize("kconfig,heads", [("", 8), ("2x2x2x2", 2), ("4x2x2x1", 6)])
def test_a_sequence_is_right_in_any_batch(kconfig, heads):
    """The cut of the work goes by the whole batch; a sequence's rows are right in every one: reversed, alone, among unused entries."""
    parent, q, cache, table, prefix = _problem(34, 7, kconfig, heads, 2, 128, 16, [1500, 2, 90, 800, 1, 300, 77], torch.bfloat16)
    for pick in (list(range(6, -1, -1)), [3], [0, 0, 5], [2, 4, 1]):
        p = prefix[pick]
        if pick == [2, 4, 1]:
            p[1] = -1
        r = _run(q[pick], cache, table[pick], p, parent)
        _check(q[pick], cache, table[pick], p, parent, r.out, r.lse)
