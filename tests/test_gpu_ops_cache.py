"""mcsd_append_kv, mcsd_read_kv and mcsd_gather_accepted_pages against plain statements (bytes equal)."""
import numpy as np
import pytest
import torch

import ops_reference as ref
from paper_2401_06706_b200 import binding, synth

pytestmark = pytest.mark.gpu
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def _np(t):
    return t.float().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def _same_bytes(got, want, dim, ps):
    """Equal bytes, except that a NaN mid may have any payload."""
    if np.array_equal(got, want):
        return True
    diff = np.argwhere(got != want)
    half = ps * dim // 2
    for at in diff:
        block, off = got[tuple(at[:-1])], int(at[-1])
        if off < 2 * half:
            return False
        word = off - (off - 2 * half) % 4
        pair = [np.ascontiguousarray(x[word:word + 4]).view(np.float16) for x in (block, want[tuple(at[:-1])])]
        if not (np.isnan(pair[0][1]) and np.isnan(pair[1][1]) and pair[0][0] == pair[1][0]):
            return False
    return True


def _rows(g, T, H, D, dtype, kind):
    x = torch.randn((T, H, D), generator=g)
    if kind == "offset":
        x = 0.05 * x + 30 * torch.randn((T, H, 1), generator=g)
    elif kind == "ties":                             # whole multiples of half a step: every border is met
        x = torch.randint(-30, 31, (T, H, D), generator=g) * 0.25
        x[..., 0], x[..., 1] = -7.5, 7.5
    elif kind == "extreme":
        x = x * 10.0 ** torch.randint(-9, 5 if dtype == torch.float16 else 7, (T, H, 1), generator=g)
        x[T // 2] = 0.0                              # a row without a range
        x[0, 0] = 3.25
    elif kind == "odd":
        x[0, 0, 3], x[T // 2, H - 1, 5], x[T - 1, 0, 7] = float("nan"), float("inf"), float("-inf")
    return x.to(dtype)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("D,ps", [(64, 16), (128, 16), (64, 128), (128, 64), (128, 32)])
@pytest.mark.parametrize("T,H,kind", [(1, 1, "plain"), (37, 3, "plain"), (50, 2, "offset"), (64, 2, "ties"), (40, 5, "extreme"), (9, 2, "odd")])
def test_append_and_read(dtype, D, ps, T, H, kind):
    dt = DTYPES[dtype]
    g = torch.Generator().manual_seed(T * 31 + D + ps)
    n_pages = T // ps + 3
    k, v = _rows(g, T, H, D, dt, kind), _rows(g, T, H, D, dt, kind)
    slots = torch.randperm(n_pages * ps, generator=g)[:T]
    if T > 4:
        slots[2], slots[3] = -1, n_pages * ps        # skipped
    before = torch.randint(0, 256, (n_pages, H, binding.mcsd_kv_block_bytes(D, ps)), generator=g, dtype=torch.uint8)
    cache = binding.KvCache(before.cuda(), D, ps)
    binding.mcsd_append_kv(cache, k.cuda(), v.cuda(), slots.cuda())
    want = ref.append(before.numpy(), _np(k), _np(v), slots.numpy(), D, ps)
    got = cache.pages.cpu().numpy()
    assert _same_bytes(got, want, D, ps)
    # read back, in every type, into outputs whose skipped rows stay
    for out_type in DTYPES.values():
        ko, vo = torch.full((T, H, D), 9.0, dtype=out_type).cuda(), torch.full((T, H, D), 9.0, dtype=out_type).cuda()
        binding.mcsd_read_kv(cache, slots.cuda(), keys=ko, values=vo)
        for t in range(T):
            page, row = divmod(int(slots[t]), ps)
            if int(slots[t]) < 0 or page >= n_pages:
                assert (ko[t] == 9).all() and (vo[t] == 9).all()
                continue
            for o, w in zip((ko, vo), ref.row_values(got, page, row, D, ps)):
                with np.errstate(over="ignore"):
                    w = torch.from_numpy(w.astype(np.float32)).to(out_type)
                assert torch.equal(torch.nan_to_num(o[t].cpu().float(), nan=-123.0), torch.nan_to_num(w.float(), nan=-123.0))


def test_a_code_is_at_most_half_a_step_off():
    """The reading of a row is within half a step (and the roundings of scale and mid) of what was written."""
    g = torch.Generator().manual_seed(3)
    x = torch.randn((500, 2, 128), generator=g)
    cache = binding.KvCache.empty(40, 2, 128, 16)
    slots = torch.randperm(40 * 16, generator=g)[:500].cuda()
    binding.mcsd_append_kv(cache, x.cuda(), x.cuda(), slots)
    k, v = binding.mcsd_read_kv(cache, slots)
    assert torch.equal(k, v)
    step = (x.amax(-1) - x.amin(-1)) / 15
    # half a step; scale and mid are off by half of 2^-10 of their size each, which the ends of the range see
    bound = step * 0.5 + (15 * step + x.abs().amax(-1)) * 2.0 ** -10
    assert ((k.cpu() - x).abs().amax(-1) <= bound).all()


def test_strided_inputs_and_outputs():
    """Keys and values as slices of one projection's output, at aligned and odd offsets."""
    g = torch.Generator().manual_seed(4)
    T, H, D, ps = 21, 3, 64, 16
    for pad in (0, 1):
        qkv = torch.randn((T, 2 * H * D + 5 * H * D + pad), generator=g, dtype=torch.float32).to(torch.bfloat16).cuda()
        k = qkv[:, pad:pad + H * D].unflatten(1, (H, D))
        v = qkv[:, 3 * H * D:4 * H * D].unflatten(1, (H, D))
        cache = binding.KvCache.empty(4, H, D, ps)
        slots = torch.randperm(64, generator=g)[:T].cuda()
        binding.mcsd_append_kv(cache, k, v, slots)
        want = ref.append(np.zeros(tuple(cache.pages.shape), np.uint8), _np(k), _np(v), slots.cpu().numpy(), D, ps)
        assert np.array_equal(cache.pages.cpu().numpy(), want)
        out = torch.full_like(qkv, 2.0)
        binding.mcsd_read_kv(cache, slots, keys=out[:, pad:pad + H * D].unflatten(1, (H, D)))
        dense, _ = binding.mcsd_read_kv(cache, slots, torch.bfloat16)
        assert torch.equal(out[:, pad:pad + H * D], dense.flatten(1)) and (out[:, pad + H * D:] == 2).all()


def test_a_cache_beyond_four_gigabytes():
    """Byte offsets pass 32 bits."""
    D, ps, H = 128, 16, 8
    block = binding.mcsd_kv_block_bytes(D, ps)
    n_pages = (5 << 30) // (H * block)
    cache = binding.KvCache.empty(n_pages, H, D, ps)
    g = torch.Generator().manual_seed(5)
    slots = torch.tensor([0, n_pages * ps - 1, (n_pages // 2) * ps + 3, n_pages * ps - 17], device="cuda")
    x = torch.randn((4, H, D), generator=g).cuda()
    binding.mcsd_append_kv(cache, x, -x, slots)
    k, v = binding.mcsd_read_kv(cache, slots)
    small = binding.KvCache.empty(1, H, D, ps)
    binding.mcsd_append_kv(small, x, -x, torch.arange(4, device="cuda"))
    k2, v2 = binding.mcsd_read_kv(small, torch.arange(4, device="cuda"))
    assert torch.equal(k, k2) and torch.equal(v, v2) and (k - x).abs().max() < 0.5


@pytest.mark.parametrize("D,ps,layers,heads", [(64, 16, 1, 1), (128, 16, 3, 2), (128, 128, 2, 5), (64, 32, 2, 8)])
@pytest.mark.parametrize("kconfig", ["2", "4x2x2x1", "1x1x1x1x1x1x1x1x1x1x1x1", "8x8x6"])
def test_accepted_rows_move(D, ps, layers, heads, kconfig):
    parent = synth.tree_from_kconfig(synth.parse_kconfig(kconfig))
    N, B = len(parent), 7
    gamma = len(synth.parse_kconfig(kconfig))
    rng = np.random.default_rng(N + ps)
    prefix = rng.integers(0, 3 * ps, B).astype(np.int32)
    W = (3 * ps + N) // ps + 1
    n_pages = B * W + 2
    table = rng.permutation(n_pages)[:B * W].reshape(B, W).astype(np.int32)
    nodes = np.full((B, gamma + 1), -1, dtype=np.int32)
    accept = rng.integers(0, gamma + 1, B).astype(np.int32)
    accept[0] = gamma
    for b in range(B):
        n = 0
        for i in range(accept[b]):
            n = int(rng.choice([c for c in range(N) if parent[c] == n]))
            nodes[b, i] = n
    table[1, prefix[1] // ps] = -1                   # a position without a page: its rows stay
    table[2, :] = n_pages + 5
    prefix[3] = -1                                   # an unused entry
    accept[4] = gamma + 100                          # clipped (the nodes behind the path are -1)
    pages = rng.integers(0, 256, (layers, n_pages, heads, binding.mcsd_kv_block_bytes(D, ps)), dtype=np.uint8)
    cache = binding.KvCache(torch.from_numpy(pages).cuda() if layers > 1 else torch.from_numpy(pages[0]).cuda(), D, ps)
    c = lambda a: torch.from_numpy(a).cuda()
    binding.mcsd_gather_accepted_pages(cache, c(table), c(prefix), c(nodes), c(accept))
    want = ref.move(pages, table, prefix, nodes, accept, D, ps)
    assert np.array_equal(cache.pages.cpu().numpy().reshape(want.shape), want)


@pytest.mark.parametrize("layers", [27, 40])
def test_accepted_rows_move_in_many_layers(layers):
    """Enough (layer, sequence, head) triples that a thread has a run of layers (4 of 27, so the last run is shorter; 6
    of 40), with paths longer than the moves it takes at once."""
    D, ps, heads, B, gamma = 64, 16, 8, 200, 6
    parent = synth.tree_from_kconfig([2, 2, 1, 1, 1, 1])
    rng = np.random.default_rng(layers)
    prefix = rng.integers(0, ps, B).astype(np.int32)
    W = (ps + len(parent)) // ps + 1
    table = rng.permutation(B * W).reshape(B, W).astype(np.int32)
    nodes = np.full((B, gamma + 1), -1, dtype=np.int32)
    accept = rng.integers(0, gamma + 1, B).astype(np.int32)
    for b in range(B):
        n = 0
        for i in range(accept[b]):
            n = int(rng.choice([c for c in range(len(parent)) if parent[c] == n]))
            nodes[b, i] = n
    pages = rng.integers(0, 256, (layers, B * W, heads, binding.mcsd_kv_block_bytes(D, ps)), dtype=np.uint8)
    cache = binding.KvCache(torch.from_numpy(pages).cuda(), D, ps)
    c = lambda a: torch.from_numpy(a).cuda()
    binding.mcsd_gather_accepted_pages(cache, c(table), c(prefix), c(nodes), c(accept))
    want = ref.move(pages, table, prefix, nodes, accept, D, ps)
    assert np.array_equal(cache.pages.cpu().numpy().reshape(want.shape), want)


def test_one_layer_of_several_and_empty_calls():
    cache = binding.KvCache.empty(4, 2, 64, 16, n_layers=3)
    x = torch.randn((5, 2, 64), device="cuda")
    binding.mcsd_append_kv(cache.layer(1), x, x, torch.arange(5, device="cuda"))
    assert (cache.pages[0] == 0).all() and (cache.pages[2] == 0).all() and (cache.pages[1] != 0).any()
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    binding.mcsd_append_kv(cache.layer(0), x[:0], x[:0], none)
    assert binding.mcsd_last_launch_count() == 0
    binding.mcsd_read_kv(cache.layer(0), none)
    i32 = dict(dtype=torch.int32, device="cuda")
    binding.mcsd_gather_accepted_pages(cache, torch.zeros((1, 2), **i32), torch.zeros(1, **i32), torch.zeros((1, 1), **i32), torch.zeros(1, **i32))
    assert binding.mcsd_last_launch_count() == 0


# ---------------------------------------------------------------- more tokens than one pass of the grid takes
def _mixed(g, T, H, D, dtype):
    """Rows of every kind, neighbouring tokens of different ones, so that the rows a thread works on together differ in all
    that a row can differ in."""
    kinds = ["plain", "offset", "ties", "extreme", "odd", "plain", "offset"]
    x = torch.empty((T, H, D), dtype=dtype)
    for i, kind in enumerate(kinds):
        n = len(range(i, T, len(kinds)))
        x[i::len(kinds)] = _rows(g, n, H, D, dtype, kind)
    return x


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("T,H,D,ps,pad", [(4099, 8, 128, 16, 0), (4099, 8, 64, 32, 0), (1777, 32, 128, 64, 0), (4099, 5, 64, 16, 0), (2311, 8, 128, 16, 1), (2311, 7, 64, 128, 3)])
def test_append_and_read_of_many_tokens(dtype, T, H, D, ps, pad):
    """Every group of threads takes several tokens, several times over, and ends on a part of its last group; strides that
    allow vectors and odd ones."""
    dt = DTYPES[dtype]
    g = torch.Generator().manual_seed(T + H + D)
    k, v = _mixed(g, T, H, D, dt), _mixed(g, T, H, D, dt)
    n_pages = T // ps + 4
    slots = torch.randperm(n_pages * ps, generator=g)[:T]
    slots[5::97] = -1
    slots[6::131] = n_pages * ps + 5                 # (outside the cache as well)
    fused = torch.zeros((T, 2 * H * D + pad), dtype=dt)
    fused[:, pad:pad + H * D], fused[:, pad + H * D:] = k.flatten(1), v.flatten(1)
    fused = fused.cuda()
    before = torch.randint(0, 256, (n_pages, H, binding.mcsd_kv_block_bytes(D, ps)), generator=g, dtype=torch.uint8)
    cache = binding.KvCache(before.cuda(), D, ps)
    binding.mcsd_append_kv(cache, fused[:, pad:pad + H * D].unflatten(1, (H, D)), fused[:, pad + H * D:].unflatten(1, (H, D)), slots.cuda())
    got, want = cache.pages.cpu().numpy(), before.numpy().copy()
    s = slots.numpy()
    here = (s >= 0) & (s < n_pages * ps)
    page, row, half = s[here] // ps, s[here] % ps, ps * D // 2
    params = []
    for which, x in enumerate((k, v)):
        codes, scale, mid = ref.quantise(_np(x)[here])
        param = np.ascontiguousarray(np.stack([scale, mid], -1).astype(np.float16)).view(np.uint8)
        for at, width, rows in ((which * half, D // 2, codes[..., 0::2] | codes[..., 1::2] << 4), (2 * half + which * 4 * ps, 4, param)):
            part = want[:, :, at:at + ps * width].reshape(n_pages, H, ps, width)                 # (a copy)
            part[page, :, row] = rows
            want[:, :, at:at + ps * width] = part.reshape(n_pages, H, -1)
        params.append((codes, scale, mid))
    # a NaN mid may have any payload; everything else is equal byte by byte
    halves = lambda a: np.ascontiguousarray(a[:, :, 2 * half:]).view(np.float16)
    same = (got[:, :, 2 * half:].reshape(n_pages, H, -1, 2) == want[:, :, 2 * half:].reshape(n_pages, H, -1, 2)).all(-1)
    assert np.array_equal(got[:, :, :2 * half], want[:, :, :2 * half])
    assert (same | np.isnan(halves(got)) & np.isnan(halves(want))).all()
    # and back, into rows at the same strides; what is skipped stays
    for out_type in DTYPES.values():
        out = torch.full((T, 2 * H * D + pad), 9.0, dtype=out_type).cuda()
        binding.mcsd_read_kv(cache, slots.cuda(), keys=out[:, pad:pad + H * D].unflatten(1, (H, D)), values=out[:, pad + H * D:].unflatten(1, (H, D)))
        out = out.cpu()
        assert (out[:, :pad] == 9).all() and (out[~torch.from_numpy(here)] == 9).all()
        for (codes, scale, mid), o in zip(params, (out[:, pad:pad + H * D], out[:, pad + H * D:])):
            exact = mid.astype(np.float64)[..., None] + scale.astype(np.float64)[..., None] * (codes - 8.0)
            w = torch.from_numpy(exact.astype(np.float32)).to(out_type).float()
            o = o.unflatten(1, (H, D))[torch.from_numpy(here)].float()
            assert ((o == w) | (torch.isnan(o) & torch.isnan(w))).all()
