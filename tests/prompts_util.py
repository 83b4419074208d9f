"""Problems of the prompt operators: a quantised cache, page tables over pages that lie anywhere, packed queries."""
from types import SimpleNamespace

import numpy as np
import torch

import prompts_reference as ref
from paper_2401_06706_b200 import binding

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def host(t):
    return t.float().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def slots_of(p, b, pos):
    pos = torch.as_tensor(pos, device="cuda")
    return p.table[b, pos // p.ps].long() * p.ps + pos % p.ps


def problem(seed, starts, counts, heads, kv, D, ps, dtype, *, spare=2, loud=1.0, pad_tokens=0):
    """starts < 0: an unused entry (its count must be 0)."""
    g = torch.Generator().manual_seed(seed)
    B = len(starts)
    need = [-(-(s + n) // ps) if s >= 0 else 0 for s, n in zip(starts, counts)]
    n_pages = sum(need) + spare
    ids = torch.randperm(n_pages, generator=g).to(torch.int32)
    table = torch.full((B, max(max(need), 1)), -1, dtype=torch.int32)
    at = 0
    for b in range(B):
        table[b, :need[b]] = ids[at:at + need[b]]
        at += need[b]
    cache = binding.KvCache.empty(n_pages, kv, D, ps)
    T = n_pages * ps
    k = torch.randn((T, kv, D), generator=g) * loud + 0.5 * torch.randn((1, kv, D), generator=g)
    binding.mcsd_append_kv(cache, k.cuda(), torch.randn((T, kv, D), generator=g).cuda(), torch.arange(T, device="cuda"))
    cu = torch.zeros(B + 1, dtype=torch.int32)
    cu[1:] = torch.tensor(counts).cumsum(0)
    q = (1.2 * torch.randn((sum(counts) + pad_tokens, heads, D), generator=g)).to(dtype)
    return SimpleNamespace(B=B, q=q.cuda(), cache=cache, table=table.cuda(), start=torch.tensor(starts, dtype=torch.int32).cuda(), cu=cu.cuda(),
                           heads=heads, kv=kv, D=D, ps=ps, max_new=max(max(counts), 1), scale=D ** -0.5)


def attention(p, max_new=None, **kw):
    return binding.ChunkAttention(p.B, max(p.q.shape[0], 1), p.heads, p.q.dtype, p.cache, p.table.shape[1], max_new=max_new or p.max_new, **kw)


def attend(p, max_new=None, scale=None, **kw):
    a = attention(p, max_new)
    r = a.mcsd_chunk_attention(p.q, p.cache, p.table, p.start, p.cu, scale=scale, **kw)
    torch.cuda.synchronize()
    return r


def within(got, want, tol, name):
    with np.errstate(invalid="ignore"):
        ok = (np.abs(got - want) <= tol) | (got == want) | (np.isnan(got) & np.isnan(want))
    assert ok.all(), (name, int((~ok).sum()), np.argwhere(~ok)[:4], got[~ok][:4], want[~ok][:4], tol[~ok][:4])


def check_attention(p, r, max_new=None, scale=None):
    want, want_lse, tol, tol_lse = ref.chunk_attention(host(p.q), p.cache.pages.cpu().numpy(), host(p.table), host(p.start), host(p.cu),
                                                       max_new or p.max_new, p.D, p.ps, p.scale if scale is None else scale, torch.finfo(p.q.dtype).eps)
    mine = np.zeros(p.q.shape[0], dtype=bool)
    for _, first, n in ref.sequences(host(p.start), host(p.cu), p.q.shape[0], max_new or p.max_new):
        mine[first:first + n] = True
    within(host(r.out).astype(np.float64)[mine], want[mine], tol[mine], "out")
    within(host(r.lse).astype(np.float64)[mine], want_lse[mine], tol_lse[mine], "lse")
    return mine


def plain_lse(p, scale=None):
    """lse of the attention, from the statement, as float32 on the GPU."""
    lse = ref.chunk_attention(host(p.q), p.cache.pages.cpu().numpy(), host(p.table), host(p.start), host(p.cu), p.max_new, p.D, p.ps,
                              p.scale if scale is None else scale, 2.0 ** -10)[1]
    return torch.tensor(np.nan_to_num(lse, nan=3.0, neginf=-np.inf), dtype=torch.float32).cuda()
