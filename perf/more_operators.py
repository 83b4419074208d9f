"""The operators of prompts and long conversations, as calls that can be measured: attention of a chunk of new tokens over
the paged 4-bit cache, the attention weight that cached rows accumulate, eviction by it, and log probabilities of given
tokens with the entropy and the top alternatives.

``run`` computes one pass: with ``own`` false in plain torch operations in 32 bits, with ``own`` true through the
package's entry points.  ``exact`` computes the same from the definitions in 64 bits.

Definitions
  chunk         token i of sequence b is row cu_tokens[b] + i of q and sits at position start[b] + i, its key and value in the
                cache like those before it; it sees positions 0 .. start[b] + i:
                s_j = scale <q, k_j>,  out = sum_j softmax(s)_j v_j,  lse = log sum_j exp(s_j)
  weights       w[p] := (p < start[b] ? decay w[p] : 0) + the sum of exp(s_p - lse) over the last `last` new tokens that see p
                and the query heads of the key head
  evict         of the len[b] rows that a sequence has, every layer and key head keeps `keep`: the first `sink`, the last
                `recent` and those of the others with the largest weights (equal ones: the lower position); they move to
                positions 0 .. keep - 1 in their order, the weights with them; rows behind stay what they were
  logprobs      of a row l: log softmax(l / T) of given tokens, the entropy of softmax(l / T), and the `top` largest tokens
                (equal logits: the lower token) with their log probabilities
"""
import math

import torch

own = False

_TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


# ---------------------------------------------------------------- the cases
def listed():
    return [
        # a short question in a short conversation: what matters is latency
        dict(name="chunk_question", op="chunk", batch=1, count=13, every=1, longest=517, ragged=0, heads=32, kv_heads=32, dim=128, dtype="fp16", page_size=16),
        # a serving step that mixes decoding sequences with three chunks of prompts
        dict(name="chunk_mixed", op="chunk", batch=24, count=253, every=8, longest=2047, ragged=1, heads=32, kv_heads=8, dim=128, dtype="bf16", page_size=16),
        # whole prompts of different lengths, nothing cached before
        dict(name="chunk_prompts", op="chunk", batch=6, count=2041, every=1, longest=0, ragged=0, heads=32, kv_heads=8, dim=128, dtype="bf16", page_size=32),
        # a chunk of a long document
        dict(name="chunk_document", op="chunk", batch=1, count=2048, every=1, longest=30011, ragged=0, heads=32, kv_heads=8, dim=128, dtype="bf16", page_size=64),
        # a decoding step that keeps the weights of its rows up to date
        dict(name="weights_decode", op="weights", batch=32, count=1, every=1, last=0, longest=4001, ragged=1, heads=32, kv_heads=8, dim=128, dtype="bf16", page_size=16),
        # the last tokens of prompts observe the rest
        dict(name="weights_window", op="weights", batch=8, count=515, every=1, last=32, longest=3500, ragged=1, heads=32, kv_heads=8, dim=128, dtype="fp16", page_size=32),
        # every token of a chunk counts
        dict(name="weights_chunk", op="weights", batch=2, count=1500, every=1, last=0, longest=2500, ragged=0, heads=16, kv_heads=16, dim=64, dtype="fp16", page_size=32),
        # one layer of a short conversation that is cut a little
        dict(name="evict_layer", op="evict", batch=2, layers=1, heads=8, dim=128, page_size=16, longest=700, ragged=0, keep=512, sink=4, recent=64),
        # all layers of long prompts, cut to a quarter
        dict(name="evict_prompts", op="evict", batch=8, layers=32, heads=8, dim=128, page_size=32, longest=4001, ragged=1, keep=1024, sink=4, recent=128),
        # the tokens of verified paths of a small batch
        dict(name="logprobs_path", op="logprobs", batch=8, kconfig="4x2x2x1", rows=0, vocab=32000, dtype="bf16", top=5, temperature=1.0),
        # all tokens of a prompt
        dict(name="logprobs_prompt", op="logprobs", batch=0, kconfig="", rows=2047, vocab=32000, dtype="bf16", top=20, temperature=1.0),
        # a large vocabulary in 32 bits
        dict(name="logprobs_large", op="logprobs", batch=0, kconfig="", rows=1021, vocab=50272, dtype="fp32", top=8, temperature=0.7),
    ]


_TREES = ["2", "1x1x1x1", "2x2x2x2", "8x2x1", "4x2x2x1", "3x3x1", "4x4x2x2x1"]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["chunk", "chunk", "weights", "evict", "logprobs"])
    if op in ("chunk", "weights"):
        c = dict(op=op, batch=_spread(rng, 1, 32), count=_spread(rng, 1, 2048), every=rng.choice([1, 1, 3, 8]), longest=_spread(rng, 1, 30000) - 1,
                 ragged=rng.choice([0, 1]), heads=0, kv_heads=rng.choice([1, 2, 4, 8, 16]), dim=rng.choice([64, 128]), dtype=rng.choice(["bf16", "fp16"]),
                 page_size=rng.choice([16, 32, 64, 128]))
        c["heads"] = c["kv_heads"] * rng.choice([1, 1, 3, 4, 8])
        if op == "weights":
            c["last"] = rng.choice([0, 1, 16, rng.randint(2, 200)])
    elif op == "evict":
        longest = _spread(rng, 8, 8000)
        keep = rng.randint(1, longest)
        c = dict(op=op, batch=_spread(rng, 1, 16), layers=_spread(rng, 1, 32), heads=rng.choice([1, 4, 8]), dim=rng.choice([64, 128]), page_size=rng.choice([16, 32, 64, 128]),
                 longest=longest, ragged=rng.choice([0, 1]), keep=keep, sink=rng.choice([0, 4, rng.randint(0, keep)]), recent=rng.randint(0, keep))
    else:
        path = rng.choice([0, 1])
        c = dict(op=op, batch=_spread(rng, 1, 64) if path else 0, kconfig=rng.choice(_TREES) if path else "", rows=0 if path else _spread(rng, 1, 2000),
                 vocab=rng.choice([32000, 50272, _spread(rng, 500, 65536)]), dtype=rng.choice(sorted(_TYPES)), top=rng.choice([0, 1, rng.randint(2, 32)]),
                 temperature=rng.choice([1.0, 0.7, 1.3]))
    # no more than the largest listed case of the operator
    most = {m: max(work(x)[m] for x in listed() if x["op"] == op) for m in ("bytes", "flops")}
    pairs = max(_padded(x) for x in listed() if x["op"] in ("chunk", "weights"))
    while any(work(c)[m] > most[m] for m in most) or op in ("chunk", "weights") and _padded(c) > pairs:
        for key in ("batch", "layers", "count", "rows", "longest"):
            if c.get(key, 1) > 1:
                c[key] = (c[key] + 1) // 2
                break
        else:
            c["heads"], c["kv_heads"] = c.get("kv_heads", 1), c.get("kv_heads", 1)
            break
    if op == "evict":
        c["keep"] = min(c["keep"], c["longest"])
    return c


# ---------------------------------------------------------------- shapes
def _parents(kconfig):
    """Parent of every node, level order, root first."""
    parent, level = [-1], [0]
    for k in (int(t) for t in kconfig.split("x") if t):
        nxt = []
        for p in level:
            for _ in range(k):
                nxt.append(len(parent))
                parent.append(p)
        level = nxt
    return parent


def _lengths(case):
    """Rows of every sequence that are cached before: from `longest` down to a quarter of it where the batch is ragged."""
    B, top = case["batch"], case["longest"]
    return [top - (3 * top * b) // (4 * B) if case["ragged"] else top for b in range(B)]


def _counts(case):
    """New tokens: chunks for every `every`-th sequence (lengths down to a half), one token for the others."""
    B, top, every = case["batch"], case["count"], case["every"]
    return [max(1, top - (top * b) // (2 * B)) if b % every == 0 else 1 for b in range(B)]


def _padded(case):
    """Scores that the plain form holds at once, which pads every chunk and every length to the longest."""
    top = min(case["count"], case.get("last") or case["count"])
    return case["batch"] * case["heads"] * top * (case["longest"] + case["count"])


def _pairs(case):
    """Visible (token, position) pairs of one query head."""
    total = 0
    for start, n in zip(_lengths(case), _counts(case)):
        k = min(n, case.get("last") or n)
        total += k * (start + n) - k * (k - 1) // 2
    return total


def work(case):
    """Bytes and operations that one pass cannot do without."""
    if case["op"] in ("chunk", "weights"):
        start, count = _lengths(case), _counts(case)
        keys = (sum(start) + sum(count)) * case["kv_heads"]
        if case["op"] == "chunk":
            return {"bytes": keys * (case["dim"] + 8) + sum(count) * case["heads"] * (4 * case["dim"] + 4), "flops": 4 * case["dim"] * case["heads"] * _pairs(case)}
        rows = sum(min(n, case["last"] or n) for n in count) * case["heads"]
        return {"bytes": keys * (case["dim"] // 2 + 4) + 4 * (keys + sum(start) * case["kv_heads"]) + rows * (2 * case["dim"] + 4),
                "flops": 2 * case["dim"] * case["heads"] * _pairs(case)}
    if case["op"] == "evict":
        rows = weights = 0
        for n in _lengths(case):
            if n > case["keep"]:
                sink = min(case["sink"], case["keep"])
                rows += case["keep"] - sink
                weights += n
        return {"bytes": case["layers"] * case["heads"] * (rows * 2 * (case["dim"] + 8 + 4) + 4 * weights) + 8 * case["batch"], "flops": 0}
    es = 4 if case["dtype"] == "fp32" else 2
    rows = case["rows"] or case["batch"] * (sum(1 for t in case["kconfig"].split("x") if t) / 2 + 1)
    return {"bytes": rows * (case["vocab"] * es + 12 + 8 * case["top"]), "flops": 0}


# ---------------------------------------------------------------- inputs
def _block(dim, page_size):
    return page_size * (dim + 8)


def _pack(x):
    """(codes [.., D / 2] bytes, (scale, mid) [.., 4] bytes) of float32 rows x: the 4-bit form of a cached row."""
    lo, hi = x.amin(-1).double(), x.amax(-1).double()
    scale = ((hi - lo) / 15).to(torch.float16)
    mid = (lo + 8 * scale.double()).to(torch.float16)
    s, m = scale.float().unsqueeze(-1), mid.float().unsqueeze(-1)
    codes = torch.where(s > 0, torch.round((x - m) / torch.where(s > 0, s, 1.0)) + 8, 8.0).clamp(0, 15).to(torch.uint8)
    return codes[..., 0::2] | (codes[..., 1::2] << 4), torch.stack([scale, mid], -1).view(torch.uint8)


def _cache(gen, n_pages, heads, dim, page_size):
    """Pages filled with quantised rows: normal keys with an offset per channel and a few louder tokens, normal values."""
    pages = torch.empty((n_pages, heads, _block(dim, page_size)), dtype=torch.uint8, device="cuda")
    offset = 0.5 * torch.randn((heads, 1, dim), generator=gen, device="cuda")
    half, at = page_size * dim // 2, max(1, (1 << 26) // (heads * page_size * dim))
    for p in range(0, n_pages, at):
        n = min(at, n_pages - p)
        k = torch.randn((n, heads, page_size, dim), generator=gen, device="cuda") + offset
        k *= torch.exp(0.3 * torch.randn((n, heads, page_size, 1), generator=gen, device="cuda"))
        (kc, kp), (vc, vp) = _pack(k), _pack(torch.randn((n, heads, page_size, dim), generator=gen, device="cuda"))
        pages[p:p + n] = torch.cat([t.reshape(n, heads, -1) for t in (kc, vc, kp, vp)], -1)
    return pages


def _binding():
    from paper_2401_06706_b200 import binding
    return binding


def _randint(gen, low, high, shape, dtype=torch.int32):
    return torch.randint(low, high, shape, generator=gen, device="cuda", dtype=dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"case": case, "op": case["op"]}
    {"chunk": _prepare_chunk, "weights": _prepare_weights, "evict": _prepare_evict, "logprobs": _prepare_logprobs}[case["op"]](case, gen, s)
    return s


def _tables(gen, need, page_size):
    """Page table of a batch that needs `need` positions a sequence, over pages that lie anywhere; and the number of pages."""
    pages = (need + page_size - 1) // page_size
    width, total = int(pages.max()), int(pages.sum())
    table = torch.full((need.shape[0], width), -1, dtype=torch.int32, device="cuda")
    table[torch.arange(width, device="cuda") < pages[:, None]] = torch.randperm(total + 2, generator=gen, device="cuda")[:total].to(torch.int32)
    return table, total + 2


def _prepare_chunk(case, gen, s):
    B, D, ps, H, kv = case["batch"], case["dim"], case["page_size"], case["heads"], case["kv_heads"]
    order = torch.randperm(B, generator=gen, device="cuda")
    s["count"] = torch.tensor(_counts(case), device="cuda")[order]
    s["start"] = torch.tensor(_lengths(case), device="cuda", dtype=torch.int32)[order]
    s["cu_tokens"] = torch.cat([torch.zeros(1, device="cuda", dtype=torch.long), s["count"].cumsum(0)]).to(torch.int32)
    s["tokens"], s["most"] = sum(_counts(case)), max(_counts(case))
    s["table"], n_pages = _tables(gen, s["start"] + s["count"], ps)
    s["pages"] = _cache(gen, n_pages, kv, D, ps)
    s["q"] = (1.2 * torch.randn((s["tokens"], H, D), generator=gen, device="cuda")).to(_TYPES[case["dtype"]])
    s["scale"] = 1 / math.sqrt(D)
    if own:
        b = _binding()
        s["cache"] = b.KvCache(s["pages"], D, ps)
        s["attention"] = b.ChunkAttention(B, s["tokens"], H, s["q"].dtype, s["cache"], s["table"].shape[1], max_new=s["most"])


def _prepare_weights(case, gen, s):
    _prepare_chunk(case, gen, s)
    # what the rows gathered before: few have much
    s["weights"] = torch.exp(2 * torch.randn((s["pages"].shape[0], case["kv_heads"], case["page_size"]), generator=gen, device="cuda"))
    # the sums of the attention that went before: of scores of this spread, up to a small difference that no row depends on
    at = torch.arange(s["tokens"], device="cuda")
    seq = torch.repeat_interleave(torch.arange(case["batch"], device="cuda"), s["count"], output_size=s["tokens"])
    seen = s["start"][seq] + at - s["cu_tokens"][seq] + 1
    spread = (s["q"].float().square().sum(-1) * (1.5 / case["dim"])).clamp(max=8)
    s["lse"] = torch.log(seen.float())[:, None] + 0.5 * spread + 0.1 * torch.randn(spread.shape, generator=gen, device="cuda")


def _prepare_evict(case, gen, s):
    B, D, ps, L, H = case["batch"], case["dim"], case["page_size"], case["layers"], case["heads"]
    s["len"] = torch.tensor(_lengths(case), device="cuda", dtype=torch.int32)[torch.randperm(B, generator=gen, device="cuda")]
    s["table"], n_pages = _tables(gen, s["len"], ps)
    s["pages"] = _randint(gen, 0, 256, (L, n_pages, H, _block(D, ps)), torch.uint8)
    s["weights"] = torch.exp(2 * torch.randn((L, n_pages, H, ps), generator=gen, device="cuda"))
    s["weights"][_randint(gen, 0, 16, s["weights"].shape) == 0] = 0.0        # rows that nobody looked at
    s["len_out"] = torch.zeros_like(s["len"])
    if own:
        s["cache"] = _binding().KvCache(s["pages"], D, ps)


def _prepare_logprobs(case, gen, s):
    V, dtype = case["vocab"], _TYPES[case["dtype"]]
    if case["kconfig"]:
        B, parent = case["batch"], _parents(case["kconfig"])
        N, depth = len(parent), sum(1 for t in case["kconfig"].split("x") if t)
        s["logits"] = (2.5 * torch.randn((B, N, V), generator=gen, device="cuda")).to(dtype)
        # a walk down the tree: a child of the node before it, as far as it got
        first, many = {}, {}
        for n, p in enumerate(parent):
            first.setdefault(p, n)
            many[p] = many.get(p, 0) + 1
        first = torch.tensor([first.get(n, 0) for n in range(N)], device="cuda")
        many = torch.tensor([many.get(n, 1) for n in range(N)], device="cuda")
        accept, node = _randint(gen, 0, depth + 1, (B,)), torch.zeros((B,), dtype=torch.int64, device="cuda")
        s["path"] = torch.full((B, depth + 1), -1, dtype=torch.int32, device="cuda")
        for i in range(depth):
            node = first[node] + (torch.rand((B,), generator=gen, device="cuda") * many[node]).long()
            s["path"][:, i] = torch.where(accept > i, node, -1).to(torch.int32)
        s["tokens"] = _randint(gen, 0, V, (B, depth + 1))
        s["tokens"][torch.arange(depth + 1, device="cuda") > accept[:, None]] = -1
    else:
        s["logits"] = (2.5 * torch.randn((case["rows"], V), generator=gen, device="cuda")).to(dtype)
        s["tokens"] = _randint(gen, 0, V, (case["rows"],))
        # most tokens of a text are likely ones
        s["tokens"] = torch.where(torch.rand(s["tokens"].shape, generator=gen, device="cuda") < 0.7, s["logits"].argmax(-1).to(torch.int32), s["tokens"])
    if own:
        b = _binding()
        s["calls"] = b.TokenLogprobs(s["tokens"].numel(), V, dtype, n_top=case["top"], device=s["logits"].device)


# ---------------------------------------------------------------- one pass
def run(state):
    return {"chunk": _run_chunk, "weights": _run_weights, "evict": _run_evict, "logprobs": _run_logprobs}[state["op"]](state)


def _rows(s, which):
    """Keys (0) or values (1) of every sequence's pages in 32 bits, [B, heads, positions, D]."""
    D, ps = s["case"]["dim"], s["case"]["page_size"]
    blocks, half = s["pages"][s["table"].long().clamp(min=0)], ps * D // 2                  # [B, pages, heads, block]
    codes = blocks[..., which * half:(which + 1) * half].unflatten(-1, (ps, D // 2))
    param = blocks[..., 2 * half + which * 4 * ps:2 * half + (which + 1) * 4 * ps].contiguous().view(torch.float16).unflatten(-1, (ps, 2)).float()
    x = param[..., 1:] + param[..., :1] * (torch.stack([codes & 15, codes >> 4], -1).flatten(-2).float() - 8)
    return x.transpose(1, 2).flatten(2, 3)


def _padded_scores(s, k, first):
    """Scores [B, kv heads, tokens, group, positions] of the tokens from `first` [B] on, -inf where nothing is seen; and which
    padded tokens there are."""
    B, kv, H, D = s["case"]["batch"], s["case"]["kv_heads"], s["case"]["heads"], s["case"]["dim"]
    n = min(s["most"], s["case"].get("last") or s["most"])
    i = first[:, None] + torch.arange(n, device="cuda")                                       # token of its sequence
    there = i < s["count"][:, None]
    row = (s["cu_tokens"][:-1, None] + i).clamp(max=s["tokens"] - 1)
    q = s["q"][row].float().view(B, n, kv, H // kv, D).transpose(1, 2).reshape(B, kv, -1, D)
    score = torch.matmul(q, k.transpose(2, 3)).mul_(s["scale"]).view(B, kv, n, H // kv, -1)
    hidden = (torch.arange(k.shape[2], device="cuda") > (s["start"][:, None] + i)[..., None]) | ~there[..., None]
    return score.masked_fill_(hidden[:, None, :, None], float("-inf")), row, there


def _run_chunk(s):
    if own:
        out = s["attention"].mcsd_chunk_attention(s["q"], s["cache"], s["table"], s["start"], s["cu_tokens"], scale=s["scale"])
        return {"out": out.out, "lse": out.lse}
    score, row, there = _padded_scores(s, _rows(s, 0), torch.zeros_like(s["count"]))
    top = score.amax(-1, keepdim=True).clamp(min=-1e30)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.flatten(2, 3), _rows(s, 1)).view(p.shape[:4] + (-1,)) / total
    back = lambda t: t.transpose(1, 2).flatten(2, 3)[there]                                   # [tokens, heads, ..]
    return {"out": back(out).to(s["q"].dtype), "lse": back(top + torch.log(total))[..., 0]}


def _run_weights(s):
    start, count, last = s["start"], s["count"], s["case"]["last"]
    if own:
        s["attention"].mcsd_accumulate_weights(s["q"], s["lse"], s["cache"], s["table"], start, s["cu_tokens"], s["weights"], scale=s["scale"], decay=0.9, last_tokens=last)
        return s["weights"]
    B, kv, H, ps = s["case"]["batch"], s["case"]["kv_heads"], s["case"]["heads"], s["case"]["page_size"]
    score, row, there = _padded_scores(s, _rows(s, 0), (count - last).clamp(min=0) if last else torch.zeros_like(count))
    lse = s["lse"][row].view(B, -1, kv, H // kv).transpose(1, 2)                               # [B, kv, tokens, group]
    got = score.sub_(lse[..., None]).exp_().sum((2, 3))                                        # [B, kv, positions]
    pos = torch.arange(got.shape[-1], device="cuda")
    b, p = torch.nonzero(pos < (start + count)[:, None], as_tuple=True)
    page, r = s["table"][b, p // ps].long(), p % ps
    s["weights"][page, :, r] = torch.where((p < start[b])[:, None], 0.9 * s["weights"][page, :, r], 0.0) + got[b, :, p]
    return s["weights"]


def _run_evict(s):
    # (weights change between two evictions: each pass has those of the start, or soon nothing would be left to move)
    case, weights = s["case"], s["weights"].clone()
    if own:
        _binding().mcsd_evict_rows(s["cache"], weights, s["table"], s["len"], case["keep"], sink=case["sink"], recent=case["recent"], len_out=s["len_out"])
        return {"pages": s["pages"], "weights": weights, "len": s["len_out"]}
    ps, D, keep = case["page_size"], case["dim"], case["keep"]
    sink = min(case["sink"], keep)
    recent = min(case["recent"], keep - sink)
    length = s["len"][:, None].long()
    pos = torch.arange(s["table"].shape[1] * ps, device="cuda").expand(length.shape[0], -1)
    page, row = s["table"].long().clamp(min=0).gather(1, pos // ps), pos % ps                   # [B, positions]
    w = weights[:, page, :, row].permute(2, 0, 3, 1)                                       # [layers, B, heads, positions]
    safe = (pos < sink) | (pos >= length - recent)
    w = torch.where(safe[None, :, None], float("inf"), w)
    w = torch.where((pos < length)[None, :, None], w, float("-inf"))
    order = torch.sort(w, dim=-1, descending=True, stable=True).indices
    rank = torch.empty_like(order).scatter_(-1, order, torch.arange(w.shape[-1], device="cuda").expand(w.shape))
    kept = (rank < keep) & (pos < length)[None, :, None]
    to = torch.cumsum(kept, -1) - 1
    l, b, h, src = torch.nonzero(kept & (length > keep)[None, :, None], as_tuple=True)
    dst = to[l, b, h, src]
    sp, sr, tp, tr = page[b, src], src % ps, page[b, dst], dst % ps
    half, pages = ps * D // 2, s["pages"]
    parts = [pages[..., x:y].unflatten(-1, (ps, -1)) for x, y in ((0, half), (half, 2 * half), (2 * half, 2 * half + 4 * ps), (2 * half + 4 * ps, 2 * half + 8 * ps))]
    parts.append(weights[..., None])
    new = [part[l, sp, h, sr] for part in parts]                                                # all reads before any write
    [part.index_put_((l, tp, h, tr), x) for part, x in zip(parts, new)]
    return {"pages": pages, "weights": weights, "len": torch.minimum(s["len"], torch.full_like(s["len"], keep))}


def _run_logprobs(s):
    if own:
        if "path" in s:
            r = s["calls"].mcsd_path_logprobs(s["logits"], s["path"], s["tokens"], temperature=s["case"]["temperature"])
        else:
            r = s["calls"].mcsd_token_logprobs(s["logits"], s["tokens"], temperature=s["case"]["temperature"])
        return {"logprobs": r.logprobs, "entropy": r.entropy, "top_ids": r.top_ids, "top_logprobs": r.top_logprobs}
    logits, tokens, V = s["logits"], s["tokens"], s["case"]["vocab"]
    there = None
    if "path" in s:
        node = torch.cat([torch.zeros_like(s["path"][:, :1]), s["path"][:, :-1]], 1).long()     # the row a token was drawn from
        there = (node >= 0) & (tokens >= 0)
        logits = logits[torch.arange(node.shape[0], device="cuda")[:, None], node.clamp(min=0)]
    l = logits.float() / s["case"]["temperature"]
    top = l.amax(-1, keepdim=True)
    e = torch.exp(l - top)
    total = e.sum(-1, keepdim=True)
    lse = top + torch.log(total)
    entropy = torch.log(total[..., 0]) - torch.where(e > 0, e * (l - top), 0.0).sum(-1) / total[..., 0]
    logprobs = l.gather(-1, tokens.long().clamp(min=0)[..., None])[..., 0] - lse[..., 0]
    # order of the logits as whole numbers, equal ones by the lower token
    bits = logits.float().add(0.0).view(torch.int32).long()
    key = torch.where(bits < 0, -(bits & 0x7fffffff), bits) * V + (V - 1 - torch.arange(V, device="cuda"))
    ids = torch.topk(key, s["case"]["top"], dim=-1).indices
    top_logprobs = l.gather(-1, ids) - lse
    ids = ids.to(torch.int32)
    if there is not None:       # (entries behind the end of a path are left as they were)
        logprobs, entropy = (torch.where(there, t, 0.0) for t in (logprobs, entropy))
        ids, top_logprobs = torch.where(there[..., None], ids, 0), torch.where(there[..., None], top_logprobs, 0.0)
    return {"logprobs": logprobs, "entropy": entropy, "top_ids": ids, "top_logprobs": top_logprobs}


# ---------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("chunk", "weights"):
        return _exact_rows(s)
    if case["op"] == "logprobs":
        return _exact_logprobs(s)
    return None         # moved bytes


def _exact_side(s, b, keys, codes_at, param_at):
    """Keys or values of sequence b in 64 bits, [heads, keys, D]."""
    ps, D, kv = s["case"]["page_size"], s["case"]["dim"], s["case"]["kv_heads"]
    block = s["pages"][s["table"][b, :(keys + ps - 1) // ps].long()].permute(1, 0, 2)
    raw = block[..., codes_at:codes_at + ps * D // 2].reshape(kv, -1, D // 2)[:, :keys]
    par = block[..., param_at:param_at + 4 * ps].contiguous().view(torch.float16).double().reshape(kv, -1, 2)[:, :keys]
    x = torch.empty((kv, keys, D), dtype=torch.float64, device="cuda")
    x[..., 0::2], x[..., 1::2] = (raw % 16).double(), (raw // 16).double()
    return par[..., 1:] + par[..., :1] * (x - 8)


def _exact_rows(s):
    case = s["case"]
    ps, D, group = case["page_size"], case["dim"], case["heads"] // case["kv_heads"]
    q, weights = s["q"], s["weights"].double() if case["op"] == "weights" else None
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(q.shape[:2], dtype=torch.float64, device="cuda")
    for b in range(case["batch"]):
        start, n, at = int(s["start"][b]), int(s["count"][b]), int(s["cu_tokens"][b])
        first = max(0, n - case["last"]) if case.get("last") else 0
        k = _exact_side(s, b, start + n, 0, ps * D)
        v = _exact_side(s, b, start + n, ps * D // 2, ps * D + 4 * ps) if weights is None else None
        pos = torch.arange(start + n, device="cuda")
        if weights is not None:
            page, row = s["table"][b, pos // ps].long(), pos % ps
            weights[page, :, row] = torch.where((pos < start)[:, None], 0.9 * weights[page, :, row], 0.0)
        for h in range(case["heads"]):
            for i in range(first, n, 512):
                rows = torch.arange(i, min(n, i + 512), device="cuda")
                score = (q[at + rows, h].double() @ k[h // group].T) * s["scale"]
                score[pos[None] > start + rows[:, None]] = -math.inf
                if weights is None:
                    lse[at + rows, h] = torch.logsumexp(score, -1)
                    out[at + rows, h] = torch.exp(score - lse[at + rows, h, None]) @ v[h // group]
                else:
                    weights[page, h // group, row] += torch.exp(score - s["lse"][at + rows, h, None].double()).sum(0)
    return {"out": out, "lse": lse} if weights is None else weights


def _exact_logprobs(s):
    case = s["case"]
    tokens = s["tokens"]
    shape = tuple(tokens.shape)
    logprobs = torch.zeros(shape, dtype=torch.float64, device="cuda")
    entropy, tops = torch.zeros_like(logprobs), torch.zeros(shape + (case["top"],), dtype=torch.float64, device="cuda")

    def fill(at, row, token):
        x = torch.log_softmax(row.double() / case["temperature"], -1)
        entropy[at] = -(x.exp() * x).sum(-1)
        logprobs[at] = x.gather(-1, token.long()[..., None])[..., 0]
        tops[at] = torch.topk(x, case["top"], -1).values

    if "path" in s:
        for b in range(shape[0]):
            for i in range(shape[1]):
                node = 0 if i == 0 else int(s["path"][b, i - 1])
                if node >= 0 and int(tokens[b, i]) >= 0:
                    fill((b, i), s["logits"][b, node], tokens[b, i])
    else:
        for i in range(0, shape[0], 256):
            fill(slice(i, i + 256), s["logits"][i:i + 256], tokens[i:i + 256])
    return {"logprobs": logprobs, "entropy": entropy, "top_ids": None, "top_logprobs": tops}
