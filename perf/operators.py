"""The operators around a verification step, as calls that can be measured: logit rules over a draft tree, page tables
and slot maps, the 4-bit key/value cache (append and read back), tree attention over it, and the move of the accepted
rows inside it.

``run`` computes one pass: with ``own`` false in plain torch operations in 32 bits, with ``own`` true through the
package's entry points.  ``exact`` computes the same from the definitions in 64 bits.

Definitions
  logit rules   for node n of sequence b and token x, c = occurrences of x among the generated tokens of b and the tokens
                on the path root -> n (root excluded: it is the last generated token), seen = c > 0 or x in the prompt:
                l := (l > 0 ? l / theta : l * theta) if seen;  l -= f * c;  l -= p * [c > 0];  l += bias(x);
                l := -inf where the mask bit of x is 0
  page tables   sequence b keeps ceil((start + count) / page_size) pages; missing ones are popped from the head of a ring of
                free pages in sequence order, surplus ones are pushed at its tail; a sequence that the ring cannot serve
                keeps what it has and gets slots of -1
  4-bit cache   a row (token, head) x[0..D): scale = half((max - min) / 15), mid = half(min + 8 scale),
                code = clamp(rint((x - mid) / scale) + 8, 0, 15), value = mid + scale * (code - 8);
                a page of one head holds [key codes | value codes | key (scale, mid) | value (scale, mid)] of its positions
  attention     key j of the prefix is seen by every node, key prefix + m by node n iff m == n or m is an ancestor of n
"""
import math

import torch

own = False

_TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
_NO_PAGES = 16          # status bit of a sequence the ring of free pages could not serve


# ---------------------------------------------------------------- the cases
def listed():
    return [
        # one conversation, the smallest tree, a short history: what matters is latency
        dict(name="rules_one_small_tree", op="rules", batch=1, kconfig="2", vocab=32000, dtype="fp32", history=61, bias=0, mask="none"),
        # a serving batch with every rule on and a grammar state per tree node
        dict(name="rules_batch_grammar", op="rules", batch=64, kconfig="2x2x2x2", vocab=50272, dtype="fp16", history=1500, bias=40, mask="table"),
        # a step of a small batch: the pages the next tree needs, and its slots
        dict(name="pages_tree_step", op="pages", batch=8, mean=45, spread=0, page_size=16, held=500, free=2000),
        # admission of a batch of long prompts of different lengths, some of them partly cached
        dict(name="pages_prompts", op="pages", batch=256, mean=4100, spread=4000, page_size=16, held=700, free=80000),
        # the rows of one tree per sequence, one layer
        dict(name="append_tree", op="append", tokens=8 * 45, heads=32, dim=128, dtype="bf16", page_size=16),
        # one layer of a long packed prompt batch
        dict(name="append_prompts", op="append", tokens=40001, heads=8, dim=128, dtype="fp16", page_size=32),
        # decoding without a tree: one token, one conversation
        dict(name="attend_one_token", op="attend", batch=1, kconfig="", heads=32, kv_heads=32, dim=128, dtype="fp16", page_size=16, longest=517, ragged=0),
        # decoding of a large batch of unequal lengths with shared heads
        dict(name="attend_decode_batch", op="attend", batch=64, kconfig="", heads=32, kv_heads=8, dim=128, dtype="bf16", page_size=16, longest=8191, ragged=1),
        # a tree step of a small batch, one key head per query head
        dict(name="attend_tree", op="attend", batch=8, kconfig="4x2x2x1", heads=32, kv_heads=32, dim=128, dtype="bf16", page_size=16, longest=2050, ragged=1),
        # the large tree over long contexts with shared heads
        dict(name="attend_long_tree", op="attend", batch=4, kconfig="4x4x2x2x1", heads=32, kv_heads=8, dim=128, dtype="bf16", page_size=32, longest=16001, ragged=1),
        # the accepted rows of a small batch, all layers
        dict(name="gather_step", op="gather", batch=8, kconfig="4x2x2x1", layers=32, heads=8, dim=128, page_size=16, longest=600),
        # the same for a large batch
        dict(name="gather_batch", op="gather", batch=256, kconfig="4x4x2x2x1", layers=32, heads=8, dim=64, page_size=32, longest=350),
    ]


_TREES = ["", "2", "1x1x1x1", "2x2x2x2", "8x2x1", "4x2x2x1", "3x3x1", "4x4x2x2x1"]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["rules", "pages", "append", "attend", "attend", "gather"])
    if op == "rules":
        c = dict(op=op, batch=_spread(rng, 1, 64), kconfig=rng.choice(_TREES[1:]), vocab=rng.choice([32000, 50272, _spread(rng, 500, 65536)]),
                 dtype=rng.choice(sorted(_TYPES)), history=_spread(rng, 1, 4000), bias=rng.choice([0, 1, rng.randint(2, 300)]),
                 mask=rng.choice(["none", "table", "rows"]))
    elif op == "pages":
        mean = _spread(rng, 1, 4000)
        c = dict(op=op, batch=_spread(rng, 1, 256), mean=mean, spread=rng.randint(0, mean - 1), page_size=rng.choice([16, 32, 64, 128]),
                 held=_spread(rng, 1, 2000), free=_spread(rng, 100, 80000))
    elif op == "append":
        c = dict(op=op, tokens=_spread(rng, 1, 40000), heads=rng.choice([1, 2, 5, 8]), dim=rng.choice([64, 128]), dtype=rng.choice(sorted(_TYPES)),
                 page_size=rng.choice([16, 32, 64, 128]))
    elif op == "attend":
        c = dict(op=op, batch=_spread(rng, 1, 48), kconfig=rng.choice(_TREES), heads=0, kv_heads=rng.choice([1, 2, 4, 8, 32]), dim=rng.choice([64, 128]),
                 dtype=rng.choice(["bf16", "fp16"]), page_size=rng.choice([16, 32, 64, 128]), longest=_spread(rng, 1, 16000), ragged=rng.choice([0, 1]))
        c["heads"] = c["kv_heads"] * rng.choice([1, 1, 3, 4, 8])
    else:
        c = dict(op=op, batch=_spread(rng, 1, 128), kconfig=rng.choice(_TREES[1:]), layers=rng.randint(1, 32), heads=rng.choice([1, 4, 8]),
                 dim=rng.choice([64, 128]), page_size=rng.choice([16, 32, 64]), longest=_spread(rng, 1, 350))
    # no more than the largest listed case of the operator
    most = {m: max(work(x)[m] for x in listed() if x["op"] == op) for m in ("bytes", "flops")}
    while any(work(c)[m] > most[m] for m in most):
        for key in ("batch", "tokens", "longest"):
            if c.get(key, 1) > 1:
                c[key] = (c[key] + 1) // 2
                break
        else:
            c["heads"], c["kv_heads"] = c.get("kv_heads", 1), c.get("kv_heads", 1)
            break
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
    """Prefix length of every sequence: from `longest` down to a quarter of it where the batch is ragged."""
    B, top = case["batch"], case["longest"]
    return [top - (3 * top * b) // (4 * B) if case["ragged"] else top for b in range(B)]


def _counts(case):
    """New tokens of every sequence of a pages case, spread evenly around the mean."""
    B = case["batch"]
    return [max(1, case["mean"] + (case["spread"] * (2 * b + 1 - B)) // B) for b in range(B)]


def work(case):
    """Bytes and operations that one pass cannot do without."""
    if case["op"] == "rules":
        n = case["batch"] * len(_parents(case["kconfig"]))
        es = 4 if case["dtype"] == "fp32" else 2
        mask = {"none": 0, "table": 64, "rows": n}[case["mask"]] * (case["vocab"] + 31) // 32 * 4
        return {"bytes": 2 * n * case["vocab"] * es + mask + case["batch"] * (4 * case["history"] + 8 * case["bias"]) + 8 * n, "flops": 0}
    if case["op"] == "pages":
        total = sum(_counts(case))
        return {"bytes": 8 * total + 8 * total // case["page_size"] + 24 * case["batch"], "flops": 0}
    if case["op"] == "append":
        es = 4 if case["dtype"] == "fp32" else 2
        row = 2 * case["dim"] * es + 2 * (case["dim"] + 8) + 2 * case["dim"] * es     # read, written, read back, returned
        return {"bytes": case["tokens"] * (case["heads"] * row + 16), "flops": 0}
    n = len(_parents(case["kconfig"]))
    if case["op"] == "attend":
        keys = sum(_lengths(case)) + case["batch"] * n
        rows = case["batch"] * n * case["heads"]
        seen = sum(_lengths(case)) * n + case["batch"] * sum(map(sum, _ancestors(case["kconfig"])))
        return {"bytes": keys * case["kv_heads"] * (case["dim"] + 8) + rows * (4 * case["dim"] + 4), "flops": 4 * case["dim"] * case["heads"] * seen}
    depth = sum(1 for t in case["kconfig"].split("x") if t)
    return {"bytes": 2 * case["batch"] * (depth / 2) * case["layers"] * case["heads"] * (case["dim"] + 8) + 1, "flops": 0}


def _ancestors(kconfig):
    """[n][m] = 1 iff m == n or m is an ancestor of n."""
    rows = []
    for n, p in enumerate(_parents(kconfig)):
        row = list(rows[p]) if n else []
        rows.append(row + [0] * (n - len(row)) + [1])
    size = len(rows)
    return [r + [0] * (size - len(r)) for r in rows]


# ---------------------------------------------------------------- inputs
def _quantise(x):
    """codes [.., D] as whole numbers, scale and mid as half [..]; x float32."""
    lo, hi = x.amin(-1).double(), x.amax(-1).double()
    scale = ((hi - lo) / 15).to(torch.float16)
    mid = (lo + 8 * scale.double()).to(torch.float16)
    s, m = scale.double().unsqueeze(-1), mid.double().unsqueeze(-1)
    codes = torch.where(s > 0, torch.round((x.double() - m) / torch.where(s > 0, s, 1.0)) + 8, 8.0).clamp(0, 15)
    return codes.to(torch.uint8), scale, mid


def _rows_to_bytes(x):
    """(codes [.., D / 2] bytes, (scale, mid) [.., 4] bytes) of rows x."""
    codes, scale, mid = _quantise(x)
    return codes[..., 0::2] | (codes[..., 1::2] << 4), torch.stack([scale, mid], -1).view(torch.uint8)


def _block(dim, page_size):
    return page_size * (dim + 8)


def _cache(gen, n_pages, heads, dim, page_size):
    """Pages filled with quantised rows: normal keys with an offset per channel and a few louder tokens, normal values."""
    pages = torch.empty((n_pages, heads, _block(dim, page_size)), dtype=torch.uint8, device="cuda")
    offset = 0.5 * torch.randn((heads, 1, dim), generator=gen, device="cuda")
    half, at = page_size * dim // 2, max(1, (1 << 26) // (heads * page_size * dim))
    for p in range(0, n_pages, at):
        n = min(at, n_pages - p)
        k = torch.randn((n, heads, page_size, dim), generator=gen, device="cuda") + offset
        k *= torch.exp(0.3 * torch.randn((n, heads, page_size, 1), generator=gen, device="cuda"))
        v = torch.randn((n, heads, page_size, dim), generator=gen, device="cuda")
        (kc, kp), (vc, vp) = _rows_to_bytes(k), _rows_to_bytes(v)
        view = pages[p:p + n]
        view[:, :, :half], view[:, :, half:2 * half] = kc.reshape(n, heads, -1), vc.reshape(n, heads, -1)
        view[:, :, 2 * half:2 * half + 4 * page_size] = kp.reshape(n, heads, -1)
        view[:, :, 2 * half + 4 * page_size:] = vp.reshape(n, heads, -1)
    return pages


def _binding():
    from paper_2401_06706_b200 import binding
    return binding


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"case": case, "op": case["op"]}
    {"rules": _prepare_rules, "pages": _prepare_pages, "append": _prepare_append, "attend": _prepare_attend, "gather": _prepare_gather}[case["op"]](case, gen, s)
    return s


def _randint(gen, low, high, shape, dtype=torch.int32):
    return torch.randint(low, high, shape, generator=gen, device="cuda", dtype=dtype)


def _prepare_rules(case, gen, s):
    B, V, parent = case["batch"], case["vocab"], _parents(case["kconfig"])
    N, H = len(parent), case["history"]
    s["anc"] = torch.tensor(_ancestors(case["kconfig"]), device="cuda").bool()
    s["logits"] = (2.5 * torch.randn((B, N, V), generator=gen, device="cuda")).to(_TYPES[case["dtype"]])
    # a history in which some tokens return often, as words do; lengths differ
    few = _randint(gen, 0, V, (B, H // 3 + 1))
    s["history"] = torch.gather(few, 1, _randint(gen, 0, H // 3 + 1, (B, H), torch.int64))
    s["history_len"] = _randint(gen, H // 2, H + 1, (B,))
    s["prompt_len"] = s["history_len"] // 2
    s["cand"] = _randint(gen, 0, V, (B, N))
    s["cand"][:, N // 2:] = torch.gather(s["history"], 1, _randint(gen, 0, H, (B, N - N // 2), torch.int64))
    s["repetition"] = 1 + 0.3 * torch.rand((B,), generator=gen, device="cuda")
    s["frequency"] = 0.5 * torch.rand((B,), generator=gen, device="cuda")
    s["presence"] = 0.5 * torch.rand((B,), generator=gen, device="cuda")
    # ids without repetition in a row
    s["bias_ids"] = torch.rand((B, V), generator=gen, device="cuda").argsort(1)[:, :case["bias"]].to(torch.int32).contiguous()
    s["bias_values"] = 4 * torch.randn((B, case["bias"]), generator=gen, device="cuda")
    words = (V + 31) // 32
    s["masks"] = s["mask_index"] = None
    if case["mask"] != "none":
        # a grammar allows few tokens in some states and most in others
        n = 64 if case["mask"] == "table" else B * N
        every = _randint(gen, -2**31, 2**31 - 1, (n, words)) & _randint(gen, -2**31, 2**31 - 1, (n, words))
        s["masks"] = torch.where(_randint(gen, 0, 2, (n, 1)) > 0, every, ~every)
        s["mask_index"] = _randint(gen, -1, n, (B, N)) if case["mask"] == "table" else torch.arange(n, device="cuda", dtype=torch.int32).view(B, N)
    if own:
        b = _binding()
        s["parent"] = parent
        s["rules"] = b.LogitRules(history=s["history"], history_len=s["history_len"], prompt_len=s["prompt_len"], repetition=s["repetition"],
                                  frequency=s["frequency"], presence=s["presence"], bias_ids=s["bias_ids"], bias_values=s["bias_values"],
                                  masks=s["masks"], mask_index=s["mask_index"])
        s["out"] = torch.empty_like(s["logits"])


def _prepare_pages(case, gen, s):
    B, ps = case["batch"], case["page_size"]
    count = torch.tensor(_counts(case), device="cuda", dtype=torch.int32)
    s["count"] = count[torch.randperm(B, generator=gen, device="cuda")]
    s["start"] = _randint(gen, 0, case["held"] * 2, (B,))
    # what is held follows the start, with some sequences that hold surplus pages of a longer tree or prompt
    s["held"] = (s["start"] + ps - 1) // ps + _randint(gen, 0, 3, (B,))
    width = (2 * case["held"] + max(_counts(case))) // ps + 3
    total, cap = int(s["held"].sum()), B * width + case["free"]
    ids = torch.randperm(cap, generator=gen, device="cuda").to(torch.int32)
    s["table"] = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    s["table"][torch.arange(width, device="cuda") < s["held"][:, None]] = ids[:total]
    head = int(_randint(gen, 0, cap, ()))
    s["ring"] = torch.full((cap,), -1, dtype=torch.int32, device="cuda")
    s["ring"][(head + torch.arange(case["free"], device="cuda")) % cap] = ids[total:total + case["free"]]
    s["ring_state"] = torch.tensor([head, case["free"], 0, 0], dtype=torch.int32, device="cuda")
    s["slots"] = torch.full((sum(_counts(case)),), -1, dtype=torch.int64, device="cuda")
    if own:
        b = _binding()
        s["plan"] = b.PageTables(s["table"], s["held"], s["ring"], s["ring_state"], ps, held_out=torch.empty_like(s["held"]),
                                 ring_state_out=torch.zeros_like(s["ring_state"]))


def _prepare_append(case, gen, s):
    T, H, D, ps = case["tokens"], case["heads"], case["dim"], case["page_size"]
    n_pages = (T + ps - 1) // ps + 3
    s["keys"] = (torch.randn((T, H, D), generator=gen, device="cuda") + 0.5 * torch.randn((H, D), generator=gen, device="cuda")).to(_TYPES[case["dtype"]])
    s["values"] = torch.randn((T, H, D), generator=gen, device="cuda").to(_TYPES[case["dtype"]])
    # runs of positions in pages that lie anywhere
    page = torch.randperm(n_pages, generator=gen, device="cuda")
    pos = torch.arange(T, device="cuda") + int(_randint(gen, 0, 2 * ps, ()))
    s["slots"] = page[pos // ps] * ps + pos % ps
    s["pages"] = torch.zeros((n_pages, H, _block(D, ps)), dtype=torch.uint8, device="cuda")
    if own:
        b = _binding()
        s["cache"] = b.KvCache(s["pages"], D, ps)
        s["keys_out"], s["values_out"] = torch.empty_like(s["keys"]), torch.empty_like(s["values"])


def _prepare_attend(case, gen, s):
    B, D, ps, parent = case["batch"], case["dim"], case["page_size"], _parents(case["kconfig"])
    N = len(parent)
    lengths = torch.tensor(_lengths(case), device="cuda", dtype=torch.int32)
    s["prefix_len"] = lengths[torch.randperm(B, generator=gen, device="cuda")].contiguous()
    width = (case["longest"] + N + ps - 1) // ps
    need = (s["prefix_len"] + N + ps - 1) // ps
    n_pages = int(need.sum()) + 2
    s["table"] = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    s["table"][torch.arange(width, device="cuda") < need[:, None]] = torch.randperm(n_pages, generator=gen, device="cuda")[:int(need.sum())].to(torch.int32)
    s["pages"] = _cache(gen, n_pages, case["kv_heads"], D, ps)
    s["q"] = (1.2 * torch.randn((B, N, case["heads"], D), generator=gen, device="cuda")).to(_TYPES[case["dtype"]])
    s["anc"] = torch.tensor(_ancestors(case["kconfig"]), device="cuda").bool()
    s["scale"] = 1 / math.sqrt(D)
    if own:
        b = _binding()
        s["cache"] = b.KvCache(s["pages"], D, ps)
        s["attention"] = b.TreeAttention(B, parent, case["heads"], s["q"].dtype, s["cache"], width)


def _prepare_gather(case, gen, s):
    B, D, ps, parent = case["batch"], case["dim"], case["page_size"], _parents(case["kconfig"])
    N, L = len(parent), case["layers"]
    s["prefix_len"] = _randint(gen, 0, case["longest"] + 1, (B,))
    width = (case["longest"] + N + ps - 1) // ps
    n_pages = B * width
    s["table"] = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32).view(B, width)
    s["pages"] = _randint(gen, 0, 256, (L, n_pages, case["heads"], _block(D, ps)), torch.uint8)
    # a walk down the tree: a child of the node before it, as far as it got
    first, many = {}, {}
    for n, p in enumerate(parent):
        first.setdefault(p, n)
        many[p] = many.get(p, 0) + 1
    depth = sum(1 for t in case["kconfig"].split("x") if t)
    node = torch.zeros((B,), dtype=torch.int64, device="cuda")
    first = torch.tensor([first.get(n, 0) for n in range(N)], device="cuda")
    many = torch.tensor([many.get(n, 1) for n in range(N)], device="cuda")
    path = torch.full((B, depth + 1), -1, dtype=torch.int32, device="cuda")
    s["accept_len"] = _randint(gen, 0, depth + 1, (B,))
    for i in range(depth):
        node = first[node] + (torch.rand((B,), generator=gen, device="cuda") * many[node]).long()
        path[:, i] = torch.where(s["accept_len"] > i, node, -1).to(torch.int32)
    s["path"] = path
    if own:
        s["cache"] = _binding().KvCache(s["pages"], D, ps)


# ---------------------------------------------------------------- one pass
def run(state):
    return {"rules": _run_rules, "pages": _run_pages, "append": _run_append, "attend": _run_attend, "gather": _run_gather}[state["op"]](state)


def _run_rules(s):
    if own:
        return _binding().mcsd_apply_logit_rules(s["logits"], s["parent"], s["cand"], s["rules"], out=s["out"])
    B, N, V = s["logits"].shape
    at = torch.arange(s["history"].shape[1], device="cuda")
    ids, live = s["history"].long(), (at < s["history_len"][:, None])
    prompt = at < s["prompt_len"][:, None]
    out_count = torch.zeros((B, V), device="cuda").scatter_add_(1, ids, (live & ~prompt).float())
    in_prompt = torch.zeros((B, V), device="cuda").scatter_add_(1, ids, (live & prompt).float()) > 0
    # tokens on the path of every node, the root's excluded
    on_path = s["anc"].clone()
    on_path[:, 0] = False
    path = s["cand"].long()[:, None, :].expand(B, N, N)
    count = out_count[:, None, :] + torch.zeros((B, N, V), device="cuda").scatter_add_(2, path, on_path[None].float().expand(B, N, N))
    row = lambda t: t[:, None, None]
    l = s["logits"].float()
    seen = (count > 0) | in_prompt[:, None, :]
    l = torch.where(seen, torch.where(l > 0, l / row(s["repetition"]), l * row(s["repetition"])), l)
    l = l - row(s["frequency"]) * count - row(s["presence"]) * (count > 0)
    bias = torch.zeros((B, V), device="cuda").scatter_(1, s["bias_ids"].long(), s["bias_values"])
    l = l + bias[:, None, :]
    if s["masks"] is not None:
        x = torch.arange(V, device="cuda")
        words = s["masks"][s["mask_index"].long().clamp(min=0)]
        allowed = ((words[..., x // 32] >> (x % 32)) & 1) > 0
        l = torch.where(allowed | (s["mask_index"] < 0)[..., None], l, float("-inf"))
    return l.to(s["logits"].dtype)


def _run_pages(s):
    if own:
        p = s["plan"]
        p.mcsd_build_page_tables(s["start"], s["count"], slots=s["slots"])
        return {"table": p.table, "held": p.held_out, "ring": p.ring, "state": p.ring_state_out[:2], "cu_tokens": p.cu_tokens, "slots": s["slots"], "status": p.status}
    ps, cap, width = s["case"]["page_size"], s["ring"].shape[0], s["table"].shape[1]
    head, free = s["ring_state"][0], s["ring_state"][1]
    start, count, held = s["start"].long(), s["count"].long(), s["held"].long()
    want = (start + count + ps - 1) // ps
    wide = want > width
    grow = torch.where(wide, 0, (want - held).clamp(min=0))
    upto = torch.cumsum(grow, 0)
    refused = wide | ((grow > 0) & (upto > free))
    grow_off = upto - grow
    surplus = torch.where(wide, 0, (held - want).clamp(min=0))
    push_off = torch.cumsum(surplus, 0) - surplus
    col = torch.arange(width, device="cuda")
    new = (col >= held[:, None]) & (col < want[:, None]) & ~refused[:, None]
    popped = s["ring"][(head + grow_off[:, None] + col - held[:, None]) % cap]
    table = torch.where(new, popped, s["table"])
    back = (col >= want[:, None]) & (col < held[:, None]) & ~wide[:, None]
    to = (head + free + push_off[:, None] + col - want[:, None]) % cap
    ring = s["ring"].clone().index_put_((to[back],), s["table"][back])
    taken = torch.where(refused, 0, grow).sum()
    held_out = torch.where(refused, held, want).to(torch.int32)
    state = torch.stack([(head + taken) % cap, free - taken + surplus.sum()]).to(torch.int32)
    cu = torch.cat([torch.zeros(1, dtype=torch.long, device="cuda"), torch.cumsum(count, 0)])
    seq = torch.repeat_interleave(torch.arange(count.shape[0], device="cuda"), count, output_size=s["slots"].shape[0])
    pos = start[seq] + torch.arange(s["slots"].shape[0], device="cuda") - cu[seq]
    slots = torch.where(refused[seq], -1, table[seq, (pos // ps).clamp(max=width - 1)].long() * ps + pos % ps)
    return {"table": table, "held": held_out, "ring": ring, "state": state, "cu_tokens": cu.to(torch.int32), "slots": slots, "status": torch.where(refused, _NO_PAGES, 0).to(torch.int32)}


def _values(codes, scale, mid):
    """Values of packed rows [.., D / 2] in 32 bits."""
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).float()
    return mid.float().unsqueeze(-1) + scale.float().unsqueeze(-1) * (c - 8)


def _split(blocks, dim, page_size):
    """Key codes, value codes, key parameters, value parameters of pages [.., block], each [.., page_size, ..]."""
    half = page_size * dim // 2
    kc, vc, kp, vp = torch.split(blocks, [half, half, 4 * page_size, 4 * page_size], -1)
    shape = blocks.shape[:-1] + (page_size,)
    return (kc.reshape(shape + (dim // 2,)), vc.reshape(shape + (dim // 2,)),
            kp.contiguous().view(torch.float16).reshape(shape + (2,)), vp.contiguous().view(torch.float16).reshape(shape + (2,)))


def _run_append(s):
    if own:
        b = _binding()
        b.mcsd_append_kv(s["cache"], s["keys"], s["values"], s["slots"])
        return b.mcsd_read_kv(s["cache"], s["slots"], keys=s["keys_out"], values=s["values_out"])
    ps, D = s["case"]["page_size"], s["case"]["dim"]
    page, row, half = s["slots"] // ps, s["slots"] % ps, ps * D // 2
    (kc, kp), (vc, vp) = _rows_to_bytes(s["keys"].float()), _rows_to_bytes(s["values"].float())
    n_pages, heads, _ = s["pages"].shape
    s["pages"][:, :, :half].view(n_pages, heads, ps, -1)[page, :, row] = kc
    s["pages"][:, :, half:2 * half].view(n_pages, heads, ps, -1)[page, :, row] = vc
    s["pages"][:, :, 2 * half:2 * half + 4 * ps].view(n_pages, heads, ps, -1)[page, :, row] = kp
    s["pages"][:, :, 2 * half + 4 * ps:].view(n_pages, heads, ps, -1)[page, :, row] = vp
    kc, vc, kp, vp = (t[page, :, row] for t in _split(s["pages"], D, ps))
    return _values(kc, kp[..., 0], kp[..., 1]).to(s["keys"].dtype), _values(vc, vp[..., 0], vp[..., 1]).to(s["keys"].dtype)


def _run_attend(s):
    if own:
        out = s["attention"].mcsd_tree_attention(s["q"], s["cache"], s["table"], s["prefix_len"], scale=s["scale"])
        return {"out": out.out, "lse": out.lse}
    D, ps = s["case"]["dim"], s["case"]["page_size"]
    B, N, heads, _ = s["q"].shape
    kv = s["case"]["kv_heads"]
    kc, vc, kp, vp = _split(s["pages"][s["table"].long().clamp(min=0)], D, ps)      # [B, pages, heads, page_size, ..]
    rows = lambda t: t.transpose(1, 2).flatten(2, 3)                                # [B, heads, positions, ..]
    k, v = rows(_values(kc, kp[..., 0], kp[..., 1])), rows(_values(vc, vp[..., 0], vp[..., 1]))
    q = s["q"].float().view(B, N, kv, heads // kv, D).transpose(1, 2).reshape(B, kv, -1, D)
    score = torch.matmul(q, k.transpose(2, 3)) * s["scale"]
    at = torch.arange(k.shape[2], device="cuda") - s["prefix_len"][:, None]         # position within the tree
    seen = (at < 0)[:, None, :] | ((at >= 0) & (at < N))[:, None, :] & s["anc"][:, at.clamp(0, N - 1)].transpose(0, 1)
    score = score.masked_fill(~seen.repeat_interleave(heads // kv, 1)[:, None], float("-inf"))
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v) / total
    back = lambda t: t.view(B, kv, N, heads // kv, -1).transpose(1, 2).reshape(B, N, heads, -1)
    return {"out": back(out).to(s["q"].dtype), "lse": back(top + torch.log(total))[..., 0]}


def _run_gather(s):
    if own:
        return _binding().mcsd_gather_accepted_pages(s["cache"], s["table"], s["prefix_len"], s["path"], s["accept_len"])
    ps, D = s["case"]["page_size"], s["case"]["dim"]
    half, pages = ps * D // 2, s["pages"]
    depth = s["path"].shape[1] - 1
    i = torch.arange(depth, device="cuda")
    moved = (i < s["accept_len"][:, None]) & (s["path"][:, :depth] > i + 1)
    seq, i = torch.nonzero(moved, as_tuple=True)
    source = s["prefix_len"][seq].long() + s["path"][seq, i]
    target = s["prefix_len"][seq].long() + 1 + i
    sp, sr, tp, tr = s["table"][seq, source // ps].long(), source % ps, s["table"][seq, target // ps].long(), target % ps
    parts = [pages[..., a:b].unflatten(-1, (ps, -1)) for a, b in ((0, half), (half, 2 * half), (2 * half, 2 * half + 4 * ps), (2 * half + 4 * ps, 2 * half + 8 * ps))]
    new = [part[:, sp, :, sr] for part in parts]                                    # all reads before any write
    [part.index_put_((torch.arange(pages.shape[0], device="cuda")[:, None, None], tp[:, None], torch.arange(pages.shape[2], device="cuda")[None, :], tr[:, None]), x.permute(1, 0, 2, 3))
     for part, x in zip(parts, new)]
    return pages


# ---------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rules":
        return _exact_rules(s)
    if case["op"] == "append":
        return tuple(_exact_row_values(s[name]) for name in ("keys", "values"))
    if case["op"] == "attend":
        return _exact_attend(s)
    return None         # whole numbers and moved bytes


def _exact_rules(s):
    B, N, V = s["logits"].shape
    out = torch.empty((B, N, V), dtype=torch.float64, device="cuda")
    cand, anc = s["cand"].cpu(), s["anc"].cpu()
    bits = torch.arange(32, device="cuda")
    for b in range(B):
        length, prompt = int(s["history_len"][b]), int(s["prompt_len"][b])
        theta, f, p = (float(s[k][b]) for k in ("repetition", "frequency", "presence"))
        made = torch.bincount(s["history"][b, prompt:length].long(), minlength=V).double()
        given = torch.bincount(s["history"][b, :prompt].long(), minlength=V) > 0
        bias = torch.zeros(V, dtype=torch.float64, device="cuda")
        bias[s["bias_ids"][b].long()] = s["bias_values"][b].double()
        for n in range(N):
            c = made.clone()
            for m in range(1, n + 1):
                if anc[n, m]:
                    c[int(cand[b, m])] += 1
            l = s["logits"][b, n].double()
            penal = torch.where(l > 0, l / theta, l * theta)
            l = torch.where((c > 0) | given, penal, l) - f * c - torch.where(c > 0, p, 0.0) + bias
            if s["masks"] is not None and int(s["mask_index"][b, n]) >= 0:
                word = s["masks"][int(s["mask_index"][b, n])]
                l[((word[:, None] >> bits) & 1).flatten()[:V] == 0] = -math.inf
            out[b, n] = l
    return out


def _exact_row_values(x):
    x = x.double()
    low, high = x.min(-1, keepdim=True).values, x.max(-1, keepdim=True).values
    scale = ((high - low) / 15).half().double()
    mid = (low + 8 * scale).half().double()
    step = ((x - mid) / scale).round().clamp(-8, 7)
    return torch.where(scale > 0, mid + scale * step, mid)


def _exact_attend(s):
    case = s["case"]
    ps, D, kv, heads = case["page_size"], case["dim"], case["kv_heads"], case["heads"]
    parent = _parents(case["kconfig"])
    B, N, group = case["batch"], len(parent), heads // kv
    out = torch.empty((B, N, heads, D), dtype=torch.float64, device="cuda")
    lse = torch.empty((B, N, heads), dtype=torch.float64, device="cuda")
    for b in range(B):
        prefix = int(s["prefix_len"][b])
        keys = prefix + N
        block = s["pages"][s["table"][b, :(keys + ps - 1) // ps].long()].permute(1, 0, 2)            # [heads, pages, block]

        def side(codes_at, param_at):
            raw = block[..., codes_at:codes_at + ps * D // 2].reshape(kv, -1, D // 2)[:, :keys]
            par = block[..., param_at:param_at + 4 * ps].contiguous().view(torch.float16).double().reshape(kv, -1, 2)[:, :keys]
            x = torch.empty((kv, keys, D), dtype=torch.float64, device="cuda")
            x[..., 0::2], x[..., 1::2] = (raw % 16).double(), (raw // 16).double()
            return par[..., 1:] + par[..., :1] * (x - 8)

        k, v = side(0, ps * D), side(ps * D // 2, ps * D + 4 * ps)
        hidden = torch.zeros((N, keys), dtype=torch.bool, device="cuda")
        hidden[:, prefix:] = True
        for n in range(N):
            m = n
            while m >= 0:
                hidden[n, prefix + m] = False
                m = parent[m]
        for h in range(heads):
            score = (s["q"][b, :, h].double() @ k[h // group].T) * s["scale"]
            score[hidden] = -math.inf
            lse[b, :, h] = torch.logsumexp(score, -1)
            out[b, :, h] = torch.exp(score - lse[b, :, h, None]) @ v[h // group]
    return {"out": out, "lse": lse}
