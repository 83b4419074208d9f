"""Plain NumPy statements, in 64 bits, of the operators around the verification step: logit rules, page tables, the 4-bit
cache, tree attention, the move of accepted rows.  One sequence, one row, one token at a time; nothing is shared with
the package but the documented memory layout."""
import numpy as np

STATUS_NO_PAGES, STATUS_BAD_MASK = 16, 32


def path(parent, n):
    """Nodes from n up to and including the root."""
    nodes = []
    while n >= 0:
        nodes.append(n)
        n = int(parent[n])
    return nodes


# ---------------------------------------------------------------- logit rules
def logit_rules(logits, parent, cand, *, history=None, history_len=None, prompt_len=None, repetition=None, frequency=None,
                presence=None, bias_ids=None, bias_values=None, masks=None, mask_index=None, nodes=None):
    """(values float64 [B, rows, V], bound on the size of what was added up, status [B]).  Rows outside `nodes` are copied."""
    B, rows, V = logits.shape
    out = logits.astype(np.float64).copy()
    size = np.abs(out)
    status = np.zeros(B, dtype=np.int32)
    penalise = repetition is not None or frequency is not None or presence is not None
    for b in range(B):
        theta = 1.0 if repetition is None else float(repetition[b])
        f = 0.0 if frequency is None else float(frequency[b])
        p = 0.0 if presence is None else float(presence[b])
        base, prompt = np.zeros(V), np.zeros(V, dtype=bool)
        if penalise and history is not None:
            length = min(max(int(history_len[b]), 0), history.shape[1])
            for i in range(length):
                t = int(history[b, i])
                if 0 <= t < V:
                    if prompt_len is not None and i < int(prompt_len[b]):
                        prompt[t] = True
                    else:
                        base[t] += 1
        bias = np.zeros(V)
        if bias_ids is not None:
            for i in range(bias_ids.shape[1]):
                if 0 <= int(bias_ids[b, i]) < V:
                    bias[int(bias_ids[b, i])] = float(bias_values[b, i])
        for n in range(rows) if nodes is None else nodes:
            count = base.copy()
            if penalise and cand is not None:
                for m in path(parent, n)[:-1]:
                    if 0 <= int(cand[b, m]) < V:
                        count[int(cand[b, m])] += 1
            l = out[b, n]
            with np.errstate(invalid="ignore", over="ignore"):
                seen = (count > 0) | prompt
                pen = np.where(l > 0, l / theta, l * theta)
                size[b, n] = np.maximum(np.abs(l), np.abs(pen)) + abs(f) * count + abs(p) * (count > 0) + np.abs(bias)
                l = np.where(seen, pen, l) - np.where(count > 0, f * count + p, 0.0)
                l = np.where(bias != 0, l + bias, l)
            if masks is not None:
                m = b * len(parent) + n if mask_index is None else int(mask_index[b, n])
                if 0 <= m < masks.shape[0]:
                    words = masks[m].astype(np.int64) & 0xFFFFFFFF
                    bits = (words[np.arange(V) // 32] >> (np.arange(V) % 32)) & 1
                    l = np.where(bits == 1, l, -np.inf)
                elif m >= 0:
                    status[b] |= STATUS_BAD_MASK
            out[b, n] = l
    return out, size, status


# ---------------------------------------------------------------- page tables
def page_tables(start, count, table, held, ring, head, free, page_size):
    """(table, held, ring, head, free, slots, cu, status) of one call, sequence by sequence."""
    table, held, ring = table.copy(), held.copy(), ring.copy()
    B, width, cap = table.shape[0], table.shape[1], ring.shape[0]
    old_table, old_held = table.copy(), held.copy()
    status, want = np.zeros(B, dtype=np.int32), held.astype(np.int64).copy()
    demand, taken, returned = 0, 0, 0
    for b in range(B):
        if start[b] < 0:
            continue
        need = -(-(int(start[b]) + max(int(count[b]), 0)) // page_size)
        if need > width:
            status[b] = STATUS_NO_PAGES
            continue
        grow = max(need - int(held[b]), 0)
        if grow and demand + grow > free:
            status[b] = STATUS_NO_PAGES
            demand += grow
            continue
        demand += grow
        for j in range(int(held[b]), need):
            table[b, j] = ring[(head + taken) % cap]
            taken += 1
        want[b] = need
    for b in range(B):
        for j in range(int(want[b]), int(old_held[b])):
            ring[(head + free + returned) % cap] = old_table[b, j]
            returned += 1
    slots, cu = [], [0]
    for b in range(B):
        n = max(int(count[b]), 0) if start[b] >= 0 else 0
        for i in range(n):
            pos = int(start[b]) + i
            page = -1 if status[b] else int(table[b, pos // page_size])
            slots.append(-1 if page < 0 else page * page_size + pos % page_size)
        cu.append(cu[-1] + n)
    return (table, want.astype(np.int32), ring, (head + taken) % cap, free - taken + returned,
            np.array(slots, dtype=np.int64), np.array(cu, dtype=np.int32), status)


# ---------------------------------------------------------------- the 4-bit cache
def _half(x):
    with np.errstate(over="ignore"):
        return np.clip(x, -65504.0, 65504.0).astype(np.float32).astype(np.float16)


def quantise(x):
    """codes uint8 [.., D], scale and mid float16 [..] of rows x."""
    x = x.astype(np.float64)
    bad = ~np.isfinite(x).all(-1)
    x = np.where(bad[..., None], 0.0, x)
    lo, hi = x.min(-1), x.max(-1)
    scale = _half((hi - lo) / 15)
    mid = _half(lo + 8 * scale.astype(np.float64))
    s, m = scale.astype(np.float64)[..., None], mid.astype(np.float64)[..., None]
    codes = np.where(s > 0, np.clip(np.rint((x - m) / np.where(s > 0, s, 1.0)) + 8, 0, 15), 8).astype(np.uint8)
    codes[bad] = 8
    return codes, np.where(bad, np.float16(0), scale), np.where(bad, np.float16(np.nan), mid)


def _views(pages, dim, ps):
    """[key codes, value codes, key parameters, value parameters] of pages [n, heads, block], as views."""
    n, heads, _ = pages.shape
    half = ps * dim // 2
    kc = pages[:, :, :half].reshape(n, heads, ps, dim // 2)
    vc = pages[:, :, half:2 * half].reshape(n, heads, ps, dim // 2)
    kp = pages[:, :, 2 * half:2 * half + 4 * ps].reshape(n, heads, ps, 4)
    vp = pages[:, :, 2 * half + 4 * ps:].reshape(n, heads, ps, 4)
    return kc, vc, kp, vp


def append(pages, keys, values, slots, dim, ps):
    pages = pages.copy()
    n, heads, _ = pages.shape
    half = ps * dim // 2
    for which, x in enumerate((keys, values)):
        codes, scale, mid = quantise(x)
        packed = codes[..., 0::2] | (codes[..., 1::2] << 4)
        param = np.stack([scale, mid], -1).astype(np.float16)
        for t, slot in enumerate(slots):
            page, row = divmod(int(slot), ps)
            if slot < 0 or page >= n:
                continue
            for h in range(heads):
                pages[page, h, which * half + row * (dim // 2):which * half + (row + 1) * (dim // 2)] = packed[t, h]
                at = 2 * half + which * 4 * ps + 4 * row
                pages[page, h, at:at + 4] = param[t, h].view(np.uint8)
    return pages


def row_values(pages, page, row, dim, ps):
    """(keys, values, key (scale, mid), value (scale, mid)) in float64, [heads, ..], of one row."""
    kc, vc, kp, vp = (v[page, :, row] for v in _views(pages, dim, ps))
    got = []
    for codes, par in ((kc, kp), (vc, vp)):
        par = np.ascontiguousarray(par).view(np.float16).astype(np.float64)
        c = np.empty(codes.shape[:-1] + (dim,))
        c[..., 0::2], c[..., 1::2] = codes & 15, codes >> 4
        got.append((par[:, 1:] + par[:, :1] * (c - 8), par))
    return got[0][0], got[1][0], got[0][1], got[1][1]


# ---------------------------------------------------------------- attention
def attention(q, pages, table, prefix_len, parent, dim, ps, scale, eps):
    """(out, lse, tolerance of out, tolerance of lse) in float64; rows of unused entries are NaN.

    The tolerance counts, per output: the final rounding (eps / 2); weights rounded to half precision, relative to the
    largest value scale among the keys (2^-12 of a weight, or 2^-25 of the largest scale where a weight underflows);
    float32 sums of D products in the scores (D 2^-24 of the sum of magnitudes, the codes taken from 0 to 15) and a few
    float32 roundings in exponentials and sums (2^-19)."""
    B, N, H, _ = q.shape
    n_pages, kv, _ = pages.shape
    out, lse = np.full(q.shape, np.nan), np.full((B, N, H), np.nan)
    tol, tol_lse = np.zeros(q.shape), np.zeros((B, N, H))
    for b in range(B):
        prefix = int(prefix_len[b])
        if prefix < 0:
            continue
        # values and parameters of every position that is there, [kv, positions, ..]
        there = [pos for pos in range(prefix + N) if pos // ps < table.shape[1] and 0 <= int(table[b, pos // ps]) < n_pages]
        index = {pos: i for i, pos in enumerate(there)}
        K, V, KP, VP = (np.zeros((kv, len(there), w)) for w in (dim, dim, 2, 2))
        for i, pos in enumerate(there):
            K[:, i], V[:, i], KP[:, i], VP[:, i] = row_values(pages, int(table[b, pos // ps]), pos % ps, dim, ps)
        common = [index[pos] for pos in there if pos < prefix]
        for n in range(N):
            seen = common + [index[prefix + m] for m in path(parent, n)[::-1] if prefix + m in index]
            if not seen:
                out[b, n], lse[b, n] = 0.0, -np.inf
                continue
            k, v, kp, vp = (x[:, seen] for x in (K, V, KP, VP))
            for h in range(H):
                g = h // (H // kv)
                qq = q[b, n, h].astype(np.float64)
                s = scale * (k[g] @ qq)
                top = s.max()
                with np.errstate(invalid="ignore", over="ignore"):
                    w = np.exp(s - top)
                    p = w / w.sum()
                    out[b, n, h] = p @ v[g]
                    lse[b, n, h] = top + np.log(w.sum())
                    ks, km, vs, vm = kp[g, :, 0], kp[g, :, 1], vp[g, :, 0], vp[g, :, 1]
                    parts = abs(scale) * np.abs(qq).sum() * (np.abs(km) + 15 * np.abs(ks)).max()
                    ds = dim * 2.0 ** -24 * parts + 2.0 ** -19
                    size = p @ (np.abs(vm) + 8 * np.abs(vs))
                    tol[b, n, h] = (eps / 2 * np.abs(out[b, n, h]) + size * (2.0 ** -12 + 2 * ds)
                                    + 8 * np.abs(vs).max() * len(seen) * 2.0 ** -25 / w.sum())
                    tol_lse[b, n, h] = ds + 2.0 ** -21 * abs(lse[b, n, h])
    return out, lse, tol, tol_lse


# ---------------------------------------------------------------- the move of accepted rows
def move(pages, table, prefix_len, nodes, accept_len, dim, ps):
    """pages [layers, n, heads, block] after the move, one row after the other."""
    pages = pages.copy()
    half = ps * dim // 2
    B, gamma = accept_len.shape[0], nodes.shape[1] - 1
    n_pages = pages.shape[1]

    def place(b, pos):
        j = pos // ps
        if j >= table.shape[1] or not 0 <= int(table[b, j]) < n_pages:
            return None
        return int(table[b, j]), pos % ps

    for b in range(B):
        if int(prefix_len[b]) < 0:
            continue
        for i in range(min(max(int(accept_len[b]), 0), gamma)):
            nd = int(nodes[b, i])
            if nd <= i + 1:
                continue
            src, dst = place(b, int(prefix_len[b]) + nd), place(b, int(prefix_len[b]) + 1 + i)
            if src is None or dst is None:
                continue
            for at, pitch in ((0, dim // 2), (half, dim // 2), (2 * half, 4), (2 * half + 4 * ps, 4)):
                pages[:, dst[0], :, at + dst[1] * pitch:at + (dst[1] + 1) * pitch] = \
                    pages[:, src[0], :, at + src[1] * pitch:at + (src[1] + 1) * pitch]
    return pages
