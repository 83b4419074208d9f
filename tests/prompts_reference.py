"""Plain NumPy statements, in 64 bits, of the operators of prompts and long conversations: attention of a chunk, the
weight that rows gather, eviction, log probabilities.  Nothing is shared with the package but the documented memory layout."""
import numpy as np

import ops_reference as ops


def sequences(start, cu, n_tokens, max_new):
    """(sequence, first row, count) of the sequences that have new tokens."""
    got = []
    for b in range(len(start)):
        first = int(cu[b])
        n = min(int(cu[b + 1]) - first, max_new, n_tokens - first)
        if int(start[b]) >= 0 and first >= 0 and n > 0:
            got.append((b, first, n))
    return got


def cached(pages, table, b, length, dim, ps):
    """(positions that are there, keys, values, key and value (scale, mid)) of a sequence, arrays [kv, positions, ..]."""
    n_pages = pages.shape[0]
    there = [p for p in range(min(length, table.shape[1] * ps)) if 0 <= int(table[b, p // ps]) < n_pages]
    rows = [ops.row_values(pages, int(table[b, p // ps]), p % ps, dim, ps) for p in there]
    kv = pages.shape[1]
    K, V, KP, VP = (np.stack([r[i] for r in rows], 1) if rows else np.zeros((kv, 0, dim if i < 2 else 2)) for i in range(4))
    return np.array(there, dtype=np.int64), K, V, KP, VP


def score_slack(q, kp, scale):
    """What float32 may do to a score: D products of a query with codes from 0 to 15 and the row's scale and mid summed in
    float32 (D 2^-24 of the sum of magnitudes), and a few roundings of the result (2^-19)."""
    parts = abs(scale) * np.abs(q).sum(-1, keepdims=True) * (np.abs(kp[:, 1]) + 15 * np.abs(kp[:, 0]))
    return q.shape[-1] * 2.0 ** -24 * parts + 2.0 ** -19


def chunk_attention(q, pages, table, start, cu, max_new, dim, ps, scale, eps):
    """(out, lse, tolerance of out, tolerance of lse); rows of no token are NaN with tolerance 0.

    The tolerance counts, per output: the final rounding (eps / 2, or 2^-25 where that is more and the type is half: its numbers below
    2^-14 are the multiples of 2^-24, so the nearest is up to 2^-25 away; bf16 has no such border above 2^-126); weights and values rounded to half precision (2^-11 of each, relative to
    what they are multiplied with; a weight that underflows is off by 2^-25 of the largest value scale); the scores' slack, twice,
    since a weight is a quotient of two exponentials."""
    T, H, _ = q.shape
    kv = pages.shape[1]
    out, lse = np.full(q.shape, np.nan), np.full((T, H), np.nan)
    tol, tol_lse = np.zeros(q.shape), np.zeros((T, H))
    for b, first, n in sequences(start, cu, T, max_new):
        at, K, V, KP, VP = cached(pages, table, b, int(start[b]) + n, dim, ps)
        seen = at[None, :] <= int(start[b]) + np.arange(n)[:, None]
        for h in range(H):
            g = h // (H // kv)
            qq = q[first:first + n, h].astype(np.float64)
            with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
                s = np.where(seen, scale * np.where(seen, qq @ np.where(np.isfinite(K[g]), K[g], 0).T, 0), -np.inf)
                bad_k, bad_v = ~np.isfinite(K[g]).all(-1), ~np.isfinite(V[g]).all(-1)
                s[:, bad_k] = np.where(seen[:, bad_k], np.nan, -np.inf)
                empty = ~seen.any(1)
                top = np.where(empty, 0.0, np.max(s, 1, initial=-np.inf))
                w = np.exp(s - top[:, None])
                total = w.sum(1)
                p = w / np.where(total == 0, 1.0, total)[:, None]
                o = p @ np.where(np.isfinite(V[g]), V[g], 0)
                o[(seen & bad_v).any(1)] = np.nan
                out[first:first + n, h] = o
                lse[first:first + n, h] = np.where(empty, -np.inf, top + np.log(total))
                kp, vp = np.nan_to_num(KP[g]), np.nan_to_num(VP[g])
                slack = score_slack(qq, kp, scale)
                ds = np.where(seen, slack, 0).max(1, initial=0.0)
                size = np.nan_to_num(p) @ (np.abs(vp[:, 1]) + 8 * np.abs(vp[:, 0]))
                loud = 8 * np.where(seen, np.abs(vp[:, 0]), 0).max(1, initial=0.0)
                floor = loud * seen.sum(1) * 2.0 ** -25 / np.where(total > 0, total, 1)
                last = np.maximum(eps / 2 * np.abs(o), 2.0 ** -25 if eps == 2.0 ** -10 else 0.0)
                tol[first:first + n, h] = last + (size * (2.0 ** -10 + 2 * ds) + floor)[:, None]
                tol_lse[first:first + n, h] = ds + 2.0 ** -21 * np.abs(np.where(empty, 0, lse[first:first + n, h]))
    return out, lse, tol, tol_lse


def accumulate(q, lse, pages, weights, table, start, cu, max_new, dim, ps, scale, decay, last):
    """(weights afterwards, tolerance): every term carries its score's slack and a few float32 roundings, the sum another 2^-20."""
    weights = weights.astype(np.float64).copy()
    tol = np.zeros_like(weights)
    T, H, _ = q.shape
    kv = pages.shape[1]
    for b, first, n in sequences(start, cu, T, max_new):
        at, K, _, KP, _ = cached(pages, table, b, int(start[b]) + n, dim, ps)
        page, row = table[b, at // ps], at % ps
        i = np.arange(max(0, n - last) if last else 0, n)
        seen = at[None, :] <= int(start[b]) + i[:, None]
        for g in range(kv):
            got, off = np.zeros(len(at)), np.zeros(len(at))
            for h in range(g * (H // kv), (g + 1) * (H // kv)):
                qq, l = q[first + i, h].astype(np.float64), lse[first + i, h].astype(np.float64)
                with np.errstate(invalid="ignore", over="ignore"):
                    p = np.where(seen & (l != -np.inf)[:, None], np.exp(scale * (qq @ K[g].T) - l[:, None]), 0.0)
                    slack = score_slack(qq, np.nan_to_num(KP[g]), scale) + 2.0 ** -21 * np.abs(np.where(np.isfinite(l), l, 0))[:, None]
                    got += p.sum(0)
                    off += (np.nan_to_num(p) * slack).sum(0)
            old = np.where((at < int(start[b])) & (decay != 0), decay * weights[page, g, row], 0.0)
            weights[page, g, row] = old + got
            tol[page, g, row] = off + 2.0 ** -20 * (np.abs(old) + np.abs(got))
    return weights, tol


def evict(pages, weights, table, length, keep, sink, recent, dim, ps):
    """(pages [layers, n, heads, block], weights [layers, n, heads, ps], lengths) afterwards, row by row; keep [B]."""
    pages, weights, out = pages.copy(), weights.copy(), np.asarray(length).copy()
    L, n_pages, heads, _ = pages.shape
    half = ps * dim // 2
    for b in range(len(length)):
        n = min(int(length[b]), table.shape[1] * ps)
        k = int(keep[b])
        if int(length[b]) < 0 or k < 0 or n <= k:
            continue
        out[b] = k
        s = min(sink, k)
        r = min(recent, k - s)
        at = [int(table[b, p // ps]) if 0 <= int(table[b, p // ps]) < n_pages else None for p in range(n)]
        for l in range(L):
            for h in range(heads):
                def weight(p):
                    w = np.nan if at[p] is None else weights[l, at[p], h, p % ps]
                    return (0, 0.0) if np.isnan(w) else (1, float(w))
                middle = sorted(range(s, n - r), key=lambda p: (-weight(p)[0], -weight(p)[1], p))[:k - s - r]
                rows = list(range(s)) + sorted(middle) + list(range(n - r, n))
                for dst, src in enumerate(rows):
                    if dst == src or at[src] is None or at[dst] is None:
                        continue
                    for x, pitch in ((0, dim // 2), (half, dim // 2), (2 * half, 4), (2 * half + 4 * ps, 4)):
                        pages[l, at[dst], h, x + dst % ps * pitch:x + (dst % ps + 1) * pitch] = \
                            pages[l, at[src], h, x + src % ps * pitch:x + (src % ps + 1) * pitch]
                    weights[l, at[dst], h, dst % ps] = weights[l, at[src], h, src % ps]
    return pages, weights, out


def logprobs(row, tokens, temperature, n_top):
    """(log probabilities, entropy, top ids, their log probabilities) of one row of logits."""
    row = row.astype(np.float64)
    V = len(row)
    nan = float("nan")
    if np.isnan(row).any() or (row == np.inf).any() or (row == -np.inf).all():
        return np.full(len(tokens), nan), nan, np.full(n_top, -1), np.full(n_top, nan)
    s = row / temperature
    top = s.max()
    w = np.exp(s - top)
    x = s - top - np.log(w.sum())
    p = w / w.sum()
    entropy = -np.where(p > 0, p * np.where(p > 0, x, 0), 0).sum()
    given = np.array([x[t] if 0 <= t < V else nan for t in tokens])
    ids = np.lexsort((np.arange(V), -row))[:n_top]
    return given, entropy, ids, x[ids]
