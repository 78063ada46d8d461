"""Plain statements, in 64 bits, of the operators around the decoding step (test infrastructure).

Written from the formulas, one row or token at a time; numpy only.
"""
import numpy as np


def ancestors(parent):
    """seen[u, v]: node v is u or lies above it."""
    n = len(parent)
    seen = np.zeros((n, n), bool)
    for u in range(n):
        v = u
        while v >= 0:
            seen[u, v] = True
            v = parent[v]
    return seen


def attention(q, k, v, cache_k, cache_v, table, length, seen, scale, tree_tokens=None):
    """q [B,N,Hq,D], k/v [B,N,Hkv,D], caches [pages,Hkv,page,D], seen [N,N] or [B,N,N] -> (out, lse, weight, reach).

    weight = sum of p_i |v_i| (what a relative error of the p_i is worth), reach = the largest scale * sum |q||k| of a
    row: the two magnitudes that rounding errors of a kernel are measured in.  spread = sum |v_i| over visible keys."""
    B, N, Hq, D = q.shape
    Hkv, page = k.shape[2], cache_k.shape[2]
    out = np.zeros((B, N, Hq, D))
    lse = np.full((B, N, Hq), -np.inf)
    weight, spread, reach = np.zeros((B, N, Hq, D)), np.zeros((B, N, Hq, D)), np.zeros((B, N, Hq))
    for b in range(B):
        n = int(min(max(length[b], 0), table.shape[1] * page))
        pos = np.arange(n)
        ids = table[b, pos // page] if n else np.zeros(0, np.int64)
        ok = (ids >= 0) & (ids < cache_k.shape[0])
        for g in range(Hkv):
            past = [np.where(ok[:, None], c[np.where(ok, ids, 0), g, pos % page].astype(np.float64), 0.0) for c in (cache_k, cache_v)]
            for u in range(N):
                if tree_tokens is not None and tree_tokens[b, u] < 0:
                    continue
                row = (seen if seen.ndim == 2 else seen[b])[u].copy()
                row[u + 1:] = False
                nodes = np.flatnonzero(row)
                keys = np.concatenate([past[0], k[b, nodes, g].astype(np.float64)])
                vals = np.concatenate([past[1], v[b, nodes, g].astype(np.float64)])
                if len(keys) == 0:
                    continue
                for h in range(g * (Hq // Hkv), (g + 1) * (Hq // Hkv)):
                    x = q[b, u, h].astype(np.float64)
                    s = scale * (keys @ x)
                    top = s.max()
                    w = np.exp(s - top)
                    lse[b, u, h] = top + np.log(w.sum())
                    p = w / w.sum()
                    out[b, u, h] = (p[:, None] * vals).sum(0)
                    weight[b, u, h] = (p[:, None] * np.abs(vals)).sum(0)
                    spread[b, u, h] = np.abs(vals).sum(0)
                    reach[b, u, h] = scale * (np.abs(keys) @ np.abs(x)).max()
    return out, lse, weight, spread, reach


def page_map(length, new, width, page, table, free, n_free):
    """Serial statement of the page map: returns (slots, granted, length, n_free, table)."""
    B, cols = table.shape
    table = table.copy()
    slots, granted, out_len = np.full((B, width), -1, np.int64), np.full(B, -1, np.int32), length.copy()
    asked, taken = 0, 0
    for b in range(B):
        n, m = int(length[b]), int(new[b])
        if n < 0 or m < 0 or m > width or -(-(n + m) // page) > cols:
            continue
        have, want = -(-n // page), -(-(n + m) // page)
        asked += want - have
        if want > have and asked > n_free:
            continue
        for c in range(have, want):
            table[b, c] = free[n_free - 1 - (asked - (want - have)) - (c - have)]
        if want > have:
            taken = asked
        granted[b], out_len[b] = m, n + m
        for j in range(m):
            slots[b, j] = int(table[b, (n + j) // page]) * page + (n + j) % page
    return slots, granted, out_len, n_free - taken, table


def page_release(length, done, page, table, free, n_free):
    free, out_len = free.copy(), length.copy()
    for b in range(len(length)):
        if done[b]:
            for c in range(-(-max(int(length[b]), 0) // page)):
                free[n_free] = table[b, c]
                n_free += 1
            out_len[b] = 0
    return free, out_len, n_free


def kv_commit(src, path, slots, cache):
    """src [L,B,N,H,D], cache [L,pages,H,page,D] (changed in place)."""
    page = cache.shape[3]
    for b in range(slots.shape[0]):
        for j in range(slots.shape[1]):
            node = j if path is None else int(path[b, j])
            s = int(slots[b, j])
            if 0 <= s < cache.shape[1] * page and 0 <= node < src.shape[2]:
                cache[:, s // page, :, s % page] = src[:, b, node]
    return cache


def process_logits(x, parent, text=None, n_text=None, n_prompt=None, tree=None, repetition=None, frequency=None, presence=None,
                   bias=None, allowed=None, mask_row=None):
    """x [B,N,V] float64; bias: per sequence a list of (token, value); allowed [masks, V] -> (out, size): size is the
    largest magnitude met on the way to each logit."""
    B, N, V = x.shape
    out, size = x.astype(np.float64).copy(), np.abs(np.where(np.isfinite(x), x, 0.0))
    for b in range(B):
        for u in range(N):
            way, at = [], u
            while at > 0 and tree is not None:
                way.append(int(tree[b, at]))
                at = int(parent[at])
            said = [] if text is None else [int(t) for t in text[b, : int(n_text[b])]]
            start = 0 if n_prompt is None else int(n_prompt[b])
            count, met = {}, set()
            for t in said[start:] + way:
                count[t] = count.get(t, 0) + 1
            met.update(said + way)
            row = out[b, u]
            r, f, p = (1.0 if repetition is None else float(repetition[b]), 0.0 if frequency is None else float(frequency[b]),
                       0.0 if presence is None else float(presence[b]))
            for t in met:
                if 0 <= t < V:
                    row[t] = row[t] / r if row[t] > 0 else row[t] * r
                    c = count.get(t, 0)
                    size[b, u, t] = max(size[b, u, t] * max(r, 1 / r), abs(f) * c, abs(p))
                    if c:
                        row[t] -= f * c + p
            if bias is not None:
                for t, value in dict(bias[b]).items():
                    if 0 <= t < V:
                        row[t] += value
                        size[b, u, t] = max(size[b, u, t], abs(value) if np.isfinite(value) else 0.0)
            if mask_row is not None and 0 <= mask_row[b, u] < len(allowed):
                row[~allowed[mask_row[b, u]]] = -np.inf
    return out, size
