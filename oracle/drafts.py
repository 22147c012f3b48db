"""Trees of drafted tokens, windows with a few first tokens, page tables and the move of accepted drafts.

TEST INFRASTRUCTURE ONLY (see the package docstring).

Plain loops.  The cache, packed rows and pages are as in oracle/paged.py; the drafts of sequence b are
its last n = cu[b + 1] - cu[b] tokens, draft i at the place base + i, base = lens[b] - n.
"""

import math

import numpy as np

from .paged import D, _values, page_of

MOST = 2 ** 31 - 1


def in_window(t, p, window, sinks):
    """Whether a token at position p may see the key at position t <= p."""
    return window == 0 or t > p - window or (sinks > 0 and t < sinks)  # (drafts without a place have t < 0)


def tree_mask(parents, cu, lens=None, window=0, sinks=0, words=1):
    """(sees: for each row the set of drafts, depth [T], rows: which belong to a sequence)."""
    T = len(parents)
    sees, depth, rows = [set() for _ in range(T)], np.zeros(T, dtype=np.int64), np.zeros(T, dtype=bool)
    for b in range(len(cu) - 1):
        n = int(cu[b + 1]) - int(cu[b])
        base = (int(lens[b]) if lens is not None else 0) - n
        for i in range(n):
            t = int(cu[b]) + i
            way, j = [], i
            while True:
                way.append(j)
                p = int(parents[int(cu[b]) + j])
                if not 0 <= p < j:
                    break
                j = p
            way.reverse()
            depth[t], rows[t] = len(way) - 1, True
            sees[t] = {j for d, j in enumerate(way) if in_window(base + d, base + len(way) - 1, window, sinks) and j < 32 * words}
    return sees, depth, rows


def words_of(sees, words):
    """Mask words of sets of drafts, int32 [T, words]."""
    out = np.zeros((len(sees), words), dtype=np.uint32)
    for t, s in enumerate(sees):
        for j in s:
            out[t, j // 32] |= np.uint32(1 << (j % 32))
    return out.view(np.int32)


def seen_keys(i, n, length, max_len, sees, depth, window, sinks):
    """Places of the tokens that row i of n sees: sees: its drafts as a set, or None for a chain."""
    base = length - n
    keys = []
    for t in range(min(length, max_len)):
        if sees is None:
            if t <= base + i and in_window(t, base + i, window, sinks):
                keys.append(t)
        elif t < base:
            if in_window(t, base + depth, window, sinks):
                keys.append(t)
        elif t - base in sees:
            keys.append(t)
    return keys


def attn_tree(q, cache, cu, lens, table, max_len, sees=None, depth=None, window=0, sinks=0, scale=None):
    """(out fp64 [T, Hq, 128], weight: sum p (|va c| + |vb|) of each, rows: which are written)."""
    T, Hq = q.shape[:2]
    pages, H, page, _ = cache["k_q"].shape
    group = Hq // H
    scale = 1 / math.sqrt(D) if scale is None else scale
    out, weight, rows = np.zeros((T, Hq, D)), np.zeros((T, Hq, D)), np.zeros(T, dtype=bool)
    for b in range(len(lens)):
        n, length = int(cu[b + 1]) - int(cu[b]), max(int(lens[b]), 0)
        there, parts = [], []
        for t in range(min(length, max_len)):
            where = page_of(table, b, t, page, pages)
            there.append(where >= 0)
            parts.append([np.stack(np.broadcast_arrays(*_values(cache, s, max(where, 0), t % page))) for s in (0, 1)])
        if parts:
            parts = np.array(parts)  # [token, key or value, alpha c or beta, head, 128]
        for i in range(n):
            t = int(cu[b]) + i
            if length - n + i < 0:
                continue
            rows[t] = True
            keys = [x for x in seen_keys(i, n, length, max_len, None if sees is None else sees[t], i if depth is None else int(depth[t]),
                                         window, sinks) if there[x]]
            if not keys:
                continue
            seen = parts[keys]
            for g in range(H):
                heads = slice(g * group, (g + 1) * group)
                with np.errstate(invalid="ignore"):
                    s = q[t, heads].astype(np.float64) @ seen[:, 0, :, g].sum(1).T * scale
                    p = np.exp(s - s.max(-1, keepdims=True))
                    p /= p.sum(-1, keepdims=True)
                    out[t, heads] = p @ seen[:, 1, :, g].sum(1)
                    weight[t, heads] = p @ np.abs(seen[:, 1, :, g]).sum(1)
    return out, weight, rows


def attn_paged_window(q, cache, lens, table, max_len, window, sinks, scale=None):
    """One token a sequence; a sequence without tokens gets zeros."""
    out, weight, _ = attn_tree(q, cache, np.arange(len(lens) + 1), lens, table, max_len, window=window, sinks=sinks, scale=scale)
    return out, weight


def attn_prompt_window(q, k, v, cu_q, cu_k, window, sinks, scale=None):
    """(out fp64 [Tq, Hq, 128], weight: sum p |v|, rows: which belong to a sequence)."""
    Tq, Hq = q.shape[:2]
    H = k.shape[1]
    scale = 1 / math.sqrt(D) if scale is None else scale
    out, weight, rows = np.zeros((Tq, Hq, D)), np.zeros((Tq, Hq, D)), np.zeros(Tq, dtype=bool)
    for b in range(len(cu_q) - 1):
        q0, k0, n, m = int(cu_q[b]), int(cu_k[b]), int(cu_q[b + 1] - cu_q[b]), int(cu_k[b + 1] - cu_k[b])
        rows[q0:q0 + n] = True
        for i in range(n):
            p = m - n + i
            keys = [k0 + t for t in range(p + 1) if in_window(t, p, window, sinks)]
            if not keys:
                continue
            for g in range(H):
                heads = slice(g * (Hq // H), (g + 1) * (Hq // H))
                K, V = k[keys, g].astype(np.float64), v[keys, g].astype(np.float64)
                with np.errstate(invalid="ignore"):
                    s = q[q0 + i, heads].astype(np.float64) @ K.T * scale
                    w = np.exp(s - s.max(-1, keepdims=True))
                    w /= w.sum(-1, keepdims=True)
                    out[q0 + i, heads], weight[q0 + i, heads] = w @ V, w @ np.abs(V)
    return out, weight, rows


def paged_release(table, page, first, end, held, pool, count):
    """(table, held, pool, count) after it."""
    table, held, pool = np.array(table), [int(x) for x in held], list(pool)
    pages, cols = len(pool), table.shape[1]
    count = min(max(int(count), 0), pages)
    for b in range(len(held)):
        have = min(max(held[b], 0), cols)
        c0 = min(-(-max(int(first[b]), 0) // page), have)
        last = int(end[b]) >= have * page
        c1 = have if last else max(int(end[b]), 0) // page
        for c in range(c0, c1):
            p, table[b, c] = int(table[b, c]), -1
            if 0 <= p < pages:
                if count < pages:
                    pool[count] = p
                count = min(count + 1, pages)
        held[b] = c0 if last else have
    return table, held, pool, count


def paged_grow(have, add, held, table, page, pool, count, rows):
    """dict of lens, cu, pos, slots, missing, table, held, count."""
    table, held, pages, cols = np.array(table), [int(x) for x in held], len(pool), np.array(table).shape[1]
    count = min(max(int(count), 0), pages)
    B = len(held)
    had = [max(int(x), 0) for x in have]
    lens = [min(h + max(int(a), 0), MOST) for h, a in zip(had, add)]
    upto = [-(-n // page) for n in lens]
    kept = [min(max(h, 0), cols) for h in held]
    need = [max(min(u, cols) - h, 0) for u, h in zip(upto, kept)]
    new = [n - h for n, h in zip(lens, had)]
    missing = (min(max(sum(need) - count, 0) + sum(max(u - cols, 0) for u in upto), MOST), min(max(sum(new) - rows, 0), MOST))
    pos, slots = np.full(rows, -1, dtype=np.int64), np.full(rows, -1, dtype=np.int64)
    if missing != (0, 0):
        return dict(lens=had, cu=[0] * (B + 1), pos=pos, slots=slots, missing=missing, table=table, held=held, count=count)
    cu, t = [0], 0
    for b in range(B):
        for c in range(kept[b], kept[b] + need[b]):
            count -= 1
            table[b, c] = pool[count]
        for p in range(had[b], lens[b]):
            pos[t] = p
            e = page_of(table, b, p, page, pages)
            slots[t] = e * page + p % page if e >= 0 else -1
            t += 1
        cu.append(t)
    return dict(lens=lens, cu=cu, pos=pos, slots=slots, missing=missing, table=table, held=[k + n for k, n in zip(kept, need)], count=count)


def kv_keep(cache, cu, lens, table, path, kept):
    """(cache after it, lens)."""
    pages, _, page, _ = cache["k_q"].shape
    out, lens_out = {n: a.copy() for n, a in cache.items()}, []
    for b in range(len(lens)):
        n = max(int(cu[b + 1]) - int(cu[b]), 0)
        base = int(lens[b]) - n
        count = min(max(int(kept[b]), 0), path.shape[1], n)
        for i in range(count):
            j = int(path[b, i])
            if not i <= j < n:
                continue
            src, dst = (page_of(table, b, base + x, page, pages) for x in (j, i))
            if src >= 0 and dst >= 0:
                for name in out:
                    out[name][dst, :, (base + i) % page] = cache[name][src, :, (base + j) % page]
        lens_out.append(max(base + count, 0))
    return out, lens_out
