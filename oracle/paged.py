"""The paged 4- or 8-bit K/V cache: positions, the quantized write, reading back, and attention.

TEST INFRASTRUCTURE ONLY (see the package docstring).

Plain loops in fp64 (fp32 where eq. 1's encoding is defined in it).  Shapes: q [T, Hq, 128],
k, v [T, Hkv, 128]; a cache is a dict of k_q, v_q uint8 [pages, Hkv, page, 64 or 128] and params
[pages, Hkv, page, 4] (k_alpha, k_beta, v_alpha, v_beta), fp32 or fp16.  Row t of a packed call is
one of the last tokens of the sequence b with cu[b] <= t < cu[b + 1]: position
lens[b] - cu[b + 1] + t.  A row of no sequence, or with a negative position, is left alone; a
position without a page in the pool is not written, reads as zeros and takes no part in attention.
"""

import math

import numpy as np

from .quant import quant_asym, store_codes, unpack_nibbles
from .rotate import rotate_rows

D = 128


def rope_frequencies(rotary, theta, scaling="none", factor=1.0, low=1.0, high=4.0, original_len=8192.0):
    f = np.array([theta ** (-2.0 * i / rotary) for i in range(rotary // 2)])
    if scaling == "linear":
        return f / factor
    if scaling == "by parts":
        kept = np.clip((original_len * f / (2 * math.pi) - low) / (high - low), 0.0, 1.0)
        return f * kept + f / factor * (1 - kept)
    return f


def rope(x, pos, freq, interleaved=False, magnitude=1.0):
    """x [T, H, 128] at positions pos [T], fp64: the first 2 len(freq) dims turn."""
    y = np.array(x, dtype=np.float64)
    if freq is None or len(freq) == 0:
        return y
    r = 2 * len(freq)
    for t, p in enumerate(pos):
        c, s = magnitude * np.cos(p * freq), magnitude * np.sin(p * freq)
        u, w = (y[t, :, 0:r:2].copy(), y[t, :, 1:r:2].copy()) if interleaved else (y[t, :, :r // 2].copy(), y[t, :, r // 2:r].copy())
        a, b = u * c - w * s, w * c + u * s
        if interleaved:
            y[t, :, 0:r:2], y[t, :, 1:r:2] = a, b
        else:
            y[t, :, :r // 2], y[t, :, r // 2:r] = a, b
    return y


def page_of(table, b, pos, page, pages):
    col = pos // page
    if pos < 0 or col >= table.shape[1]:
        return -1
    e = int(table[b, col])
    return e if 0 <= e < pages else -1


def places(T, cu, lens, table, page, pages):
    """(position, page) of each row; position -1: left alone, page -1: not in the pool."""
    pos, where = np.full(T, -1, dtype=np.int64), np.full(T, -1, dtype=np.int64)
    for b in range(len(lens)):
        for t in range(int(cu[b]), min(int(cu[b + 1]), T)):
            p = int(lens[b]) - int(cu[b + 1]) + t
            if p >= 0:
                pos[t], where[t] = p, page_of(table, b, p, page, pages)
    return pos, where


def rope_kv_write(q, k, v, cache, cu, lens, table, freq, interleaved=False, magnitude=1.0, k_clip=1.0, v_clip=1.0):
    """Returns dict(q_rot, k_rot fp64; rows: which are written; k_q, v_q, params: the cache after;
    k_codes, v_codes, k32: codes and quantizer input of each row)."""
    T = q.shape[0]
    pages, _, page, row = cache["k_q"].shape
    bits = row // 16
    pos, where = places(T, cu, lens, table, page, pages)
    live = pos >= 0
    p0 = np.where(live, pos, 0)
    turned = [rotate_rows(rope(x, p0, freq, interleaved, magnitude), None, D) for x in (q, k)]
    fp16 = cache["params"].dtype == np.float16
    k32 = turned[1].astype(np.float32)
    kc, ka, kb = quant_asym(k32, bits=bits, group=D, clip=k_clip, param_fp16=fp16)
    vc, va, vb = quant_asym(np.asarray(v, dtype=np.float32), bits=bits, group=D, clip=v_clip, param_fp16=fp16)
    out = {n: a.copy() for n, a in cache.items()}
    for t in range(T):
        if live[t] and where[t] >= 0:
            at = (where[t], slice(None), pos[t] % page)
            out["k_q"][at], out["v_q"][at] = store_codes(kc[t], bits), store_codes(vc[t], bits)
            out["params"][at] = np.concatenate([ka[t], kb[t], va[t], vb[t]], axis=-1)
    return dict(out, q_rot=turned[0], k_rot=turned[1], rows=live, where=where, pos=pos, k_codes=kc, v_codes=vc, k32=k32)


def _values(cache, which, page, off):
    """fp64 [Hkv, 128] of one slot, and the parts alpha c and beta."""
    codes = cache["k_q" if which == 0 else "v_q"][page, :, off]
    c = unpack_nibbles(codes, signed=False) if codes.shape[-1] == D // 2 else codes.astype(np.int64)
    p = cache["params"][page, :, off].astype(np.float64)
    return p[:, 2 * which, None] * c, p[:, 2 * which + 1, None]


def kv_read(cache, cu, lens, table, T, plain_basis=False):
    """(k, v fp64 [T, Hkv, 128], rows: which are written)."""
    pages, H, page, _ = cache["k_q"].shape
    pos, where = places(T, cu, lens, table, page, pages)
    k, v = np.zeros((T, H, D)), np.zeros((T, H, D))
    for t in range(T):
        if where[t] >= 0:
            for out, i in ((k, 0), (v, 1)):
                a, b = _values(cache, i, where[t], pos[t] % page)
                out[t] = a + b
    if plain_basis:
        k = rotate_rows(k, None, D)
    return k, v, pos >= 0


def attn_paged(q, cache, lens, table, max_len, scale=None):
    """(out fp64 [B, Hq, 128], weight: sum_t p (|va c| + |vb|) of each, for tolerances)."""
    B, Hq = q.shape[:2]
    pages, H, page, _ = cache["k_q"].shape
    scale = 1 / math.sqrt(D) if scale is None else scale
    out, weight = np.zeros((B, Hq, D)), np.zeros((B, Hq, D))
    for b in range(B):
        n = min(max(int(lens[b]), 0), max_len)
        at = [(page_of(table, b, t, page, pages), t % page) for t in range(n)]
        at = [x for x in at if x[0] >= 0]
        if not at:
            continue
        ks, vs = ([_values(cache, i, *x) for x in at] for i in (0, 1))
        for h in range(Hq):
            g = h // (Hq // H)
            K = np.stack([a[g] + c[g] for a, c in ks])
            s = K @ q[b, h].astype(np.float64) * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            va, vb = np.stack([a[g] for a, _ in vs]), np.stack([c[g] for _, c in vs])
            out[b, h] = p @ (va + vb)
            weight[b, h] = p @ (np.abs(va) + np.abs(vb))
    return out, weight


def attn_prompt(q, k, v, cu_q, cu_k, scale=None, causal=True):
    """(out fp64 [Tq, Hq, 128], weight: sum_t p |v|, rows: which belong to a sequence)."""
    Tq, Hq = q.shape[:2]
    H = k.shape[1]
    scale = 1 / math.sqrt(D) if scale is None else scale
    out, weight, rows = np.zeros((Tq, Hq, D)), np.zeros((Tq, Hq, D)), np.zeros(Tq, dtype=bool)
    for b in range(len(cu_q) - 1):
        q0, q1, k0, k1 = int(cu_q[b]), int(cu_q[b + 1]), int(cu_k[b]), int(cu_k[b + 1])
        n, m = q1 - q0, k1 - k0
        rows[q0:q1] = True
        for i in range(n):
            see = min(m, m - n + i + 1) if causal else m
            if see <= 0:
                continue
            for h in range(Hq):
                g = h // (Hq // H)
                K, V = k[k0:k0 + see, g].astype(np.float64), v[k0:k0 + see, g].astype(np.float64)
                s = K @ q[q0 + i, h].astype(np.float64) * scale
                p = np.exp(s - s.max())
                p /= p.sum()
                out[q0 + i, h], weight[q0 + i, h] = p @ V, p @ np.abs(V)
    return out, weight, rows
