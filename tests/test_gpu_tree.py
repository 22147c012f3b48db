"""Trees of drafts over the pages, windows with a few first tokens, on the GPU against oracle/drafts.py.

Tolerances as in tests/test_gpu_paged.py: weights and outputs rounded to fp16 (2^-11 each of sum p |v| and of the
value, 2^-25 below), 32-bit scores (2e-5 of the weights).  Masks, depths and moved bytes are whole numbers.
"""

import numpy as np
import pytest
import torch

from oracle import drafts as od
from oracle import paged as opg
from paper_2405_16406_amd import sq
from test_gpu_paged import DEV, attention_close, check_write, device_cache, f64, filled, heads_of, ints, rng, spread_table, up

pytestmark = pytest.mark.gpu


def tree(g, n, near=8):
    """A parent before each draft, or -1."""
    return [int(g.integers(max(-1, i - near), i)) for i in range(n)]


def packed(counts, before=0):
    return np.concatenate([[before], before + np.cumsum(counts)])


TREES = [  # drafts of each sequence, tokens before them, window, sinks, words beside the least
    ([1], [0], 0, 0, 0),
    ([5, 0, 33, 64], [11, 3, 100, 0], 0, 0, 0),
    ([16, 7], [300, 2], 5, 0, 1),
    ([40], [1], 3, 8, 0),
    ([70, 2, 129], [9, 50, 1000], 4, 2, 2),
    ([1] * 70, list(range(70)), 0, 0, 0),
    ([300], [7], 0, 0, 0),
]


@pytest.mark.parametrize("case", TREES, ids=lambda c: f"{len(c[0])}x{max(c[0])}-w{c[2]}-s{c[3]}")
def test_tree_mask(case):
    counts, before, window, sinks, more = case
    g = rng(sum(counts))
    cu = packed(counts, 2)
    T = int(cu[-1]) + 3
    parents = np.concatenate([[9, 9]] + [tree(g, n) for n in counts] + [[9] * 3]).astype(np.int64)
    lens = [n + b for n, b in zip(counts, before)]
    words = -(-max(counts) // 32) + more
    sees, depth, rows = od.tree_mask(parents, cu, lens, window, sinks, words)
    wide = torch.full((T, words + 3), 7, dtype=torch.int32, device=DEV)
    out = wide[:, 1:1 + words], torch.full((T,), 7, dtype=torch.int32, device=DEV)
    sq.tree_mask(ints(parents), ints(cu), 0, ints(lens) if window and sinks else None, window, sinks, out=out)
    got = out[0].cpu().numpy()
    assert np.array_equal(got[rows], od.words_of(sees, words)[rows])
    assert np.array_equal(out[1].cpu().numpy()[rows], depth[rows])
    assert np.all(got[~rows] == 7) and np.all(out[1].cpu().numpy()[~rows] == 7) and torch.all(wide[:, 0] == 7) and torch.all(wide[:, 1 + words:] == 7)


def test_tree_mask_of_bad_parents_and_few_words():
    """A parent that is not before its draft makes a root; drafts past the words have no bits."""
    parents = [5, 1, 0, -7, 3, 2 ** 31 - 1, 5] + [i - 1 for i in range(7, 80)]
    sees, depth, _ = od.tree_mask(parents, [0, 80], words=1)
    mask, d = sq.tree_mask(ints(parents), ints([0, 80]), 32)
    assert mask.shape == (80, 1)
    assert np.array_equal(mask.cpu().numpy(), od.words_of(sees, 1)) and np.array_equal(d.cpu().numpy(), depth)


def test_tree_mask_of_a_long_chain():
    """More drafts than the parents that lie near, one chain: the last word of each row."""
    n = 4200
    mask, depth = sq.tree_mask(ints(np.arange(n) - 1), ints([0, n]), n)
    assert np.array_equal(depth.cpu().numpy(), np.arange(n))
    bits = np.unpackbits(mask.cpu().numpy().view(np.uint8), axis=1, bitorder="little")[:, :n]
    assert np.array_equal(bits, np.tril(np.ones((n, n), dtype=np.uint8)))


def test_tree_mask_of_more_drafts_than_it_goes_up_from():
    """Drafts from 2^14 on have depth 0 and no bits; those before have all that there is."""
    n = (1 << 14) + 150
    mask, depth = sq.tree_mask(ints([-1] + [0] * 39 + [i - 1 for i in range(40, n)]), ints([0, n]), 64)
    want = np.minimum(np.arange(n), 1)
    want[40:] = np.arange(40, n) - 38
    want[1 << 14:] = 0
    assert np.array_equal(depth.cpu().numpy(), want)
    bits = np.unpackbits(mask.cpu().numpy().view(np.uint8), axis=1, bitorder="little")
    sees = np.zeros((n, 64), dtype=np.uint8)
    sees[:, 0] = sees[40:, 39] = 1
    for i in range(1, 39):
        sees[i, i] = 1
    sees[39, 39] = 1
    for i in range(40, n):
        sees[i, 40:min(i, 63) + 1] = 1
    sees[1 << 14:] = 0
    assert np.array_equal(bits, sees)
    with pytest.raises(sq.SqError):
        sq.tree_mask(ints([-1]), ints([0, 1]), (1 << 14) + 1)


WRITE = [  # Hq, Hkv, page, bits, params, rotary, interleaved, drafts, tokens before
    (8, 2, 16, 4, np.float32, 128, False, [5, 1, 40], [11, 0, 100]),
    (4, 4, 64, 8, np.float16, 96, True, [33], [70]),
    (32, 8, 16, 4, np.float32, 0, False, [7, 2], [3, 31]),
]


@pytest.mark.parametrize("case", WRITE, ids=lambda c: f"{c[0]}x{c[1]}-b{c[3]}-r{c[5]}")
def test_write_by_depth(case):
    """The write of a tree: each draft turned by its depth, at its own place."""
    Hq, H, page, bits, dt, rotary, inter, new, past = case
    g = rng(Hq + page)
    lens = [n + p for n, p in zip(new, past)]
    cu, T = packed(new, 1), sum(new) + 2
    depth = np.concatenate([[9]] + [od.tree_mask(tree(g, n), [0, n])[1] for n in new] + [[9]])
    table, pages = spread_table(g, lens, page)
    q, k, v = (heads_of(g, T, h) for h in (Hq, H, H))
    freq = opg.rope_frequencies(rotary, 10000.0) if rotary else None
    cache = filled(g, pages, H, page, bits, dt)
    o = opg.rope_kv_write(q, k, v, cache, cu, lens, table, None)  # places, and values' codes
    at = np.zeros(T, dtype=np.int64)
    for b, n in enumerate(new):
        at[cu[b]:cu[b + 1]] = past[b] + depth[cu[b]:cu[b + 1]]
    turned = [opg.rotate_rows(opg.rope(x, at, freq, inter), None, 128) for x in (q, k)]
    kc, ka, kb = opg.quant_asym(turned[1].astype(np.float32), bits=bits, group=128, clip=1.0, param_fp16=dt == np.float16)
    for t in np.nonzero(o["where"] >= 0)[0]:
        to = (o["where"][t], slice(None), o["pos"][t] % page)
        o["k_q"][to] = opg.store_codes(kc[t], bits)
        o["params"][to + (slice(0, 2),)] = np.concatenate([ka[t], kb[t]], axis=-1)
    o |= dict(q_rot=turned[0], k32=turned[1].astype(np.float32))
    dc = device_cache(cache)
    out = torch.full((T, Hq, 128), 7.0, dtype=torch.float16, device=DEV)
    sq.rope_kv_write(up(q), up(k), up(v), dc, ints(table), ints(lens), None if freq is None else up(freq), cu=ints(cu),
                     interleaved=inter, out=out, depth=ints(depth))
    torch.cuda.synchronize()
    check_write(o, out, dc, q, bits, o["rows"])
    assert torch.all(out[0] == 7.0) and torch.all(out[-1] == 7.0)


def test_write_of_a_chain_is_the_plain_one():
    """Depths that count up, without and with cu: bit for bit what the write does without them."""
    g = rng(3)
    new, lens, page = [9, 4], [500, 4], 16
    cu, T = packed(new), sum(new)
    table, pages = spread_table(g, lens, page)
    q, k, v = (up(heads_of(g, T, h)) for h in (8, 2, 2))
    freq = up(opg.rope_frequencies(128, 10000.0))
    cache = filled(g, pages, 2, page, 4, np.float32)
    a, b = device_cache(cache), device_cache(cache)
    qa = sq.rope_kv_write(q, k, v, a, ints(table), ints(lens), freq, cu=ints(cu))
    qb = sq.rope_kv_write(q, k, v, b, ints(table), ints(lens), freq, cu=ints(cu), depth=ints([*range(9), *range(4)]))
    assert torch.equal(qa, qb) and all(torch.equal(x, y) for x, y in zip(a, b))
    args = (q[:2], k[:2], v[:2])
    qa = sq.rope_kv_write(*args, a, ints(table), ints(lens), freq)
    qb = sq.rope_kv_write(*args, b, ints(table), ints(lens), freq, depth=ints([0, 0]))
    assert torch.equal(qa, qb) and all(torch.equal(x, y) for x, y in zip(a, b))


ATTN = [  # Hq, Hkv, page, bits, params, drafts, tokens before, window, sinks
    (4, 1, 16, 4, np.float32, [3, 1, 0, 2], [0, 17, 9, 60], 0, 0),         # one column of rows
    (8, 2, 16, 4, np.float32, [7, 5], [100, 250], 0, 0),                   # two
    (8, 2, 32, 4, np.float16, [16, 3, 33], [63, 64, 65], 0, 0),            # four, uneven
    (32, 32, 16, 8, np.float32, [7, 2], [130, 5], 0, 0),
    (64, 8, 64, 8, np.float16, [9, 1], [200, 0], 0, 0),
    (17, 1, 16, 4, np.float32, [4], [300], 0, 0),                          # rows across columns and tiles
    (8, 2, 16, 4, np.float32, [6, 12, 2], [500, 40, 3], 40, 4),
    (4, 4, 16, 8, np.float16, [40, 1], [700, 800], 100, 70),               # first tokens beyond a block
    (8, 1, 128, 4, np.float16, [9], [1000], 1, 0),
    (16, 2, 16, 4, np.float32, [70, 5], [90, 2000], 64, 16),
    (64, 8, 32, 4, np.float16, [32, 5, 17], [1500, 700, 64], 0, 0),        # two columns
    (32, 32, 16, 8, np.float32, [20, 33], [300, 1100], 0, 0),
    (64, 8, 16, 8, np.float16, [16, 7], [900, 600], 500, 20),
    (36, 12, 16, 4, np.float32, [11, 6, 23], [1200, 800, 5], 700, 3),      # rows across columns
    (8, 2, 16, 4, np.float32, [9], [7000], 0, 0),                          # many chunks
    (8, 2, 16, 4, np.float16, [6, 3], [600, 1000], 0, 0),                  # eight waves
    (16, 4, 32, 8, np.float32, [12, 2], [950, 300], 0, 0),
    (8, 1, 16, 4, np.float32, [20, 1], [1255, 0], 0, 0),
    (8, 2, 16, 8, np.float32, [5], [2500], 0, 0),                          # one column, a few chunks
    (8, 2, 32, 8, np.float16, [3, 8], [1700, 100], 0, 0),
    (8, 2, 16, 4, np.float16, [4, 1], [3000, 1500], 0, 0),
    (64, 8, 16, 8, np.float16, [33, 20], [900, 1400], 0, 0),               # two columns
]


def attn_case(case, bits=None):
    Hq, H, page, bits, dt, new, past, window, sinks = case
    g = rng(Hq * 7 + sum(new))
    lens = [n + p for n, p in zip(new, past)]
    cu, T = packed(new, 1), sum(new) + 3
    table, pages = spread_table(g, lens, page)
    cache = filled(g, pages, H, page, bits, dt)
    q = heads_of(g, T, Hq)
    parents = np.concatenate([[0]] + [tree(g, n) for n in new] + [[0, 0]]).astype(np.int64)
    return g, Hq, H, lens, cu, T, table, cache, q, parents, window, sinks


@pytest.mark.parametrize("chain", [False, True], ids=["tree", "chain"])
@pytest.mark.parametrize("case", ATTN, ids=lambda c: f"{c[0]}x{c[1]}-b{c[3]}-{np.dtype(c[4]).name}-{max(c[5])}of{max(c[6])}-w{c[7]}s{c[8]}")
def test_attn_tree(case, chain):
    g, Hq, H, lens, cu, T, table, cache, q, parents, window, sinks = attn_case(case)
    most = max(lens)
    words = -(-max(np.diff(cu)) // 32)
    sees, depth, rows = od.tree_mask(parents, cu, lens, window, sinks, words)
    args = {} if chain else dict(mask=up(od.words_of(sees, words)), depth=ints(depth))
    wide = torch.full((T, Hq + 1, 128), 7.0, dtype=torch.float16, device=DEV)
    sq.attn_tree(up(q), device_cache(cache), ints(table), ints(lens), ints(cu), most, window=window, sinks=sinks, out=wide[:, :Hq], **args)
    torch.cuda.synchronize()
    want, weight, rows = od.attn_tree(q, cache, cu, lens, table, most, None if chain else sees, None if chain else depth, window, sinks)
    attention_close(wide[:, :Hq][up(rows)], want[rows], weight[rows], 2e-5)
    assert torch.all(wide[:, :Hq][up(~rows)] == 7.0) and torch.all(wide[:, Hq:] == 7.0)


def test_rows_and_masks_at_their_ends():
    """Rows that see nothing, not themselves, later drafts, one draft in the last word; drafts beyond the words; rows
    without a place; a length beyond max_len; pages that are missing."""
    g = rng(11)
    Hq, H, page = 8, 2, 16
    new, lens = [40, 6, 5], [40, 4, 260]  # the second has two rows before its first token
    cu, T = packed(new), sum(new)
    table, pages = spread_table(g, lens, page)
    table[2, 3], table[2, 5] = -1, pages
    cache = filled(g, pages, H, page, 4, np.float32)
    q = heads_of(g, T, Hq)
    sees = [set(map(int, np.nonzero(g.random(40) < 0.3)[0])) for _ in range(T)]
    sees[0], sees[1], sees[2], sees[3] = set(), {31}, {32}, {39}
    for words in (1, 2):
        known = [{j for j in s if j < 32 * words} for s in sees]
        mask = up(od.words_of(sees, 2))[:, :words]
        for max_len in (260, 37):
            out = torch.full((T, Hq, 128), 7.0, dtype=torch.float16, device=DEV)
            sq.attn_tree(up(q), device_cache(cache), ints(table), ints(lens), ints(cu), max_len, mask=mask, out=out)
            want, weight, rows = od.attn_tree(q, cache, cu, lens, table, max_len, known)
            assert not rows[40:42].any() and rows.sum() == T - 2
            attention_close(out[up(rows)], want[rows], weight[rows], 2e-5)
            assert not out[0].any() and torch.all(out[40:42] == 7.0)


def test_depths_of_any_size():
    """Depths below 0 and huge ones move the window no further than they say, and out of nothing."""
    g = rng(12)
    lens, cu = [300], [0, 4]
    table, pages = spread_table(g, lens, 16)
    cache = filled(g, pages, 2, 16, 4, np.float32)
    q = heads_of(g, 4, 8)
    depth = [-5, 0, 2 ** 31 - 1, 3]
    sees = [{0}, {1}, {0, 2}, {3}]
    got = sq.attn_tree(up(q), device_cache(cache), ints(table), ints(lens), ints(cu), 300, mask=up(od.words_of(sees, 1)), depth=ints(depth),
                       window=50, sinks=3)
    want, weight, _ = od.attn_tree(q, cache, cu, lens, table, 300, sees, [0, 0, 2 ** 30, 3], 50, 3)
    attention_close(got, want, weight, 2e-5)


@pytest.mark.parametrize("mode", ["tree", "chain"])
@pytest.mark.parametrize("bits,dt", [(4, np.float32), (8, np.float16)])
def test_hidden_parameters_that_are_not_finite(bits, dt, mode):
    """NaN and infinities in the parameters of tokens that a row does not see, before the window and among the drafts,
    change nothing; a row that sees one of them is NaN."""
    g = rng(13)
    Hq, H, page, window, sinks = 8, 2, 16, 20, 2
    lens, cu, n = [200], [0, 9], 9
    table, pages = spread_table(g, lens, page)
    cache = filled(g, pages, H, page, bits, dt)
    q = heads_of(g, n, Hq)
    sees, depth, _ = od.tree_mask([-1, 0, 0, 1, 2, 3, 4, 4, -1], cu, lens, window, sinks)
    bad = 200 - 9 + 4  # the draft 4, and one token before every window
    for t, x in ((100, np.nan), (bad, np.nan), (bad, np.inf)):
        c = {name: a.copy() for name, a in cache.items()}
        c["params"][table[0, t // page], :, t % page] = x
        args = dict(mask=up(od.words_of(sees, 1)), depth=ints(depth)) if mode == "tree" else {}
        got = sq.attn_tree(up(q), device_cache(c), ints(table), ints(lens), ints(cu), 200, window=window, sinks=sinks, **args)
        want, weight, _ = od.attn_tree(q, cache, cu, lens, table, 200, *((sees, depth) if mode == "tree" else (None, None)), window, sinks)
        clean = [i for i in range(n) if t == 100 or (4 not in sees[i] if mode == "tree" else i < 4)]
        attention_close(got[clean], want[clean], weight[clean], 2e-5)
        assert torch.isnan(got[[i for i in range(n) if i not in clean]]).all()


def test_queries_that_are_not_finite():
    """NaN in the rows of such a query that see a token, zeros in those that see none, and nothing beside them."""
    g = rng(14)
    lens, cu = [60, 2], [0, 4, 6]
    table, pages = spread_table(g, lens, 16)
    cache = filled(g, pages, 2, 16, 4, np.float32)
    q = heads_of(g, 6, 8)
    clean = q.copy()
    q[1, 3, 5], q[4, 0, 0] = np.nan, np.inf
    sees = [{0}, {0, 1}, {2}, {3}, set(), {1}]
    got = sq.attn_tree(up(q), device_cache(cache), ints(table), ints(lens), ints(cu), 60, mask=up(od.words_of(sees, 1)))
    want, weight, _ = od.attn_tree(clean, cache, cu, lens, table, 60, sees)
    assert torch.isnan(got[1, 3]).all() and not got[4].any()
    got[1, 3] = up(want[1, 3].astype(np.float16))
    attention_close(got, want, weight, 2e-5)


STEP = [  # Hq, Hkv, page, bits, params, lens, max_len, window, sinks
    (8, 2, 16, 4, np.float32, [1, 2, 15, 64, 65, 0, 200, 1000], 1000, 64, 4),
    (8, 2, 16, 4, np.float32, [3000, 700], 3000, 1, 0),
    (32, 8, 64, 4, np.float16, [5000], 5000, 1000, 130),
    (4, 4, 16, 8, np.float32, [257, 31, 1], 300, 100, 0),
    (33, 1, 32, 8, np.float16, [900, 40], 1 << 20, 257, 1),
    (8, 8, 16, 4, np.float32, [600, 90], 600, 5000, 9),     # wider than any length
    (8, 2, 16, 4, np.float32, [600, 90], 600, 100, 5000),   # all first tokens
]


@pytest.mark.parametrize("case", STEP, ids=lambda c: f"{c[0]}x{c[1]}-b{c[3]}-w{c[7]}s{c[8]}-{max(c[5])}")
def test_attn_paged_window(case):
    Hq, H, page, bits, dt, lens, most, window, sinks = case
    g = rng(Hq + window)
    table, pages = spread_table(g, lens, page)
    for b, n in enumerate(lens):  # pages wholly between the first tokens and the window are no longer there
        for c in range(-(-sinks // page), max(0, n - window) // page):
            table[b, c] = -1
    cache = filled(g, pages, H, page, bits, dt)
    q = heads_of(g, len(lens), Hq)
    got = sq.attn_paged(up(q), device_cache(cache), ints(table), ints(lens), most, window=window, sinks=sinks)
    want, weight = od.attn_paged_window(q, cache, lens, table, most, window, sinks)
    attention_close(got, want, weight, 2e-5)
    assert not got[up(np.array(lens) == 0)].any()


PROMPT = [  # Hq, Hkv, rows of q, keys, window, sinks
    (4, 4, [300], [300], 64, 4),
    (8, 2, [100, 1, 257, 0, 40], [100, 70, 300, 5, 900], 100, 0),
    (8, 1, [130], [700], 1, 70),
    (4, 2, [64, 65], [64, 65], 1000, 3),
    (2, 2, [700], [700], 129, 64),
    (2, 2, [5, 3], [3000, 2000], 500, 10),     # few rows over many keys: parts
    (6, 2, [40], [30], 8, 2),                  # rows before the first key
    (8, 8, [600, 520], [900, 2200], 300, 200),
    (32, 32, [1100], [1100], 200, 1),          # whole tiles of 256 rows
]


@pytest.mark.parametrize("case", PROMPT, ids=lambda c: f"{c[0]}x{c[1]}-{max(c[2])}of{max(c[3])}-w{c[4]}s{c[5]}")
def test_attn_prompt_window(case):
    Hq, H, nq, nk, window, sinks = case
    g = rng(Hq + window + sum(nq))
    cu_q, cu_k = packed(nq, 1), packed(nk, 2)
    Tq, Tk = int(cu_q[-1]) + 2, int(cu_k[-1]) + 1
    q, k, v = heads_of(g, Tq, Hq), heads_of(g, Tk, H), heads_of(g, Tk, H)
    out = torch.full((Tq, Hq, 128), 7.0, dtype=torch.float16, device=DEV)
    sq.attn_prompt(up(q), up(k), up(v), ints(cu_q), ints(cu_k), window=window, sinks=sinks, out=out)
    want, weight, rows = od.attn_prompt_window(q, k, v, cu_q, cu_k, window, sinks)
    attention_close(out[up(rows)], want[rows], weight[rows], 2e-5)
    assert torch.all(out[up(~rows)] == 7.0)


@pytest.mark.parametrize("Hq,nq,nk", [(2, 300, 300), (2, 4, 3000), (130, 300, 300)], ids=["halves", "parts", "whole"])
def test_prompt_keys_behind_the_window(Hq, nq, nk):
    """What is not finite in keys and values that a row does not see leaves it alone; the rows that see it are not finite."""
    g = rng(21)
    window, sinks, bad = 50, 3, nk - nq // 2 - 20
    q, k, v = heads_of(g, nq, Hq), heads_of(g, nk, Hq), heads_of(g, nk, Hq)
    want, weight, _ = od.attn_prompt_window(q, k, v, [0, nq], [0, nk], window, sinks)
    sees = np.array([bad <= nk - nq + i < bad + window for i in range(nq)])
    assert sees.any()
    for what, x in ((k, np.nan), (v, np.inf), (v, np.nan)):
        old = what[bad].copy()
        what[bad] = x
        got = sq.attn_prompt(up(q), up(k), up(v), ints([0, nq]), ints([0, nk]), window=window, sinks=sinks)
        what[bad] = old
        if not sees.all():
            attention_close(got[up(~sees)], want[~sees], weight[~sees], 2e-5)
        assert not torch.isfinite(got[up(sees)]).any()


@pytest.mark.parametrize("Hq,H,nq", [(2, 2, [300, 1, 37]), (130, 130, [300, 1, 37]), (24, 2, [25, 0, 3])], ids=["halves", "whole", "shared"])
def test_prompt_window_into_a_wider_tensor(Hq, H, nq):
    """Rows of a strided out, the last ones of a wave's 32 among them; what lies beside them and between the sequences stays."""
    g = rng(Hq)
    nk = [n + 40 for n in nq]
    cu_q, cu_k = packed(nq, 2), packed(nk)
    T = int(cu_q[-1]) + 3
    q, k, v = up(heads_of(g, T, Hq)), up(heads_of(g, int(cu_k[-1]), H)), up(heads_of(g, int(cu_k[-1]), H))
    wide = torch.full((T, Hq + 2, 128), 7.0, dtype=torch.float16, device=DEV)
    want = torch.full((T, Hq, 128), 7.0, dtype=torch.float16, device=DEV)
    for out in (wide[:, 1:-1], want):
        sq.attn_prompt(q, k, v, ints(cu_q), ints(cu_k), window=33, sinks=2, out=out)
    assert torch.equal(wide[:, 1:-1], want) and torch.all(wide[:, 0] == 7.0) and torch.all(wide[:, -1] == 7.0)
    assert torch.all(want[:2] == 7.0) and torch.all(want[-3:] == 7.0)
    ref, weight, rows = od.attn_prompt_window(*(x.cpu().numpy() for x in (q, k, v)), cu_q, cu_k, 33, 2)
    attention_close(want[up(rows)], ref[rows], weight[rows], 2e-5)


KEEP = [(4, np.float32, 16, 2), (8, np.float16, 32, 5), (4, np.float16, 64, 1), (8, np.float32, 16, 32)]


@pytest.mark.parametrize("bits,dt,page,H", KEEP)
def test_kv_keep(bits, dt, page, H):
    g = rng(page + H)
    new, past = [16, 1, 0, 40, 5, 9, 64, 6], [10, 30, 4, 61, 0, 100, 7, 3]
    lens = [n + p for n, p in zip(new, past)]
    lens[7] = 4  # two drafts without a place
    cu = packed(new, 3)
    table, pages = spread_table(g, lens, page)
    table[5, (100 + 3) // page] = -1
    cache = filled(g, pages, H, page, bits, dt)
    path = np.tile(np.arange(40), (8, 1))
    path[0, :5] = [1, 2, 6, 7, 15]
    path[3, :40] = np.arange(40)
    path[3, 20:] = 39
    path[4, :5] = [4, 0, 7, -1, 2 ** 31 - 1]
    path[5, :4] = [0, 3, 5, 8]
    path[6, :40] = np.sort(g.permutation(64)[:40])
    path[7, :4] = [1, 3, 4, 5]
    kept = [5, 1, 3, 40, 5, 4, 99, 4]
    want, lens_out = od.kv_keep(cache, cu, lens, table, path, kept)
    dc = device_cache(cache)
    wide = torch.full((8, 43), 1, dtype=torch.int32, device=DEV)
    wide[:, :40] = ints(path)
    got = sq.kv_keep(dc, ints(table), ints(lens), ints(cu), wide[:, :40], ints(kept))
    assert got.tolist() == lens_out
    for t, name in zip(dc, ("k_q", "v_q", "params")):
        assert np.array_equal(t.cpu().numpy(), want[name])


def test_keep_nothing():
    g = rng(2)
    table, pages = spread_table(g, [20, 30], 16)
    cache = filled(g, pages, 2, 16, 4, np.float32)
    dc = device_cache(cache)
    got = sq.kv_keep(dc, ints(table), ints([20, 30]), ints([0, 4, 9]), ints([[0], [0]]), ints([0, -3]))
    assert got.tolist() == [16, 25] and all(np.array_equal(t.cpu().numpy(), cache[n]) for t, n in zip(dc, ("k_q", "v_q", "params")))


def test_many_sequences():
    """More sequences than one step of the searches, some without drafts, in several chunks."""
    g = rng(31)
    B, Hq, H, page = 150, 8, 2, 16
    new = [int(x) for x in g.integers(0, 5, B)]
    new[7], new[140] = 30, 17
    lens = [n + int(x) for n, x in zip(new, g.integers(0, 90, B))]
    lens[3], lens[149] = new[3] + 1500, new[149] + 900
    cu, T = packed(new, 3), sum(new) + 5
    table, pages = spread_table(g, lens, page)
    cache = filled(g, pages, H, page, 4, np.float16)
    q = heads_of(g, T, Hq)
    parents = np.concatenate([[0] * 3] + [np.array(tree(g, n), dtype=np.int64) for n in new] + [[0] * 2]).astype(np.int64)
    mask, depth = sq.tree_mask(ints(parents), ints(cu), 30)
    sees, want_depth, rows = od.tree_mask(parents, cu)
    assert np.array_equal(mask.cpu().numpy()[rows], od.words_of(sees, 1)[rows]) and np.array_equal(depth.cpu().numpy()[rows], want_depth[rows])
    n = sq.attn_tree_workspace_bytes(B, T, max(lens), Hq, H)
    assert n > 0
    ws = torch.full((n + 16,), 255, dtype=torch.uint8, device=DEV)
    out = torch.full((T, Hq, 128), 7.0, dtype=torch.float16, device=DEV)
    sq.attn_tree(up(q), device_cache(cache), ints(table), ints(lens), ints(cu), max(lens), mask=mask, out=out, workspace=ws)
    want, weight, rows = od.attn_tree(q, cache, cu, lens, table, max(lens), sees)
    attention_close(out[up(rows)], want[rows], weight[rows], 2e-5)
    assert torch.all(out[up(~rows)] == 7.0) and torch.all(ws[n:] == 255)


def test_a_chain_is_what_the_chunk_of_a_prompt_is():
    """A chunk's rows over the pages against the same keys read back and attended in fp16 (rounded there: 2^-11 of keys,
    16 of them in a score of this size, and of values)."""
    g = rng(32)
    Hq, H, page, n, length = 16, 4, 32, 300, 1300
    table, pages = spread_table(g, [length], page)
    dc = device_cache(filled(g, pages, H, page, 8, np.float32))
    q = up(heads_of(g, n, Hq))
    for window, sinks in ((0, 0), (200, 5)):
        got = sq.attn_tree(q, dc, ints(table), ints([length]), ints([0, n]), length, window=window, sinks=sinks)
        k, v = sq.kv_read(dc, ints(table), ints([length]), ints([0, length]), length)
        want = sq.attn_prompt(q, k, v, ints([0, n]), ints([0, length]), window=window, sinks=sinks)
        size = f64(v).max()
        assert np.abs(f64(got) - f64(want)).max() <= (2.0 ** -11 * 16 + 3 * 2.0 ** -11) * size


def test_a_window_of_everything_is_no_window():
    g = rng(33)
    lens, page = [300, 20], 16
    table, pages = spread_table(g, lens, page)
    dc = device_cache(filled(g, pages, 2, page, 4, np.float32))
    q = up(heads_of(g, 2, 8))
    a = sq.attn_paged(q, dc, ints(table), ints(lens), 300)
    for window, sinks in ((300, 0), (2 ** 30 - 1, 0), (1, 2 ** 30 - 1), (5, 295)):
        b = sq.attn_paged(q, dc, ints(table), ints(lens), 300, window=window, sinks=sinks)
        assert np.abs(f64(a) - f64(b)).max() <= 2 * (2.0 ** -11 + 2e-5) * 8
    p = up(heads_of(g, 90, 8)), up(heads_of(g, 90, 2)), up(heads_of(g, 90, 2))
    cu = ints([0, 90])
    a = sq.attn_prompt(*p, cu, cu)
    for window, sinks in ((90, 0), (2 ** 30 - 1, 0), (3, 87)):
        assert torch.equal(a, sq.attn_prompt(*p, cu, cu, window=window, sinks=sinks)), (window, sinks)


@pytest.mark.parametrize("scale", [-0.1, 0.0, 2.0])
def test_scales(scale):
    g = rng(34)
    lens, cu = [150, 70], [0, 9, 15]
    table, pages = spread_table(g, lens, 16)
    cache = filled(g, pages, 2, 16, 4, np.float32, 0.5)
    q = heads_of(g, 15, 8, 0.5)
    sees, depth, _ = od.tree_mask(tree(g, 9) + tree(g, 6), cu)
    got = sq.attn_tree(up(q), device_cache(cache), ints(table), ints(lens), ints(cu), 150, mask=up(od.words_of(sees, 1)), scale=scale)
    want, weight, _ = od.attn_tree(q, cache, cu, lens, table, 150, sees, scale=scale)
    # fp32 scores: 130 roundings of scale sum |q k|
    attention_close(got, want, weight, 2e-5 + 130 * 2.0 ** -24 * abs(scale) * 128 * 0.5)


@pytest.mark.parametrize("std", [2.0 ** -23, 2.0 ** -14, 2.0 ** 9])
def test_queries_of_any_size(std):
    """Queries of subnormal and of large numbers, with a scale that makes the scores the same; one row far below the others."""
    g = rng(35)
    lens, cu = [200], [0, 8]
    table, pages = spread_table(g, lens, 16)
    cache = filled(g, pages, 2, 16, 4, np.float32)
    q = heads_of(g, 8, 8, std)
    q[3] = heads_of(g, 1, 8, std * 2.0 ** -6)[0]
    scale = 128 ** -0.5 / std
    got = sq.attn_tree(up(q), device_cache(cache), ints(table), ints(lens), ints(cu), 200, scale=scale)
    want, weight, _ = od.attn_tree(q, cache, cu, lens, table, 200, scale=scale)
    attention_close(got, want, weight, 2e-5)


def test_slots_that_were_never_written():
    """A zeroed cache, and drafts that see such slots."""
    g = rng(36)
    got = sq.attn_tree(up(heads_of(g, 5, 8)), sq.kv_cache(5, 16, 2), ints([[4, 2, 0]]), ints([41]), ints([0, 5]), 41)
    assert not got.any()


@pytest.mark.parametrize("bits", [4, 8])
def test_pages_beyond_32_bits(bits):
    """A pool of more than 4 GiB of codes: attention over its last pages, and a draft moved among them."""
    H, page, row = 64, 128, 16 * bits
    pages = (2 ** 32 + 2 ** 28) // (H * page * row)
    k_q = torch.zeros((pages, H, page, row), dtype=torch.uint8, device=DEV)
    cache = k_q, torch.zeros_like(k_q), torch.zeros((pages, H, page, 4), dtype=torch.float16, device=DEV)
    g = rng(37)
    small = filled(g, 2, H, page, bits, np.float16)
    for t, n in zip(cache, ("k_q", "v_q", "params")):
        t[pages - 2:] = up(small[n])
    table, near = [[pages - 1, pages - 2]], [[1, 0]]
    q = up(heads_of(g, 12, H))
    args = ints([230]), ints([0, 12]), 230
    want = sq.attn_tree(q, device_cache(small), ints(near), *args)
    assert torch.equal(sq.attn_tree(q, cache, ints(table), *args), want)
    want = sq.attn_paged(q[:1], device_cache(small), ints(near), ints([230]), 230, window=60, sinks=4)
    assert torch.equal(sq.attn_paged(q[:1], cache, ints(table), ints([230]), 230, window=60, sinks=4), want)
    dc = device_cache(small)
    path, kept = ints([[0, 3, 7, 11]]), ints([4])
    assert sq.kv_keep(dc, ints(near), ints([260 - 9]), ints([0, 12]), path, kept).tolist() == [243]
    sq.kv_keep(cache, ints(table), ints([251]), ints([0, 12]), path, kept)
    assert all(torch.equal(a[pages - 2:], b) for a, b in zip(cache, dc))


def test_two_graphs_that_share_a_workspace():
    """Captured trees of different sizes over one workspace, replayed in turn with eager work between: each as eager."""
    g = rng(41)
    Hq, H, page = 32, 8, 16
    calls, buffers = [], []
    size = 0
    for new, past, window in (([16], [2000], 0), ([3, 9, 1], [900, 70, 400], 0), ([8], [1500], 300)):
        lens, cu = [n + p for n, p in zip(new, past)], packed(new)
        table, pages = spread_table(g, lens, page)
        sees, depth, _ = od.tree_mask(sum((tree(g, n) for n in new), []), cu, lens, window, 2)
        args = dict(mask=up(od.words_of(sees, 1)), depth=ints(depth), window=window, sinks=2 if window else 0)
        cache = device_cache(filled(g, pages, H, page, 4, np.float32))
        q = up(heads_of(g, sum(new), Hq))
        place = cache, ints(table), ints(lens), ints(cu), max(lens)
        size = max(size, sq.attn_tree_workspace_bytes(len(new), sum(new), max(lens), Hq, H, window, args["sinks"]))
        buffers.append((q, torch.empty_like(q)))
        calls.append((place, args))
    ws = torch.full((size,), 255, dtype=torch.uint8, device=DEV)

    def call(k):
        (q, out), (place, args) = buffers[k], calls[k]
        sq.attn_tree(q, *place, out=out, workspace=ws, **args)

    for k in range(3):
        call(k)
    torch.cuda.synchronize()
    graphs = []
    for k in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(k)
        graphs.append(graph)
    for turn in range(4):
        for k in range(2):
            buffers[k][0].copy_(up(heads_of(g, buffers[k][0].shape[0], Hq)))
        wants = [sq.attn_tree(buffers[k][0], *calls[k][0], **calls[k][1]) for k in range(3)]
        for k in (0, 1) if turn % 2 else (1, 0):
            graphs[k].replay()
            call(2)
        torch.cuda.synchronize()
        for k in range(3):
            assert torch.equal(buffers[k][1], wants[k]), (turn, k)


def test_another_stream():
    g = rng(42)
    lens, cu = [700], [0, 20]
    table, pages = spread_table(g, lens, 16)
    dc = device_cache(filled(g, pages, 2, 16, 4, np.float32))
    q = up(heads_of(g, 20, 8))
    args = dc, ints(table), ints(lens), ints(cu), 700
    want = sq.attn_tree(q, *args)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        late = q * 1.0
        got = sq.attn_tree(late, *args)
    side.synchronize()
    assert torch.equal(got, want)


def test_empty_calls():
    cache = sq.kv_cache(2, 16, 2)
    none, one = ints([]), ints([0])
    q = torch.empty((0, 8, 128), dtype=torch.float16, device=DEV)
    assert sq.attn_tree(q, cache, ints([[0]]), ints([5]), ints([0, 0]), 5).shape == (0, 8, 128)
    assert sq.attn_tree(q, cache, none.view(0, 1), none, one, 5).shape == (0, 8, 128)
    assert sq.attn_paged(q, cache, none.view(0, 1), none, 5, window=4).shape == (0, 8, 128)
    assert sq.attn_prompt(q, q[:, :2], q[:, :2], one, one, window=4).shape == (0, 8, 128)
    mask, depth = sq.tree_mask(none, ints([0, 0]), 4)
    assert mask.shape == (0, 1) and depth.shape == (0,)
    assert sq.kv_keep(cache, none.view(0, 1), none, one, none.view(0, 1), none).shape == (0,)
    sq.paged_release(none.view(0, 1), 16, none, none, none, ints([0, 0]), one)
    # drafts without any sequence that has some
    out = torch.full((3, 8, 128), 7.0, dtype=torch.float16, device=DEV)
    sq.attn_tree(out.clone(), cache, ints([[0], [1]]), ints([5, 3]), ints([2, 2, 2]), 5, out=out)
    assert torch.all(out == 7.0)


def test_binding_refusals():
    cache = sq.kv_cache(2, 16, 2)
    q = torch.zeros((4, 8, 128), dtype=torch.float16, device=DEV)
    t, lens, cu = ints([[0, 1]]), ints([20]), ints([0, 4])
    mask = ints([[1], [3], [5], [9]])
    ok = lambda **k: sq.attn_tree(q, cache, t, lens, cu, 20, **k)  # noqa: E731
    ok(mask=mask)
    for bad in (dict(mask=mask[:3]), dict(mask=mask.t()), dict(mask=mask.long()), dict(mask=mask, depth=ints([0, 1])), dict(out=q[:3]),
                dict(workspace=torch.empty((64, 2), dtype=torch.uint8, device=DEV)[:, 0])):
        with pytest.raises((TypeError, ValueError)):
            ok(**bad)
    for bad in (dict(depth=ints([0, 1, 2, 3])), dict(window=-1), dict(window=1 << 30), dict(scale=float("nan"))):
        with pytest.raises(sq.SqError):
            ok(**bad)
    with pytest.raises(sq.SqError):  # in place
        ok(out=q)
    with pytest.raises(ValueError):
        sq.attn_prompt(q, q[:, :2], q[:, :2], cu, cu, causal=False, window=3)
    with pytest.raises(ValueError):
        sq.tree_mask(ints([0, 1]), cu, 4, out=(mask, ints([0, 0])))
    with pytest.raises(sq.SqError):
        sq.tree_mask(ints([0, 1, 1, 2]), cu, 4, window=3, sinks=1)
    with pytest.raises(sq.SqError):
        sq.kv_keep(cache, t, lens, cu, ints([[0, 1]]), ints([1]), out=lens)
    with pytest.raises(ValueError):
        sq.kv_keep(cache, t, lens, cu, ints([[0, 1], [0, 1]]), ints([1]))
    with pytest.raises(ValueError):
        sq.paged_grow(lens, lens, ints([1, 1]), t, 16, ints([0, 0]), ints([2]), 4)
    with pytest.raises(sq.SqError):
        sq.paged_grow(lens, lens, ints([1]), t, 24, ints([0, 0]), ints([2]), 4)


@pytest.mark.parametrize("window,sinks,bits", [(0, 0, 4), (60, 4, 8)])
def test_a_server_that_drafts(window, sinks, bits):
    """Prompts, then steps of drafts: pages handed out, masks, the write by depth, attention, a check that keeps some
    path, its move, and pages given back; each call's input is the one before's output, and each is the oracle's on
    it.  A token's keys in the cache are, in the end, those of the text written at once."""
    g = rng(51 + bits)
    B, Hq, H, page, cols, pages = 3, 8, 2, 16, 14, 60
    freq = opg.rope_frequencies(128, 10000.0)
    dfreq = up(freq)
    cache = sq.kv_cache(pages, page, H, bits)
    held, pool, count = ints([0] * B), ints(g.permutation(pages)), ints([pages])
    table = ints(np.full((B, cols), -1))
    have = ints([0] * B)
    texts = [np.zeros((0, 2 * H, 128), dtype=np.float16) for _ in range(B)]  # keys and values before positions
    for step in range(6):
        new = [int(x) for x in g.integers(20, 90, B)] if step == 0 else [int(x) for x in g.integers(1, 12, B)]
        T = sum(new)
        lens, cu, pos, slots, missing = sq.paged_grow(have, ints(new), held, table, page, pool, count, T)
        assert missing.tolist() == [0, 0]
        base, bounds = have.tolist(), cu.tolist()
        parents = sum(([i - 1 for i in range(n)] if step == 0 else tree(g, n, 4) for n in new), [])
        mask, depth = sq.tree_mask(ints(parents), cu, max(new), lens=lens, window=window, sinks=sinks)
        sees, want_depth, _ = od.tree_mask(parents, bounds, lens.tolist(), window, sinks, mask.shape[1])
        assert np.array_equal(mask.cpu().numpy(), od.words_of(sees, mask.shape[1])) and depth.tolist() == list(want_depth)
        q, kv = heads_of(g, T, Hq), heads_of(g, T, 2 * H)
        qr = sq.rope_kv_write(up(q), up(kv)[:, :H], up(kv)[:, H:], cache, table, lens, dfreq, cu=cu, depth=depth)
        # each row's slot holds its value's codes
        host = {n: t.cpu().numpy() for n, t in zip(("k_q", "v_q", "params"), cache)}
        codes, a, b = opg.quant_asym(kv[:, H:].astype(np.float32), bits=bits, group=128, clip=1.0, param_fp16=False)
        for t, s in enumerate(slots.tolist()):
            assert np.array_equal(host["v_q"][s // page, :, s % page], opg.store_codes(codes[t], bits))
        out = sq.attn_tree(qr, cache, table, lens, cu, cols * page, mask=mask, depth=depth, window=window, sinks=sinks)
        want, weight, _ = od.attn_tree(qr.cpu().numpy(), host, bounds, lens.tolist(), table.cpu().numpy(), cols * page, sees, want_depth,
                                       window, sinks)
        attention_close(out, want, weight, 2e-5)
        # the check: a way down from a root, or nothing; prompts are kept whole
        paths = []
        for b in range(B):
            mine = parents[bounds[b]:bounds[b + 1]]
            end = new[b] - 1 if step == 0 else int(g.integers(-1, new[b]))
            way = []
            while end >= 0:
                way.append(end)
                end = mine[end]
            paths.append(way[::-1])
            texts[b] = np.concatenate([texts[b], kv[[bounds[b] + i for i in paths[b]]]])
        longest = max(1, max(len(p) for p in paths))
        have = sq.kv_keep(cache, table, lens, cu, ints([p + [0] * (longest - len(p)) for p in paths]), ints([len(p) for p in paths]))
        assert have.tolist() == [n + len(p) for n, p in zip(base, paths)]
        sq.paged_release(table, page, have, ints([2 ** 31 - 1] * B), held, pool, count)
        assert count.item() == pages - sum(held.tolist()) and held.tolist() == [-(-n // page) for n in have.tolist()]
    # the same text written in one call
    total = have.tolist()
    cu, rows = packed(total), sum(total)
    kv = up(np.concatenate(texts))
    again = sq.kv_cache(pages, page, H, bits)
    sq.rope_kv_write(up(heads_of(g, rows, Hq)), kv[:, :H], kv[:, H:], again, table, have, dfreq, cu=ints(cu))
    a, b = (sq.kv_read(c, table, have, ints(cu), rows) for c in (cache, again))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_a_captured_step_of_drafts():
    """A whole step in one graph, replayed while the sequences grow, with eager work between: each replay as eager."""
    g = rng(61)
    B, Hq, H, page, cols, pages, n = 2, 8, 2, 16, 20, 60, 6
    dfreq = up(opg.rope_frequencies(128, 10000.0))
    T = B * n

    def state():
        return dict(cache=sq.kv_cache(pages, page, H), held=ints([0] * B), pool=ints(range(pages)), count=ints([pages]),
                    table=ints(np.full((B, cols), -1)), have=ints([0] * B))

    parents, path, kept, add = ints(np.zeros(T)), ints(np.zeros((B, n))), ints([0] * B), ints([n] * B)
    qkv = torch.zeros((T, Hq + 2 * H, 128), dtype=torch.float16, device=DEV)
    ws = torch.empty(sq.attn_tree_workspace_bytes(B, T, cols * page, Hq, H), dtype=torch.uint8, device=DEV)
    outs = [ints([0] * B), ints([0] * (B + 1)), ints([0] * T), torch.zeros(T, dtype=torch.int64, device=DEV), ints([0, 0])]
    mask, depth, out = ints(np.zeros((T, 1))), ints([0] * T), torch.empty((T, Hq, 128), dtype=torch.float16, device=DEV)
    qr, after, far = torch.empty_like(out), ints([0] * B), ints([2 ** 31 - 1] * B)

    def step(s):
        lens, cu, *_ = sq.paged_grow(s["have"], add, s["held"], s["table"], page, s["pool"], s["count"], T, out=outs)
        sq.tree_mask(parents, cu, n, out=(mask, depth))
        sq.rope_kv_write(qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:], s["cache"], s["table"], lens, dfreq, cu=cu, out=qr, depth=depth)
        sq.attn_tree(qr, s["cache"], s["table"], lens, cu, cols * page, mask=mask, depth=depth, out=out, workspace=ws)
        sq.kv_keep(s["cache"], s["table"], lens, cu, path, kept, out=after)
        s["have"].copy_(after)
        sq.paged_release(s["table"], page, s["have"], far, s["held"], s["pool"], s["count"])

    eager, captured = state(), state()
    step(state())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(captured)
    for turn in range(12):
        ways = []
        trees = [tree(g, n, 3) for _ in range(B)]
        for t in trees:
            end, way = int(g.integers(0, n)), []
            while end >= 0:
                way.append(end)
                end = t[end]
            ways.append(way[::-1])
        parents.copy_(ints(sum(trees, [])))
        path.copy_(ints([w + [0] * (n - len(w)) for w in ways]))
        kept.copy_(ints([len(w) for w in ways]))
        qkv.copy_(up(heads_of(g, T, Hq + 2 * H)))
        step(eager)
        want = out.clone()
        out.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), turn
        for x, y in zip(eager["cache"], captured["cache"]):
            assert torch.equal(x, y), turn
        assert all(torch.equal(eager[k], captured[k]) for k in ("held", "pool", "count", "table", "have")), turn
    assert min(eager["have"].tolist()) > 12
