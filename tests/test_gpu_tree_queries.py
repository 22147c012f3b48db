"""Attention of several rows over the pages where the rows of one workgroup have queries of very different sizes:
each row has the precision that it has alone.

Tolerances as in tests/test_gpu_paged.py.  A row's scores are off by its own roundings: the products are exact, their
sums fp32, and whatever brings queries into fp16's range may lose 2^-24 of the row's largest element in each of 128
terms, 2^-24 * 16 * sqrt(128) of a score of this size (which is below 16): 1.1e-5 beside the 1e-5 that sums of 32 bits
take of the 2e-5 in general, so 3.2e-5 here.
"""

import numpy as np
import pytest
import torch

from oracle import drafts as od
from paper_2405_16406_amd import sq
from test_gpu_paged import attention_close, device_cache, f64, filled, heads_of, ints, rng, spread_table, up

pytestmark = pytest.mark.gpu

SCORES = 3.2e-5
# Hq, Hkv, params, drafts, tokens before: one column of 16 rows and four waves, eight waves, two columns, chunks joined
FORMS = {"one": (8, 2, np.float32, [7, 3], [100, 30]), "eight": (8, 2, np.float16, [6, 3], [600, 1000]),
         "two": (64, 8, np.float32, [32, 5, 17], [1500, 700, 64]), "two, fp16": (64, 8, np.float16, [33, 20], [900, 1400]),
         "joined": (8, 2, np.float16, [3, 8], [3000, 100])}


def case_of(g, form, bits, page=16):
    Hq, H, dt, new, past = FORMS[form]
    lens = [n + p for n, p in zip(new, past)]
    cu = np.concatenate([[0], np.cumsum(new)])
    table, pages = spread_table(g, lens, page)
    return Hq, filled(g, pages, H, page, bits, dt), lens, cu, table, int(cu[-1])


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("other", [np.inf, np.nan, 6e4, 1.0], ids=str)
@pytest.mark.parametrize("size", [-12, -16, -20])
@pytest.mark.parametrize("form", FORMS)
def test_small_rows_beside_a_large_one(form, size, other, bits):
    """Small queries, and one row of the same heads with a single large element, or one that is not finite."""
    g = rng(81)
    Hq, cache, lens, cu, table, T = case_of(g, form, bits)
    std = 2.0 ** size
    q = heads_of(g, T, Hq, std)
    large = np.zeros((T, Hq), dtype=bool)
    large[cu[:-1], ::4] = large[2] = True
    q[large, 9] = other
    scale = 128 ** -0.5 / std
    got = sq.attn_tree(up(q), device_cache(cache), ints(table), ints(lens), ints(cu), max(lens), scale=scale)
    with np.errstate(all="ignore"):
        want, weight, _ = od.attn_tree(q, cache, cu, lens, table, max(lens), scale=scale)
    attention_close(got[up(~large)], want[~large], weight[~large], SCORES)
    finite = torch.isfinite(got[up(large)])
    assert finite.all() if np.isfinite(other) else not finite.any()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("form", FORMS)
def test_rows_of_every_size(form, bits):
    """Rows from 2^-20 to 2^0 of the largest, with a scale that makes the scores of one size ordinary: these are compared."""
    g = rng(82)
    Hq, cache, lens, cu, table, T = case_of(g, form, bits)
    q = heads_of(g, T, Hq)
    q *= (2.0 ** -(np.arange(T * Hq) % 21)).reshape(T, Hq, 1).astype(np.float16)
    for step in (0, 5, 10, 15, 20):
        mine = (np.arange(T * Hq) % 21).reshape(T, Hq) == step
        scale = 128 ** -0.5 * 2.0 ** step
        got = sq.attn_tree(up(q), device_cache(cache), ints(table), ints(lens), ints(cu), max(lens), scale=scale)
        want, weight, _ = od.attn_tree(q, cache, cu, lens, table, max(lens), scale=scale)
        attention_close(got[up(mine)], want[mine], weight[mine], SCORES)


@pytest.mark.parametrize("step", [8, 9, 10, 11, 12])
def test_two_sizes(step):
    """Half the rows 2^-step of the others, around the ratio from which each row is scaled for itself."""
    g = rng(83 + step)
    Hq, cache, lens, cu, table, T = case_of(g, "two", 4)
    q = heads_of(g, T, Hq)
    q[:, ::2] *= np.float16(2.0 ** -step)
    scale = 128 ** -0.5 * 2.0 ** step
    got = sq.attn_tree(up(q), device_cache(cache), ints(table), ints(lens), ints(cu), max(lens), scale=scale)
    want, weight, _ = od.attn_tree(q, cache, cu, lens, table, max(lens), scale=scale)
    attention_close(got[:, ::2], want[:, ::2], weight[:, ::2], SCORES)


@pytest.mark.parametrize("form", ["one", "two"])
def test_what_rows_do_not_see_beside_rows_of_another_size(form):
    """Pages that are missing, tokens before a window, a draft without a bit, parameters that are not finite in
    hidden places, a row of zeros, where small rows stand beside one with an infinity."""
    g = rng(84)
    Hq, cache, lens, cu, table, T = case_of(g, form, 4)
    most, window, sinks, std = max(lens), 40, 3, 2.0 ** -16
    q = heads_of(g, T, Hq, std)
    large = np.zeros((T, Hq), dtype=bool)
    large[cu[:-1], ::4] = True
    q[large, 5] = np.inf
    q[cu[1] - 1, 1] = 0
    missing = table.copy()
    for b, n in enumerate(lens):
        missing[b, (n - 20) // 16] = -1
    parents = np.concatenate([g.integers(-1, np.maximum(1, np.arange(n))) for n in np.diff(cu)])
    words = 2
    sees, depth, _ = od.tree_mask(parents, cu, lens, window, sinks, words)
    sees[cu[1] - 2] = set()
    scale = 128 ** -0.5 / std
    args = dict(mask=up(od.words_of(sees, words)), depth=ints(depth), window=window, sinks=sinks, scale=scale)
    with np.errstate(all="ignore"):
        want, weight, _ = od.attn_tree(q, cache, cu, lens, missing, most, sees, depth, window, sinks, scale)
    hidden = {n: a.copy() for n, a in cache.items()}
    for b, n in enumerate(lens):
        old = n - int(np.diff(cu)[b]) - window - 10  # a token that no row sees any more
        if old > sinks:
            hidden["params"][table[b, old // 16], :, old % 16] = np.nan
    for c in (cache, hidden):
        got = sq.attn_tree(up(q), device_cache(c), ints(missing), ints(lens), ints(cu), most, **args)
        attention_close(got[up(~large)], want[~large], weight[~large], SCORES)
        assert torch.isnan(got[up(large)]).all()


def test_a_row_by_itself_and_in_company():
    """The same row alone and beside others a million times as large: the same up to the roundings."""
    g = rng(85)
    table, pages = spread_table(g, [300], 16)
    cache = device_cache(filled(g, pages, 2, 16, 4, np.float32))
    q = heads_of(g, 1, 8, 2.0 ** -16)
    scale = 128 ** -0.5 * 2.0 ** 16
    place = cache, ints(table), ints([300]), ints([0, 1])
    alone = f64(sq.attn_tree(up(q), *place, 300, scale=scale))
    for other in (0.0, 1.0, 60000.0, np.inf, np.nan):
        both = q.copy()
        both[0, [0, 5]] = other
        got = f64(sq.attn_tree(up(both), *place, 300, scale=scale))
        rest = [h for h in range(8) if h not in (0, 5)]
        assert np.abs(got[0, rest] - alone[0, rest]).max() <= 2 * (2.0 ** -11 + SCORES) * 8
