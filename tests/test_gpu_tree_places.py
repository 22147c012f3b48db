"""Sequences with more drafts than tokens: the first drafts have no place in the cache, and positions below 0.

Tolerances as in tests/test_gpu_paged.py.
"""

import numpy as np
import pytest
import torch

from oracle import drafts as od
from paper_2405_16406_amd import sq
from test_gpu_paged import DEV, attention_close, device_cache, filled, heads_of, ints, rng, spread_table, up

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("window,sinks", [(0, 0), (0, 3), (2, 0), (3, 1), (2, 9), (30, 0)])
def test_drafts_without_a_place(window, sinks, bits):
    g = rng(111)
    Hq, H, page = 8, 2, 16
    new, lens = [36, 4, 9, 20], [29, 0, 60, 3]
    cu = np.concatenate([[0], np.cumsum(new)])
    table, pages = spread_table(g, lens, page)
    cache = filled(g, pages, H, page, bits, np.float32)
    parents = np.concatenate([[int(g.integers(-1, i + 1)) for i in range(n)] for n in new])
    sees, depth, rows = od.tree_mask(parents, cu, lens, window, sinks, 2)
    mask, d = sq.tree_mask(ints(parents), ints(cu), max(new), ints(lens), window, sinks)
    assert np.array_equal(mask.cpu().numpy(), od.words_of(sees, 2)) and np.array_equal(d.cpu().numpy(), depth)
    q = heads_of(g, int(cu[-1]), Hq)
    for tree in (dict(mask=mask, depth=d), {}):
        out = torch.full((len(q), Hq, 128), 7.0, dtype=torch.float16, device=DEV)
        sq.attn_tree(up(q), device_cache(cache), ints(table), ints(lens), ints(cu), 64, window=window, sinks=sinks, out=out, **tree)
        want, weight, rows = od.attn_tree(q, cache, cu, lens, table, 64, sees if tree else None, depth if tree else None, window, sinks)
        assert rows.sum() == 29 + 0 + 9 + 3
        attention_close(out[up(rows)], want[rows], weight[rows], 2e-5)
        assert torch.all(out[up(~rows)] == 7.0)
