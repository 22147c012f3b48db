"""Parameters that are not finite in tokens that some rows of a workgroup see and others do not, in every form of the
attention of several rows: one and two columns, four and eight waves, uncut and joined.

Tolerances as in tests/test_gpu_paged.py.
"""

import numpy as np
import pytest
import torch

from oracle import drafts as od
from paper_2405_16406_amd import sq
from test_gpu_paged import attention_close, device_cache, filled, heads_of, ints, rng, spread_table, up

pytestmark = pytest.mark.gpu

# Hq, Hkv, params, drafts, tokens before, window; tests/test_tree_forms_host.py has what each reaches
FORMS = {"one column": (8, 2, np.float32, [30], [100], 60), "eight waves": (8, 2, np.float16, [14], [1200], 1100),
         "two columns": (64, 8, np.float16, [33], [900], 700), "two columns, joined": (64, 8, np.float32, [40, 33], [2900, 2000], 2500),
         "one column, joined": (8, 2, np.float16, [12], [3200], 3000)}


@pytest.mark.parametrize("mode", ["tree", "chain"])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("form", FORMS)
def test_parameters_that_some_rows_see(form, bits, mode):
    Hq, H, dt, new, past, window = FORMS[form]
    g = rng(101 + bits)
    page, sinks, n = 16, 2, new[0]
    lens, cu = [a + b for a, b in zip(new, past)], np.concatenate([[0], np.cumsum(new)])
    table, pages = spread_table(g, lens, page)
    cache = filled(g, pages, H, page, bits, dt)
    q = heads_of(g, int(cu[-1]), Hq)
    parents = np.concatenate([np.maximum(np.arange(m) - g.integers(1, 4, m), -1) for m in new])
    sees, depth, _ = od.tree_mask(parents, cu, lens, window, sinks, 2)
    chain = mode == "chain"
    args = dict(window=window, sinks=sinks) | ({} if chain else dict(mask=up(od.words_of(sees, 2)), depth=ints(depth)))
    want, weight, _ = od.attn_tree(q, cache, cu, lens, table, max(lens), None if chain else sees, None if chain else depth, window, sinks)
    base, at = past[0], range(n) if chain else depth
    half = int(np.median(list(at)[:n]))
    lost = base + half - window  # rows at `half` and deeper have left this token behind
    draft = n // 2
    for t, see in ((lost, [at[i] < half for i in range(n)]),
                   (base + draft, [i >= draft if chain else draft in sees[i] for i in range(n)])):
        see = np.array(see + [False] * (len(q) - n))
        assert t >= sinks and see.any() and not see[:n].all()
        # all four parameters, or the value's offset alone, which gives infinite values and ordinary weights
        for what, x in ((slice(0, 4), np.nan), (slice(0, 4), np.inf), (3, np.inf), (3, np.nan)):
            c = {name: a.copy() for name, a in cache.items()}
            c["params"][table[0, t // page], :, t % page, what] = x
            got = sq.attn_tree(up(q), device_cache(c), ints(table), ints(lens), ints(cu), max(lens), **args)
            attention_close(got[up(~see)], want[~see], weight[~see], 2e-5)
            if what == 3 and x == np.inf:
                assert torch.all(got[up(see)] == np.inf)
            else:
                assert torch.isnan(got[up(see)]).all()
