"""Attention of the paged cache and of prompts where queries, keys or scores leave the ordinary range.

What is NaN by the definition (a NaN score, scores that are all -inf, a score of +inf) is NaN, and
only there; a row without tokens is zero whatever its query holds.  Tolerances as in
tests/test_gpu_paged.py.
"""

import numpy as np
import pytest
import torch

from oracle import paged as opg
from paper_2405_16406_amd import sq
from test_gpu_paged import attention_close, device_cache, f64, filled, heads_of, ints, prompt_scores, rng, spread_table, up

pytestmark = pytest.mark.gpu

# (lengths, max_len): uncut sequences; chunks joined by one wave; by eight.  The last two sequences have
# no token and no page
PAGED_FORMS = {"uncut": ([40, 17, 0, 33], 64), "few_chunks": ([700, 300, 0, 90], 700), "many_chunks": ([2600, 30, 0, 900], 4096)}


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("form", PAGED_FORMS)
@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
def test_paged_attention_of_queries_not_finite(form, value, bits):
    lens, most = PAGED_FORMS[form]
    g = rng(51)
    Hq, H, page = 8, 2, 16
    table, pages = spread_table(g, lens, page)
    table[3] = pages
    cache = filled(g, pages, H, page, bits, np.float32)
    q = heads_of(g, 4, Hq)
    want, weight = opg.attn_paged(q, cache, lens, table, most)
    bad = np.zeros((4, Hq), dtype=bool)
    bad[0, 3] = bad[1, 6] = bad[2, 0] = bad[3, 5] = True
    q[bad, 7] = value
    got = f64(sq.attn_paged(up(q), device_cache(cache), ints(table), ints(lens), most))
    seen = bad & np.array([True, True, False, False])[:, None]
    assert np.all(np.isnan(got[seen]))
    attention_close(torch.from_numpy(got[~seen]), want[~seen], weight[~seen], 2e-5)
    assert np.all(got[2:] == 0)


# rows and keys of the sequences, heads: each form of the prompt's division (halves, whole tiles, parts);
# of the last sequence's three rows the first two see no key
PROMPT_FORMS = {"halves": ([200, 3], [200, 1], 2), "whole": ([90, 3], [90, 1], 300), "parts": ([40, 3], [3000, 1], 2)}


@pytest.mark.parametrize("form", PROMPT_FORMS)
@pytest.mark.parametrize("what", ["query", "only key", "score"])
def test_prompt_attention_of_rows_not_finite(form, what):
    nq, nk, H = PROMPT_FORMS[form]
    g = rng(52)
    cu_q, cu_k = (np.concatenate([[0], np.cumsum(n)]) for n in (nq, nk))
    n, m = int(cu_q[-1]), int(cu_k[-1])
    q, k, v = heads_of(g, n, H), heads_of(g, m, H), heads_of(g, m, H)
    want, weight, _ = opg.attn_prompt(q, k, v, cu_q, cu_k)
    scores = prompt_scores(q, k, 128 ** -0.5)
    bad = np.zeros((n, H), dtype=bool)
    q[-3, 1, 3] = q[-2, 0, 3] = np.nan  # these see nothing
    if what == "query":
        bad[5, 1] = bad[n - 1, 0] = True
        q[bad, 3] = np.nan
    else:  # the one key that the last row sees: a NaN, or a score of -inf
        bad[n - 1, 1] = True
        k[-1, 1, 3] = np.nan if what == "only key" else -np.inf
        q[n - 1, 1, 3] = 1
    got = f64(sq.attn_prompt(up(q), up(k), up(v), ints(cu_q), ints(cu_k)))
    assert np.all(np.isnan(got[bad]))
    attention_close(torch.from_numpy(got[~bad]), want[~bad], weight[~bad], scores)
    assert np.all(got[-3:-1] == 0)
