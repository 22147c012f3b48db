"""Attention where finite inputs make very large scores: the softmax stays one of finite numbers.

A softmax factor is 2^(s - m).  In fp32 s has steps of 2^-23 |s|, and from 2^24 on (base 2) these are
larger than 1: the difference must be that of the rounded numbers, or the largest factor is not 1 but
2 to the power of a rounding error.  The scores here are so far apart that rounding does not change
which is the largest, so the result is the value of that key (or the mean of equal ones), with the
tolerances of tests/test_gpu_paged.py.
"""

import numpy as np
import pytest

from oracle import paged as opg
from paper_2405_16406_amd import sq
from test_gpu_paged import attention_close, device_cache, filled, heads_of, ints, rng, spread_table, up

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("lens,most", [([60, 200], 256), ([900, 70], 900)], ids=["uncut", "chunks"])
@pytest.mark.parametrize("power", [*range(20, 32), 39])
def test_paged_attention_of_large_scores(power, lens, most, sign, bits):
    """k_beta = +-(1 + j 2^-10), j different for each token: scores of one query differ by 2^-10 of their
    size, 2^10 and more, where fp32 rounds them by 2^-22 of it; v_alpha's logarithm adds less than 8."""
    g = rng(71)
    H, page = 2, 16
    table, pages = spread_table(g, lens, page)
    cache = filled(g, pages, H, page, bits, np.float32)
    cache["k_q"][...] = 0
    order = np.stack([g.permutation(pages * page).reshape(pages, page) for _ in range(H)], axis=1)
    cache["params"][..., 0] = 1
    cache["params"][..., 1] = sign * (1 + order * 2.0 ** -10)
    q = np.zeros((2, 8, 128), dtype=np.float16)
    q[:, :, 5] = 1
    q[:, 3, 5] = 0  # a head of ordinary scores beside them
    scale = 1.37 * 2.0 ** power
    got = sq.attn_paged(up(q), device_cache(cache), ints(table), ints(lens), most, scale=scale)
    want, weight = opg.attn_paged(q, cache, lens, table, most, scale)
    attention_close(got, want, weight, 2e-5)


# rows and keys, heads: each form of the prompt's division (halves, whole tiles, parts)
PROMPT_FORMS = {"halves": ([200, 40], [300, 40], 2), "whole": ([90, 10], [130, 10], 300), "parts": ([40, 3], [3000, 3], 2)}


@pytest.mark.parametrize("form", PROMPT_FORMS)
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("power", [16, 20, 24, 25, 26, 28, 30, 39])
def test_prompt_attention_of_large_scores(power, sign, form):
    """Scores are +-(1 + j) scale, j from 0 to 2046: exact in the products, rounded once by the scale, and
    at least 2^16 apart unless equal."""
    nq, nk, H = PROMPT_FORMS[form]
    g = rng(72)
    cu_q, cu_k = (np.concatenate([[0], np.cumsum(n)]) for n in (nq, nk))
    n, m = int(cu_q[-1]), int(cu_k[-1])
    q, k, v = np.zeros((n, H, 128), np.float16), heads_of(g, m, H), heads_of(g, m, H)
    k[:, :, 9] = sign * (1 + np.stack([g.permutation(m) % 2047 for _ in range(H)], axis=1))
    q[:, :, 9] = 1
    q[::3, :, 9] = 0  # rows of ordinary scores among them
    scale = 1.37 * 2.0 ** power
    got = sq.attn_prompt(up(q), up(k), up(v), ints(cu_q), ints(cu_k), scale=scale)
    want, weight, _ = opg.attn_prompt(q, k, v, cu_q, cu_k, scale)
    attention_close(got, want, weight, 2.0 ** -18)
