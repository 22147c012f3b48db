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
from test_gpu_paged import attention_close, device_cache, filled, ints, rng, spread_table, up

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
