"""Slots of the cache that were never written: both ways to the attention read them as zeros."""

import numpy as np
import pytest

from oracle import paged as opg
from paper_2405_16406_amd import sq
from test_gpu_paged import attention_close, device_cache, filled, heads_of, ints, rng, spread_table, up

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dt", [np.float32, np.float16])
@pytest.mark.parametrize("lens,most", [([150, 40], 150), ([700, 90], 700)], ids=["uncut", "chunks"])
@pytest.mark.parametrize("offset", [0.0, 0.25])
def test_value_scales_of_zero(lens, most, dt, bits, offset):
    """v_alpha 0 and codes 0, as in a zeroed cache: the value is v_beta; the token keeps its part in the
    softmax (k_alpha 0 gives the score k_beta sum(q)).  Beside the tokens' factor, which is
    1 for these and v_alpha (2^-6 .. 1) otherwise, all fp16 weights stay normal numbers."""
    g = rng(61)
    H, page = 2, 16
    table, pages = spread_table(g, lens, page)
    cache = filled(g, pages, H, page, bits, dt)
    empty = g.random((pages, H, page)) < 0.3
    cache["params"][empty] = 0
    cache["params"][empty, 3] = offset
    for n in ("k_q", "v_q"):
        cache[n][empty] = 0
    q = heads_of(g, 2, 8)
    got = sq.attn_paged(up(q), device_cache(cache), ints(table), ints(lens), most)
    want, weight = opg.attn_paged(q, cache, lens, table, most)
    attention_close(got, want, weight, 2e-5)


def test_a_zeroed_cache():
    g = rng(62)
    cache = sq.kv_cache(5, 16, 2)
    got = sq.attn_paged(up(heads_of(g, 1, 8)), cache, ints([[4, 2, 0]]), ints([41]), 41)
    assert not got.any()
