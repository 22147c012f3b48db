"""Sizes of the paged calls at which the kernels loop: workgroups of several tokens in the write, waves
with several blocks of tokens and joins of many chunks in the decode attention, searches through more
than 64 sequences.  tests/test_paged_host.py checks that the cases reach these forms.

Tolerances as in tests/test_gpu_paged.py.
"""

import numpy as np
import pytest
import torch

from oracle import paged as opg
from paper_2405_16406_amd import sq
from test_gpu_paged import (DEV, attention_close, check_write, device_cache, filled, heads_of, ints, prompt_scores, rng, spread_table,
                            up)

pytestmark = pytest.mark.gpu


# Hq, Hkv, page, bits, params, rotary, interleaved, clip, rows in all, tokens a workgroup
WRITE = [
    (64, 8, 16, 4, np.float32, 128, False, 1.0, 1100, 1),   # four waves with six tasks
    (8, 2, 32, 4, np.float32, 128, False, 1.0, 2049, 2),
    (32, 8, 16, 8, np.float16, 128, True, 0.95, 2051, 2),
    (5, 1, 16, 8, np.float32, 64, False, 1.0, 4099, 4),
    (8, 2, 16, 4, np.float16, 96, False, 0.9, 4097, 4),
    (4, 4, 16, 4, np.float32, 128, False, 0.9, 8197, 8),
    (3, 1, 64, 8, np.float32, 32, True, 1.0, 8193, 8),
    (3, 3, 16, 4, np.float32, 0, False, 1.0, 8193, 8),
]


@pytest.mark.parametrize("case", WRITE, ids=lambda c: f"{c[0]}x{c[1]}-b{c[3]}-{np.dtype(c[4]).name}-r{c[5]}{'i' if c[6] else 'h'}-{c[8]}")
def test_write_of_many_rows(case):
    """Sequences of 1 to 60 rows, some empty, so that borders and missing pages lie inside workgroups."""
    Hq, H, page, bits, dt, rotary, inter, clip, T, _ = case
    g = rng(T)
    new = []
    while sum(new) < T - 8:
        new.append(min(int(g.choice([0, 1, 2, 7, 33, 60])), T - 8 - sum(new)))
    past = [int(x) for x in g.integers(0, 50, len(new))]
    lens = [n + p for n, p in zip(new, past)]
    lens[1] = max(0, new[1] - 2)  # its first two rows (of two or more) have no position
    cu = np.concatenate([[3], 3 + np.cumsum(new)])  # three rows before the first sequence, five behind the last
    table, pages = spread_table(g, lens, page)
    table[g.random(table.shape) < 0.05] = pages + 7
    q, k, v = (heads_of(g, T, h) for h in (Hq, H, H))
    freq = opg.rope_frequencies(rotary, 10000.0) if rotary else None
    cache = filled(g, pages, H, page, bits, dt)
    o = opg.rope_kv_write(q, k, v, cache, cu, lens, table, freq, inter, 1.0, clip, clip)
    assert 0 < (o["where"][o["rows"]] < 0).sum() < T // 4
    dc = device_cache(cache)
    out = torch.full((T, Hq, 128), 7.0, dtype=torch.float16, device=DEV)
    k_out = torch.full((T, H, 128), 7.0, dtype=torch.float16, device=DEV)
    sq.rope_kv_write(up(q), up(k), up(v), dc, ints(table), ints(lens), None if freq is None else up(freq), cu=ints(cu), interleaved=inter,
                     k_clip=clip, v_clip=clip, out=out, k_out=k_out)
    torch.cuda.synchronize()
    check_write(o, out, dc, q, bits, o["rows"])
    left = torch.tensor(~o["rows"], device=DEV)
    assert torch.all(out[left] == 7.0) and torch.all(k_out[left] == 7.0)
    kr = o["k_rot"][o["rows"]]
    assert np.all(np.abs(k_out[~left].cpu().numpy().astype(np.float64) - kr) <= 2.0 ** -11 * 1.001 * np.abs(kr) + 2.0 ** -25)
    # the same rows in calls of one token a workgroup give the same bytes
    dc2 = device_cache(cache)
    out2 = torch.full_like(out, 7.0)
    for t0 in range(0, T, 1000):
        part = slice(t0, min(t0 + 1000, T))
        n = part.stop - t0
        # a row's position is lens - cu[b + 1] + t: the call on rows t0 .. has cu and the rows shifted alike
        sq.rope_kv_write(up(q[part]), up(k[part]), up(v[part]), dc2, ints(table), ints(lens), None if freq is None else up(freq),
                         cu=ints(cu - t0), interleaved=inter, k_clip=clip, v_clip=clip, out=out2[part])
        assert n <= 1000
    assert torch.equal(out, out2) and all(torch.equal(a, b) for a, b in zip(dc, dc2))


# Hq, Hkv, page, bits, params, lens, max_len, how the scores go along the sequence
PAGED = [
    (8, 2, 16, 4, np.float32, [3000, 769, 1], 1 << 20, "flat"),      # several blocks of 64 tokens for each wave
    (8, 2, 16, 4, np.float32, [3000, 1500, 700], 1 << 20, "rising"),
    (4, 4, 64, 8, np.float16, [2500, 1100, 0], 1 << 20, "rising"),
    (17, 1, 32, 8, np.float32, [2900, 260], 1 << 20, "falling"),
    (4, 2, 128, 4, np.float16, [3333, 4000], 1 << 20, "steep"),
    (4, 2, 16, 8, np.float16, [3333], 1 << 18, "steep"),
    (16, 1, 16, 4, np.float32, [5000], 131072, "rising"),            # chunks joined by eight waves, one round
    (2, 1, 16, 8, np.float32, [17100], 131072, "rising"),            # and two
    (2, 1, 64, 4, np.float16, [20001], 131072, "steep"),
]


@pytest.mark.parametrize("case", PAGED, ids=lambda c: f"{c[0]}x{c[1]}-b{c[3]}-{np.dtype(c[4]).name}-{max(c[5])}of{c[6]}-{c[7]}")
def test_paged_attention_over_many_blocks(case):
    """Scores that rise by 8 (rising) or 40 (steep) in natural units move the running maximum on states that
    are not empty.  Missing pages lie in every part of the sequences."""
    Hq, H, page, bits, dt, lens, most, way = case
    g = rng(Hq * bits + max(lens))
    B = len(lens)
    table, pages = spread_table(g, lens, page)
    cache = filled(g, pages, H, page, bits, dt)
    q = heads_of(g, B, Hq)
    rise = {"flat": 0.0, "rising": 8.0, "falling": -8.0, "steep": 40.0}[way]
    for b, n in enumerate(lens):
        cols = -(-n // page)
        for c in range(cols):  # the offsets k_beta raise the scores of sum(q) = 128
            step = rise / 128 ** 0.5 * (np.arange(page) + c * page) / max(n, 1)
            beta = cache["params"][table[b, c], :, :, 1].astype(np.float64) + step
            cache["params"][table[b, c], :, :, 1] = beta.astype(dt)
        table[b, :cols][g.random(cols) < 0.04] = -1
    q = (q.astype(np.float64) + (128 - q.astype(np.float64).sum(-1, keepdims=True)) / 128).astype(np.float16)
    got = sq.attn_paged(up(q), device_cache(cache), ints(table), ints(lens), most)
    want, weight = opg.attn_paged(q, cache, lens, table, most)
    # scores: 34 roundings in the sum of q, four in two chained products, two in the sums with k_beta and
    # log2 v_alpha, each of 2^-24 of sum |q| (|k_alpha c| + |k_beta|) at most
    top = 2.0 ** bits - 1
    p = np.abs(cache["params"].astype(np.float64))
    size = np.abs(q.astype(np.float64)).sum(-1).max() * (p[..., 0] * top + p[..., 1]).max() / 128 ** 0.5
    attention_close(got, want, weight, 2.0 ** -24 * 40 * size + 2.0 ** -18)
    assert torch.equal(got, sq.attn_paged(up(q), device_cache(cache), ints(table), ints(lens), most))


def many(count, seed, sizes):
    g = np.random.Generator(np.random.PCG64(seed))
    return [int(x) for x in g.choice(sizes, count)]


# Hq, Hkv, queries, keys: more than 64 sequences
PROMPT = [
    (8, 8, many(130, 1, [0, 1, 5, 30]), many(130, 2, [0, 1, 9, 60])),         # whole tiles
    (4, 2, many(100, 3, [0, 1, 3, 8]), many(100, 4, [0, 2, 40, 70])),         # halves
    (2, 1, many(66, 5, [0, 1, 2]), [*many(64, 6, [0, 100, 1000]), 90000, 170000]),  # parts
]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("case", PROMPT, ids=["whole", "halves", "parts"])
def test_prompt_attention_of_many_sequences(case, causal):
    Hq, H, nq, nk = case
    g = rng(sum(nq))
    cu_q, cu_k = (np.concatenate([[0], np.cumsum(n)]) for n in (nq, nk))
    Tq, Tk = int(cu_q[-1]) + 1, int(cu_k[-1])
    q, k, v = heads_of(g, Tq, Hq), heads_of(g, Tk, H), heads_of(g, Tk, H)
    out = torch.full((Tq, Hq, 128), 7.0, dtype=torch.float16, device=DEV)
    sq.attn_prompt(up(q), up(k), up(v), ints(cu_q), ints(cu_k), causal=causal, out=out)
    want, weight, rows = opg.attn_prompt(q, k, v, cu_q, cu_k, causal=causal)
    attention_close(out[torch.tensor(rows, device=DEV)], want[rows], weight[rows], prompt_scores(q, k, 128 ** -0.5))
    assert torch.all(out[-1] == 7.0)
