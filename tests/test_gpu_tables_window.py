"""Pages that a moving window leaves behind, given back step by step while sequences grow, lose drafts and end: with
`first` from the end of the call before, the pool, the table and what a window's attention reads are those of calls
that look at everything from the first tokens on."""

import numpy as np
import pytest
import torch

from oracle import drafts as od
from paper_2405_16406_amd import sq
from test_gpu_paged import DEV, device_cache, filled, heads_of, ints, rng, up

pytestmark = pytest.mark.gpu

BIG = 2 ** 31 - 1


@pytest.mark.parametrize("page,window,sinks", [(16, 40, 4), (16, 33, 0), (32, 64, 33), (16, 1, 16), (16, 100, 70)])
def test_a_window_that_moves(page, window, sinks):
    g = rng(page + window)
    B, cols, pages, Hq, H = 5, 40, 150, 4, 2
    table, held, pool, count = ints(np.full((B, cols), -1)), ints([0] * B), ints(g.permutation(pages)), ints([pages])
    have, past = ints([0] * B), ints([0] * B)  # tokens, and the end of the last release
    freq = up(np.ones(64))
    cache, whole = sq.kv_cache(pages, page, H), sq.kv_cache(B * cols, page, H)
    every = ints(np.arange(B * cols).reshape(B, cols))  # a table that keeps all pages
    released = 0
    for step in range(60):
        tokens = have.tolist()
        add = [int(g.integers(1, 30)) if n + 30 <= cols * page else 0 for n in tokens]
        lens, cu, pos, slots, missing = sq.paged_grow(have, ints(add), held, table, page, pool, count, sum(add))
        assert missing.tolist() == [0, 0]
        T = sum(add)
        q, k, v = (up(heads_of(g, T, h)) for h in (Hq, H, H))
        if T:
            qr = sq.rope_kv_write(q, k, v, cache, table, lens, freq, cu=cu)
            sq.rope_kv_write(q, k, v, whole, every, lens, freq, cu=cu)
            got = sq.attn_tree(qr, cache, table, lens, cu, cols * page, window=window, sinks=sinks)
            assert torch.equal(got, sq.attn_tree(qr, whole, every, lens, cu, cols * page, window=window, sinks=sinks)), step
        # some of the new tokens are taken back, some sequences end
        over = [bool(g.random() < 0.04) for _ in range(B)]
        kept = [0 if o else n - int(g.integers(0, min(a, 5) + 1)) for n, a, o in zip(lens.tolist(), add, over)]
        have = ints(kept)
        sq.paged_release(table, page, have, ints([BIG] * B), held, pool, count)
        end = have - window
        before = [x.cpu().numpy().tolist() for x in (table, held, pool, count)]
        want = od.paged_release(np.array(before[0]), page, [sinks] * B, end.tolist(), before[1], before[2], before[3][0])
        past = torch.where(have == 0, 0, past)
        first = (past // page * page).clamp(min=sinks).to(torch.int32)
        sq.paged_release(table, page, first, end, held, pool, count)
        past = torch.maximum(past, end).to(torch.int32)
        assert np.array_equal(table.cpu().numpy(), want[0]) and held.tolist() == want[1]
        assert pool.tolist() == want[2] and count.item() == want[3]
        released += count.item() - before[3][0]
        inside = [x for x in table.flatten().tolist() if x >= 0]
        assert sorted(inside + pool[:count.item()].tolist()) == list(range(pages))
    assert released > 40


def test_a_window_that_moves_in_a_graph():
    """Tables, `first` and `end` on the device: a captured step replayed against the eager one."""
    g = rng(3)
    B, cols, pages, page, window, sinks = 3, 30, 80, 16, 48, 5
    add = ints([7, 1, 16])

    def state():
        return dict(table=ints(np.full((B, cols), -1)), held=ints([0] * B), pool=ints(range(pages)), count=ints([pages]),
                    have=ints([0] * B), past=ints([0] * B))

    def step(s):
        lens, *_ = sq.paged_grow(s["have"], add, s["held"], s["table"], page, s["pool"], s["count"], 24)
        s["have"].copy_(lens)
        end = lens - window
        sq.paged_release(s["table"], page, (s["past"] // page * page).clamp(min=sinks).to(torch.int32), end, s["held"], s["pool"], s["count"])
        s["past"].copy_(torch.maximum(s["past"], end))

    eager, captured = state(), state()
    step(state())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(captured)
    for turn in range(28):
        step(eager)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(eager[k], captured[k]) for k in eager), turn
    assert eager["have"].tolist() == [28 * 7, 28, 28 * 16]
    for b, n in enumerate(eager["have"].tolist()):
        row = eager["table"][b].tolist()
        gone = range(-(-sinks // page), max(0, n - window) // page)
        assert all(row[c] == -1 for c in gone) and all(row[c] >= 0 for c in range(-(-n // page)) if c not in gone)
