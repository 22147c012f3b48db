"""Page tables on the GPU against oracle/drafts.py: pages back to the pool, pages, lengths and rows of a step."""

import numpy as np
import pytest
import torch

from oracle import drafts as od
from paper_2405_16406_amd import sq
from test_gpu_paged import DEV, ints, rng

pytestmark = pytest.mark.gpu


def state(g, held, cols, spare):
    """A table in which sequence b holds held[b] blocks, and a pool with `spare` free pages."""
    pages = sum(held) + spare
    order = [int(x) for x in g.permutation(pages)]
    table = np.full((len(held), cols), -1, dtype=np.int64)
    at = 0
    for b, n in enumerate(held):
        table[b, :n] = order[at:at + n]
        at += n
    return table, order[at:] + [-9] * at, spare


def check_grow(have, add, held, table, page, pool, count, rows):
    o = od.paged_grow(have, add, held, table, page, pool, count, rows)
    wide = torch.full((len(held), table.shape[1] + 2), 77, dtype=torch.int32, device=DEV)
    t = wide[:, :table.shape[1]]
    t.copy_(ints(table))
    h, p, c = ints(held), ints(pool), ints([count])
    lens, cu, pos, slots, missing = sq.paged_grow(ints(have), ints(add), h, t, page, p, c, rows)
    for name, got in (("lens", lens), ("cu", cu), ("pos", pos), ("slots", slots), ("missing", missing), ("held", h)):
        assert got.tolist() == [int(x) for x in o[name]], name
    assert np.array_equal(t.cpu().numpy(), o["table"]) and torch.all(wide[:, table.shape[1]:] == 77)
    assert p.tolist() == list(pool)
    good = o["missing"] == (0, 0)
    assert c.item() == (o["count"] if good else count)
    return o


GROW = [  # tokens before, new ones, blocks held beyond what they need, page, columns beside the most needed, spare pages, rows beside
    ([0], [1], [0], 16, 0, 1, 0),
    ([15, 16, 17, 0], [1, 1, 1, 0], [0, 0, 0, 0], 16, 0, 5, 0),
    ([100, 3, 0, 64], [16, 16, 300, 1], [0, 2, 0, 1], 32, 3, 40, 7),
    ([5] * 1030, [1, 12] * 515, [0] * 1030, 16, 1, 700, 1),        # more sequences than one batch, rows by the second kernel
    ([0, 7], [5000, 3000], [0, 0], 16, 0, 600, 3),
    ([0] * 2100, [0] * 2100, [0] * 2100, 128, 1, 1, 5),
    ([9] * 3000, [1] * 3000, [0] * 3000, 16, 0, 3, 2),
]


@pytest.mark.parametrize("case", GROW, ids=lambda c: f"{len(c[0])}-p{c[3]}-{sum(c[1])}")
def test_grow(case):
    have, add, more, page, cols, spare, rows = case
    g = rng(len(have))
    held = [-(-h // page) + m for h, m in zip(have, more)]
    most = max(max(-(-(h + a) // page) for h, a in zip(have, add)), max(held), 1)
    table, pool, count = state(g, held, most + cols, spare)
    o = check_grow(have, add, held, table, page, pool, count, sum(add) + rows)
    assert o["missing"] == (0, 0)


def test_grow_takes_odd_numbers():
    """Values below 0, blocks beyond the table, entries that are no pages: what they count as."""
    g = rng(1)
    table, pool, count = state(g, [3, 2, 4], 5, 9)
    table[0, 1], table[2, 3] = 999, -4
    check_grow([-5, 20, 50], [33, -7, 20], [3, -1, 77], table, 16, pool, count, 60)
    check_grow([10, 20, 50], [10, 1, 1], [3, 2, 4], table, 16, pool, 1 << 30, 60)  # a count beyond the pool


@pytest.mark.parametrize("rows", [60, 5000])
@pytest.mark.parametrize("what", ["pages", "columns", "rows", "all", "tokens"])
def test_grow_or_nothing(what, rows):
    g = rng(2)
    table, pool, count = state(g, [1, 0, 2], 4, 3)
    have, add = [10, 0, 20], [20, 16, 10]
    if what == "pages":
        count = 1
    if what in ("columns", "all"):
        add[1] = 16 * 5 + 1
    if what in ("rows", "all"):
        rows = 45
    if what == "tokens":
        have[1], add[1] = 2 ** 31 - 10, 2 ** 31 - 1
    o = check_grow(have, add, [1, 0, 2], table, 16, pool, count, rows)
    assert o["missing"] != (0, 0) and o["cu"][-1] == 0 and set(o["slots"]) == {-1}


def test_grow_without_sequences():
    lens, cu, pos, slots, missing = sq.paged_grow(ints([]), ints([]), ints([]), ints([]).view(0, 1), 16, ints([0]), ints([1]), 4)
    assert cu.tolist() == [0] and pos.tolist() == slots.tolist() == [-1] * 4 and missing.tolist() == [0, 0]


def check_release(table, page, first, end, held, pool, count):
    want = od.paged_release(table, page, first, end, held, pool, count)
    t, h, p, c = ints(table), ints(held), ints(pool), ints([count])
    sq.paged_release(t, page, ints(first), ints(end), h, p, c)
    assert np.array_equal(t.cpu().numpy(), want[0]) and h.tolist() == want[1]
    assert p.tolist() == want[2] and c.item() == want[3]
    return want


def test_release():
    g = rng(3)
    big = 2 ** 31 - 1
    held = [4, 3, 0, 6, 5, 2, 1]
    table, pool, count = state(g, held, 8, 4)
    table[3, 2], table[4, 0] = -1, 10 ** 6
    # a whole sequence, behind 20 tokens, nothing held, a window's middle, an end inside a page, before the first, first behind the end
    check_release(table, 16, [0, 20, 0, 17, 0, -50, 40], [big, big, big, 79, 33, -1, 3], held, pool, count)
    check_release(table, 16, [0] * 7, [big] * 7, [99, -2, 3, 6, 5, 2, 1], pool, count)  # held beyond and below the table
    check_release(table, 16, [16] * 7, [64] * 7, held, pool, count)


@pytest.mark.parametrize("B,blocks", [(2500, 3), (3, 5000), (1, 1)])
def test_release_of_many(B, blocks):
    g = rng(B)
    held = [int(x) for x in g.integers(0, blocks + 1, B)]
    held[0] = blocks
    table, pool, count = state(g, held, blocks + 1, 7)
    first = [int(x) for x in g.integers(0, 16 * blocks, B)]
    end = [int(x) if g.random() < 0.5 else 2 ** 31 - 1 for x in g.integers(0, 16 * blocks, B)]
    check_release(table, 16, first, end, held, pool, count)


def test_a_pool_that_is_full():
    """More pages come back than the pool has room for (one was released twice): none is written past its end."""
    g = rng(5)
    table, pool, count = state(g, [3, 3], 3, 0)
    table[1] = table[0]
    wide = torch.full((9,), 55, dtype=torch.int32, device=DEV)
    p = wide[1:7]
    p.copy_(ints(pool))
    want = od.paged_release(table, 16, [0, 0], [99, 99], [3, 3], pool, 2)
    c = ints([2])
    sq.paged_release(ints(table), 16, ints([0, 0]), ints([99, 99]), ints([3, 3]), p, c)
    assert p.tolist() == want[2] and c.item() == 6 and wide[0] == 55 and torch.all(wide[7:] == 55)


def test_steps_of_a_server():
    """Many steps: sequences come, grow, lose drafts and end; no page is ever in two places."""
    g = rng(7)
    B, page, cols, pages = 9, 16, 12, 70
    table = ints(np.full((B, cols), -1))
    held, pool, count = ints([0] * B), ints(g.permutation(pages)), ints([pages])
    have, big = [0] * B, 2 ** 31 - 1
    for step in range(25):
        first, add = [], []
        for b in range(B):
            if g.random() < 0.15:
                have[b] = 0  # ended: another prompt takes its place
            first.append(have[b])
            add.append(int(g.integers(1, 50)) if have[b] == 0 else int(g.integers(0, 6)))
            if have[b] + add[b] > cols * page:
                add[b] = 0
        before = [t.cpu().numpy().tolist() for t in (table, held, pool, count)]
        o = od.paged_release(np.array(before[0]), page, first, [big] * B, before[1], before[2], before[3][0])
        sq.paged_release(table, page, ints(first), ints([big] * B), held, pool, count)
        lens, cu, pos, slots, missing = sq.paged_grow(ints(have), ints(add), held, table, page, pool, count, sum(add))
        w = od.paged_grow(have, add, o[1], o[0], page, o[2], o[3], sum(add))
        assert lens.tolist() == w["lens"] and slots.tolist() == list(w["slots"]) and missing.tolist() == list(w["missing"])
        assert np.array_equal(table.cpu().numpy(), w["table"]) and count.item() == w["count"]
        inside = [int(table[b, c]) for b in range(B) for c in range(int(held[b]))]
        free = pool[:count.item()].tolist()
        assert sorted(inside + free) == list(range(pages))
        if missing.tolist() == [0, 0]:
            have = [n - min(int(g.integers(0, 3)), a) for n, a in zip(lens.tolist(), add)]
