"""Runs of tokens and splits of the attention of several rows over the pages (csrc/paged.h, paged_plan.h compiled
alone, no GPU), and the oracle's own pins."""

import ctypes
import os
import random
import subprocess

import numpy as np
import pytest

from oracle import drafts as od
from oracle import paged as opg
from paper_2405_16406_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))
I64 = ctypes.c_int64


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("drafts") / "drafts.so")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", f"-I{build.CSRC}", os.path.join(HERE, "drafts_host.cpp"),
                        "-o", out], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return ctypes.CDLL(out)


def run_of(host, low, end, window, sinks):
    out = (ctypes.c_int32 * 3)()
    host.token_run(low, end, window, sinks, out)
    return tuple(out)


def plan_of(host, B, T, max_len, window=0, sinks=0, hq=32, hkv=8, single=False, cus=256):
    out = (ctypes.c_int32 * 4)()
    host.tree_plan(I64(B), I64(T), int(single), I64(max_len), window, sinks, hq, hkv, cus, out)
    return tuple(out)


def test_a_run_holds_what_its_rows_see(host):
    """Every token that a row at `low` or later sees before `end`, each once, and whole blocks of 64 in order."""
    rng = random.Random(1)
    for _ in range(1500):
        low, rows = rng.randrange(-5, 900), rng.randrange(1, 90)
        window = rng.choice([0, 1, 2, 63, 64, 65, rng.randrange(1, 1000)])
        sinks = rng.choice([0, 1, 4, 64, 65, rng.randrange(300)])
        end = rng.choice([low + rows, low + 1, rng.randrange(0, 1000)])
        head, start, tokens = run_of(host, low, end, window, sinks)
        places = [host.run_position(head, start, x) for x in range(tokens)]
        assert places == sorted(set(places)) and all(0 <= x < max(end, 0) for x in places)
        for p in range(low, low + rows):
            assert {t for t in range(min(p + 1, end)) if od.in_window(t, p, window, sinks)} <= set(places)
        assert head % 64 == 0 and start % 64 == 0
        if window:
            assert tokens <= sinks + 63 + window + 63 + max(0, end - low)
        else:
            assert (head, start, tokens) == (0, 0, max(end, 0))


def test_runs_at_the_ends_of_32_bits(host):
    most = 2 ** 30
    assert run_of(host, most - 2, most - 1, most - 1, most - 1) == (0, 0, most - 1)
    assert run_of(host, most - 2, most - 1, 1, most - 1)[2] <= most - 1
    assert run_of(host, -2 ** 24, 5, most - 1, 0) == (0, 0, 5)
    assert run_of(host, 0, -7, 3, 3) == (0, 0, 0)


def test_plans_cover_every_row_and_token(host):
    rng = random.Random(2)
    for _ in range(4000):
        hkv = rng.choice([1, 2, 8, 32])
        group = rng.choice([1, 4, 8, 17, 33])
        B = int(2 ** rng.uniform(0, 8))
        counts = [int(2 ** rng.uniform(0, 8)) - 1 for _ in range(B)]
        T = sum(counts)
        if T == 0:
            continue
        max_len = int(2 ** rng.uniform(0, 29))
        window, sinks = rng.choice([(0, 0), (0, 77), (int(2 ** rng.uniform(0, 20)), rng.choice([0, 4, 1000]))])
        cus = rng.choice([256, 304, 64, 1])
        rb, tiles, chunks, tokens = plan_of(host, B, T, max_len, window, sinks, group * hkv, hkv, cus=cus)
        assert rb in (1, 2) and tokens % 256 == 0 and chunks >= 1
        assert tiles >= sum(-(-n * group // (16 * rb)) for n in counts)
        assert tiles <= (T * group + B * (16 * rb - 1)) // (16 * rb)
        # the longest run of a tile fits its chunks
        most = max(counts)
        for length in (max_len, rng.randrange(1, max_len + 1)):
            base = length - most
            for low, end in ((base, length), (base + rng.randrange(most), length)):
                assert run_of(host, low, min(end, max_len), window, sinks)[2] <= chunks * tokens
        assert tiles * hkv * chunks < 2 ** 24 + 16 * cus * tiles  # (a grid of 256 threads a workgroup)
        single = plan_of(host, B, B, max_len, window, sinks, group * hkv, hkv, True, cus)
        assert single[1] == B * -(-group // (16 * single[0]))
        assert run_of(host, max_len - 1, max_len, window, sinks)[2] <= single[2] * single[3]


def test_the_largest_grids(host):
    """2^24 rows and heads, one long sequence or many, stay below 2^32 threads."""
    for B, T, hq, hkv in ((1, 2 ** 18 - 2, 64, 8), (2 ** 17 - 1, 2 ** 17, 64, 64), (1, 1, 2 ** 16, 2 ** 16), (2 ** 23 - 1, 2 ** 23, 1, 1),
                          (1, 2 ** 24 - 2, 1, 1)):
        for max_len in (1, 2 ** 30 - 1):
            rb, tiles, chunks, _ = plan_of(host, B, T, max_len, hq=hq, hkv=hkv)
            assert tiles * hkv * chunks < 2 ** 24, (B, T, hq, hkv, tiles, chunks)


def test_plans_of_known_sizes(host):
    """The measured choices."""
    assert plan_of(host, 1, 16, 2064)[0] == 1            # 12.8 us, two columns 13.5
    assert plan_of(host, 1, 64, 131072)[0] == 2
    assert plan_of(host, 1, 4, 131072)[0] == 1           # 16 rows are one column
    assert plan_of(host, 64, 64, 8192, 2048, 4, 64, 8, True)[2] == 1  # equal runs, uncut


def test_every_form_is_tested(host):
    """The sizes of tests/test_gpu_tree.py reach one and two columns, uncut tiles, and both joins."""
    t = pytest.importorskip("test_gpu_tree")
    forms = set()
    for hq, h, _, bits, _, new, past, window, sinks in t.ATTN:
        rb, _, chunks, _ = plan_of(host, len(new), sum(new) + 3, max(n + p for n, p in zip(new, past)), window, sinks, hq, h)
        forms.add((bits, rb, "one" if chunks == 1 else "few" if chunks <= 8 else "many"))
    assert {(b, r) for b, r, _ in forms} == {(4, 1), (4, 2), (8, 1), (8, 2)}
    assert {c for _, _, c in forms} == {"one", "few", "many"}
    assert {c for _, r, c in forms if r == 2} >= {"few"}


def test_every_kernel_is_tested(host):
    """Codes, parameters, columns and waves of the kernels that those sizes reach, and whether their runs are cut."""
    t = pytest.importorskip("test_gpu_tree")
    forms = set()
    for hq, h, _, bits, params, new, past, window, sinks in t.ATTN:
        args = (len(new), sum(new) + 3, max(n + p for n, p in zip(new, past)), window, sinks, hq, h)
        rb, _, chunks, _ = plan_of(host, *args)
        waves = host.tree_waves(I64(args[0]), I64(args[1]), 0, I64(args[2]), *args[3:], 256)
        forms.add((bits, np.dtype(params).itemsize, rb, waves, chunks > 1))
    for bits in (4, 8):
        for size in (2, 4):
            assert {f[2:] for f in forms if f[:2] == (bits, size)} >= {(1, 4, True), (1, 8, False), (2, 4, True)}, (bits, size)


def test_short_runs_of_few_workgroups_stay_uncut(host):
    def waves(B, T, run, single=0, hq=32, hkv=8, cus=256):
        plan = plan_of(host, B, T, run, hq=hq, hkv=hkv, single=bool(single), cus=cus)
        w = host.tree_waves(I64(B), I64(T), single, I64(run), 0, 0, hq, hkv, cus)
        assert w in (4, 8) and plan[3] % (64 * w) == 0 and plan[2] * plan[3] >= run and (w == 4 or (plan[0] == 1 and plan[2] == 1))
        return w
    assert [waves(1, 16, n) for n in (1, 256, 257, 1280, 1281, 2 ** 30 - 1)] == [4, 4, 8, 8, 4, 4]
    assert [waves(n, n, 1000, 1) for n in (1, 32, 33, 64)] == [8, 8, 4, 4]  # a workgroup for each compute unit
    assert waves(1, 64, 1200, cus=64) == 4


# ------------------------------------------------------------------ the oracle

def test_oracle_of_a_chain_is_causal_attention():
    g = np.random.default_rng(3)
    from test_gpu_paged import filled
    cache = filled(g, 6, 2, 16, 4, np.float32)
    table = np.array([[3, 1, 0], [2, 4, 5]])
    q = g.standard_normal((9, 4, 128))
    out, _, rows = od.attn_tree(q, cache, [0, 5, 9], [40, 9], table, 48)
    k, v, _ = opg.kv_read(cache, [0, 40, 49], [40, 9], table, 49)
    want, _, _ = opg.attn_prompt(q, k, v, [0, 5, 9], [0, 40, 49])
    assert rows.all() and np.allclose(out, want, atol=1e-12)
    # a tree that is a chain
    sees, depth, _ = od.tree_mask([-1, 0, 1, 2, 3, -1, 0, 1, 2], [0, 5, 9])
    assert np.allclose(od.attn_tree(q, cache, [0, 5, 9], [40, 9], table, 48, sees, depth)[0], want, atol=1e-12)
    # the last row of each alone is decode attention
    one, _ = opg.attn_paged(q[[4, 8]], cache, [40, 9], table, 48)
    assert np.allclose(od.attn_paged_window(q[[4, 8]], cache, [40, 9], table, 48, 0, 0)[0], one, atol=1e-12)
    assert np.allclose(od.attn_paged_window(q[[4, 8]], cache, [40, 9], table, 48, 48, 0)[0], one, atol=1e-12)


def test_oracle_of_a_branch_is_its_path():
    """Attention of a draft in a tree: that of the chain of its ancestors, written one behind the other."""
    g = np.random.default_rng(4)
    from test_gpu_paged import filled
    cache = filled(g, 4, 1, 16, 8, np.float32)
    table = np.array([[2, 0, 3]])
    q = g.standard_normal((6, 2, 128))
    sees, depth, _ = od.tree_mask([-1, 0, 0, 1, 2, 4], [0, 6])
    assert sees[5] == {0, 2, 4, 5} and list(depth) == [0, 1, 1, 2, 2, 3]
    out, _, _ = od.attn_tree(q, cache, [0, 6], [30], table, 48, sees, depth)
    moved, lens = od.kv_keep(cache, [0, 6], [30], table, np.array([[0, 2, 4, 5]]), [4])
    assert lens == [28]
    alone, _, _ = od.attn_tree(q[[5]], moved, [0, 1], [28], table, 48)
    assert np.allclose(out[5], alone[0], atol=1e-12)


def test_oracle_windows():
    assert [t for t in range(10) if od.in_window(t, 9, 3, 2)] == [0, 1, 7, 8, 9]
    g = np.random.default_rng(5)
    q, k, v = g.standard_normal((5, 1, 128)), g.standard_normal((8, 1, 128)), g.standard_normal((8, 1, 128))
    out, _, _ = od.attn_prompt_window(q, k, v, [0, 5], [0, 8], 2, 1)
    keep = [0, 6, 7]
    want, _, _ = opg.attn_prompt(q[4:], k[keep], v[keep], [0, 1], [0, 3])
    assert np.allclose(out[4], want[0], atol=1e-12)
    assert np.allclose(od.attn_prompt_window(q, k, v, [0, 5], [0, 8], 8, 0)[0], opg.attn_prompt(q, k, v, [0, 5], [0, 8])[0], atol=1e-12)


def test_oracle_of_tables():
    table = [[5, 6, -1], [7, -1, -1]]
    o = od.paged_grow([20, 16], [13, 1], [2, 1], table, 16, [1, 2, 3, 4, 0, 0, 0, 0], 4, 20)
    assert o["table"].tolist() == [[5, 6, 4], [7, 3, -1]] and o["held"] == [3, 2] and o["count"] == 2 and o["missing"] == (0, 0)
    assert list(o["pos"][:14]) == list(range(20, 33)) + [16] and list(o["slots"][[0, 12, 13, 14]]) == [6 * 16 + 4, 4 * 16, 3 * 16, -1]
    t, held, pool, count = od.paged_release(o["table"], 16, [17, 0], [99, 99], o["held"], [1, 2, 3, 4, 0, 0, 0, 0], 2)
    assert t.tolist() == [[5, 6, -1], [-1, -1, -1]] and held == [2, 0] and pool[:5] == [1, 2, 4, 7, 3] and count == 5
