"""Index arithmetic and splits of the paged cache (csrc/paged.h, paged_plan.h compiled alone, no GPU)."""

import ctypes
import os
import random
import subprocess

import numpy as np
import pytest

from oracle import paged as opg
from paper_2405_16406_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("paged") / "paged.so")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", f"-I{build.CSRC}", os.path.join(HERE, "paged_host.cpp"),
                        "-o", out], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    lib = ctypes.CDLL(out)
    lib.row_slot.restype = ctypes.c_int64
    return lib


def slot(host, ln, end, t, row, pages, shift, heads, h):
    row = np.asarray(row, dtype=np.int32)
    return host.row_slot(ln, end, ctypes.c_int64(t), row.ctypes.data_as(ctypes.c_void_p), len(row), pages, shift, heads, h)


def test_slots_and_bad_pages(host):
    # 3 new rows 4 .. 6 of a sequence of 34 tokens, pages of 16: positions 31, 32, 33
    row = [7, 2, 5]
    assert slot(host, 34, 7, 4, row, 8, 4, 3, 0) == (2 * 3 + 0) * 16 + 15
    assert slot(host, 34, 7, 5, row, 8, 4, 3, 2) == (5 * 3 + 2) * 16 + 0
    # entries outside the pool, positions past the table, before the sequence
    for bad in (8, -1, 2 ** 31 - 1, -2 ** 31):
        assert slot(host, 34, 7, 5, [7, 2, bad], 8, 4, 3, 2) == -1
    assert slot(host, 49, 7, 6, row, 8, 4, 3, 0) == -1
    assert slot(host, 2, 7, 4, row, 8, 4, 3, 0) == -1
    # malformed lengths and row bounds stay in the table or have no place
    for ln, end, t in ((2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1), (-2 ** 31, 2 ** 31 - 1, 0), (2 ** 31 - 1, 0, 5)):
        assert slot(host, ln, end, t, row, 8, 4, 3, 0) == -1


def test_slots_past_32_bits(host):
    pages, shift, heads = 2 ** 20, 7, 64
    s = slot(host, 128, 1, 0, [pages - 1], pages, shift, heads, 63)
    assert s == pages * heads * 128 - 1 > 2 ** 32


def test_slots_against_the_oracle(host):
    rng = random.Random(1)
    for _ in range(300):
        shift, pages, heads, cols = rng.randrange(4, 9), rng.randrange(1, 9), rng.randrange(1, 5), rng.randrange(1, 7)
        row = [rng.randrange(-2, pages + 2) for _ in range(cols)]
        ln, new = rng.randrange(0, (cols + 1) << shift), rng.randrange(1, 70)
        pos, where = opg.places(new, [0, new], [ln], np.array([row]), 1 << shift, pages)
        for t in range(new):
            got = slot(host, ln, new, t, row, pages, shift, heads, heads - 1)
            want = -1 if where[t] < 0 else (where[t] * heads + heads - 1) * (1 << shift) + pos[t] % (1 << shift)
            assert got == want


def test_paged_split_covers_every_token(host):
    rng, out = random.Random(2), (ctypes.c_int32 * 2)()
    sizes = [(1, 1, 1, 1, 256), (1, 2 ** 30 - 1, 32, 8, 256), (2 ** 17, 2 ** 30 - 1, 64, 8, 256), (1, 255, 64, 8, 1)]
    for _ in range(3000):
        hkv = rng.choice([1, 2, 8, 32])
        sizes.append((int(2 ** rng.uniform(0, 12)), int(2 ** rng.uniform(0, 30)) - 1 or 1, hkv * rng.choice([1, 4, 8, 17, 33]), hkv,
                      rng.choice([256, 304, 64, 1])))
    for B, n, hq, hkv, cus in sizes:
        host.paged_split(ctypes.c_int64(B), ctypes.c_int64(n), hq, hkv, cus, out)
        chunks, tokens = out
        assert chunks >= 1 and tokens >= 256 and tokens % 256 == 0
        assert (chunks - 1) * tokens < n <= chunks * tokens
        groups = B * hkv * -(-(hq // hkv) // 16)
        assert groups * chunks <= groups + 8 * cus + 4 * cus  # workgroups stay bounded


def plan_of(host, B, Tq, Tk, hq, hkv, cus=256):
    out = (ctypes.c_int32 * 3)()
    host.prompt_plan(ctypes.c_int64(B), ctypes.c_int64(Tq), ctypes.c_int64(Tk), hq, hkv, cus, out)
    return tuple(out)


def test_prompt_plans_are_bounded(host):
    rng = random.Random(3)
    for _ in range(3000):
        hkv = rng.choice([1, 8, 32])
        hq, B = hkv * rng.choice([1, 4, 8, 17]), int(2 ** rng.uniform(0, 10))
        Tq, Tk, cus = int(2 ** rng.uniform(0, 20)), int(2 ** rng.uniform(0, 20)), rng.choice([256, 64, 1])
        half, splits, per = plan_of(host, B, Tq, Tk, hq, hkv, cus)
        assert splits >= 1 and half in (0, 1) and not (half and splits > 1)
        if splits > 1:
            assert per >= 4 and Tq * hq * splits <= 1 << 18
            for tiles in (0, 1, per, per + 1, -(-Tk // 64), rng.randrange(1 << 20)):  # any sequence fits its parts
                part = host.prompt_part(tiles, splits, per)
                assert part >= per and part * splits >= tiles
    assert plan_of(host, 0, 4, 4, 8, 8) == plan_of(host, 4, 0, 4, 8, 8) == plan_of(host, 4, 4, 0, 8, 8) == (0, 1, 0)


def test_prompt_plans_of_known_sizes(host):
    """The measured choices: whole tiles, halves, and parts."""
    assert plan_of(host, 1, 8192, 8192, 32, 32)[:2] == (0, 1)
    assert plan_of(host, 1, 2048, 2048, 32, 32)[:2] == (1, 1)
    assert plan_of(host, 1, 1024, 1024, 64, 8)[:2] == (1, 1)
    half, splits, per = plan_of(host, 2, 41, 22560, 32, 8)
    assert half == 0 and splits > 16 and per == 12


def test_every_prompt_form_is_tested(host):
    """The sizes of tests/test_gpu_paged.py reach whole tiles, halves and parts."""
    t = pytest.importorskip("test_gpu_paged")
    plans = [plan_of(host, len(nq), sum(nq) + 3, sum(nk) + 2, hq, h) for hq, h, nq, nk in t.PROMPT]
    assert {(half, splits > 1) for half, splits, _ in plans} == {(0, False), (1, False), (0, True)}


def test_every_looping_form_is_tested(host):
    """The sizes of tests/test_gpu_paged_sizes.py reach writes of several tokens a workgroup and several
    tasks a wave, waves with several blocks, the join beyond one round of its loads, and each division of a
    prompt with more than 64 sequences."""
    t = pytest.importorskip("test_gpu_paged_sizes")
    out = (ctypes.c_int32 * 2)()
    for hq, h, *_, rows, tokens in t.WRITE:
        host.rope_plan(ctypes.c_int64(rows), hq, h, out)
        assert out[0] == tokens
    assert {w[-1] for w in t.WRITE} == {1, 2, 4, 8}
    host.rope_plan(ctypes.c_int64(1100), 64, 8, out)
    assert out[1] == 4 < 4 + 1 + 1  # waves, tasks
    blocks, joined = set(), set()
    for hq, h, _, bits, _, lens, most, _ in t.PAGED:
        host.paged_split(ctypes.c_int64(len(lens)), ctypes.c_int64(most), hq, h, 256, out)
        chunks, tokens = out
        blocks.add((bits, min(tokens, max(lens)) // 256))
        joined.add((chunks > 8, -(-max(lens) // tokens)))
    assert {b for b, n in blocks if n >= 3} == {4, 8}
    assert any(eight and 8 < n <= 64 for eight, n in joined) and any(eight and n > 64 for eight, n in joined)
    plans = [plan_of(host, len(nq), sum(nq) + 1, sum(nk), hq, h) for hq, h, nq, nk in t.PROMPT]
    assert [(half, splits > 1) for half, splits, _ in plans] == [(0, False), (1, False), (0, True)]
    assert all(len(nq) > 64 for _, _, nq, _ in t.PROMPT)
