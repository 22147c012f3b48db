"""How prompts with a window are divided (csrc/paged_plan.h compiled alone, no GPU)."""

import ctypes
import os
import random
import subprocess

import pytest

from paper_2405_16406_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))
I64 = ctypes.c_int64


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("prompt_window") / "prompt_window.so")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", f"-I{build.CSRC}", os.path.join(HERE, "prompt_window_host.cpp"),
                        "-o", out], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return ctypes.CDLL(out)


def plan_of(host, B, Tq, Tk, window, sinks, hq, hkv, cus=256):
    out = (ctypes.c_int32 * 3)()
    host.window_plan(I64(B), I64(Tq), I64(Tk), window, sinks, hq, hkv, cus, out)
    return tuple(out)


def run_of(host, low, last, window, sinks):
    out = (ctypes.c_int32 * 3)()
    host.tile_run(low, last, window, sinks, out)
    return tuple(out)


def test_a_window_plans_for_the_keys_that_it_leaves(host):
    """The parts of any tile's run fit the plan, however long the sequences are."""
    rng = random.Random(5)
    for _ in range(3000):
        B, hkv = int(2 ** rng.uniform(0, 5)), rng.choice([1, 2, 8])
        hq = hkv * rng.choice([1, 4, 17])
        Tq, Tk = int(2 ** rng.uniform(0, 12)), int(2 ** rng.uniform(0, 18))
        window, sinks = int(2 ** rng.uniform(0, 16)), rng.choice([0, 4, 64, 1000])
        half, splits, per = plan_of(host, B, Tq, Tk, window, sinks, hq, hkv, rng.choice([256, 304]))
        assert splits >= 1 and not (half and splits > 1)
        low = rng.randrange(0, Tk)
        tokens = run_of(host, low, min(low + rng.randrange(256), Tk - 1), window, sinks)[2]
        assert tokens <= sinks + 63 + window + 63 + 256
        tiles = -(-tokens // 64)
        assert splits == 1 or host.window_part(tiles, splits, per) * splits >= tiles
    # a window of everything plans as none does; one of little needs no parts
    assert plan_of(host, 1, 4, 3000, 1 << 29, 0, 2, 2)[1] > 1 and plan_of(host, 1, 4, 3000, 50, 0, 2, 2)[1] == 1
    assert plan_of(host, 1, 4, 1 << 30, (1 << 30) - 1, (1 << 30) - 1, 2, 2)[1] > 1


@pytest.mark.parametrize("cus", [256, 304])
def test_every_division_is_tested(host, cus):
    """The sizes of tests/test_gpu_prompt_window.py are what they are called."""
    t = pytest.importorskip("test_gpu_prompt_window")
    for name, cases in (("parts", t.PARTS), ("whole", t.WHOLE), ("halves", t.HALVES)):
        for hq, h, nq, nk, window, sinks in cases:
            half, splits, _ = plan_of(host, len(nq), sum(nq) + 3, sum(nk) + 3, window, sinks, hq, h, cus)
            assert (half, splits > 1) == {"parts": (0, True), "whole": (0, False), "halves": (1, False)}[name], (hq, nq, nk, window)
    for name, (hq, h, n, m, window, sinks, *_) in t.HIDDEN.items():
        half, splits, _ = plan_of(host, 1, n, m, window, sinks, hq, h, 256)
        assert (half, splits > 1) == {"p": (0, True), "w": (0, False), "h": (1, False)}[name[0]], name


def test_parts_lie_where_rows_differ(host):
    """Some part lies wholly in the first tokens, some before one row's window, and some past another row."""
    t = pytest.importorskip("test_gpu_prompt_window")
    first = before = past = joined = 0
    for hq, h, nq, nk, window, sinks in t.PARTS:
        _, splits, per = plan_of(host, len(nq), sum(nq) + 3, sum(nk) + 3, window, sinks, hq, h)
        group = hq // h
        for n, m in zip(nq, nk):
            for r0 in range(0, n * group, 256):
                low, last = m - n + r0 // group, m - n + min(r0 + 255, n * group - 1) // group
                head, start, tokens = run_of(host, max(low, -1), last, window, sinks)
                tiles = -(-tokens // 64)
                part = host.window_part(tiles, splits, per)
                joined = max(joined, -(-tiles // part) if tiles else 0)
                for t0 in range(0, tiles, part):
                    places = range(64 * t0, min(64 * (t0 + part), tokens))
                    keys = [x if x < head else x - head + start for x in (places[0], places[-1])]
                    first += keys[1] < sinks and head > 0
                    before += sinks <= keys[0] and keys[1] <= last - window
                    past += keys[0] > low
    assert first and before and past and joined > 4
