"""Pins of oracle/paged.py: closed forms and invariants (no GPU)."""

import math

import numpy as np
import pytest

from oracle import paged as opg
from oracle.quant import quant_asym
from paper_2405_16406_amd import sq


def rng(seed):
    return np.random.Generator(np.random.PCG64(seed))


def empty(pages, heads, page, bits, dt=np.float32):
    return dict(k_q=np.zeros((pages, heads, page, 16 * bits), np.uint8), v_q=np.zeros((pages, heads, page, 16 * bits), np.uint8),
                params=np.zeros((pages, heads, page, 4), dt))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rotary", [128, 64, 32])
def test_rope_scores_depend_on_the_distance(rotary, interleaved):
    f = opg.rope_frequencies(rotary, 10000.0)
    x, y = rng(1).standard_normal((2, 1, 1, 128))
    dots = [np.vdot(opg.rope(x, [p], f, interleaved), opg.rope(y, [p + 5], f, interleaved)) for p in (0, 3, 1000, 100000)]
    assert np.allclose(dots, dots[0], rtol=0, atol=1e-8)
    assert np.allclose(np.linalg.norm(opg.rope(x, [77], f, interleaved)), np.linalg.norm(x))
    assert np.array_equal(opg.rope(x, [77], f, interleaved)[..., rotary:], x[..., rotary:])


def test_rope_layouts_are_a_permutation_of_each_other():
    f = opg.rope_frequencies(64, 500.0)
    x = rng(2).standard_normal((3, 2, 128))
    perm = np.concatenate([np.stack([np.arange(32), np.arange(32) + 32], 1).ravel(), np.arange(64, 128)])
    pos = [4, 0, 9]
    assert np.allclose(opg.rope(x, pos, f)[..., perm], opg.rope(x[..., perm], pos, f, True))


def test_rope_quarter_turn():
    x = np.zeros((1, 1, 128))
    x[0, 0, 0] = 3.0
    y = opg.rope(x, [1], np.array([math.pi / 2] + [0.0] * 63), magnitude=2.0)
    assert abs(y[0, 0, 0]) < 1e-15 and y[0, 0, 64] == 6.0


@pytest.mark.parametrize("rotary,scaling", [(128, "none"), (96, "linear"), (64, "by parts"), (16, "by parts")])
def test_library_frequencies(rotary, scaling):
    kw = dict(scaling=scaling, factor=8.0, low=1.0, high=4.0, original_len=8192.0)
    got = sq.rope_frequencies(rotary, 500000.0, **kw).numpy()
    want = opg.rope_frequencies(rotary, 500000.0, **kw)
    assert np.all(np.abs(got - want) <= 1e-14 * want)
    if scaling == "by parts":  # the ends of the ramp
        plain = opg.rope_frequencies(rotary, 500000.0)
        turns = 8192.0 * plain / (2 * math.pi)
        assert np.allclose(want[turns >= 4], plain[turns >= 4]) and np.allclose(want[turns <= 1], plain[turns <= 1] / 8)


@pytest.mark.parametrize("bits,dt", [(4, np.float32), (8, np.float16)])
def test_write_then_read_is_within_half_a_level(bits, dt):
    g = rng(3)
    T, Hq, H = 21, 4, 2
    q, k, v = (g.standard_normal((T, h, 128)).astype(np.float16) for h in (Hq, H, H))
    cu, lens = [0, 5, 5, 21], [20, 3, 16]
    table = np.array([[3, 1], [0, 0], [2, 9]])  # 9: not in the pool
    cache = empty(4, H, 16, bits, dt)
    f = opg.rope_frequencies(128, 10000.0)
    o = opg.rope_kv_write(q, k, v, cache, cu, lens, table, f)
    kk, vv, rows = opg.kv_read(o, cu, lens, table, T)
    assert rows.all() and np.array_equal(o["pos"][:5], [15, 16, 17, 18, 19])
    for t in range(T):
        half = o["params"][o["where"][t], :, o["pos"][t] % 16].astype(np.float64)
        slack = 1.001 if dt == np.float32 else 1.6  # rounded ends may lie inside the range
        assert np.all(np.abs(vv[t] - v[t]) <= slack * half[:, 2:3] / 2 + 1e-6)
        assert np.all(np.abs(kk[t] - o["k_rot"][t]) <= slack * half[:, 0:1] / 2 + 1e-6)
    plain, _, _ = opg.kv_read(o, cu, lens, table, T, plain_basis=True)
    assert np.allclose(np.linalg.norm(plain, axis=-1), np.linalg.norm(kk, axis=-1))
    # only the rows' slots changed
    assert not o["k_q"][0].any() and not o["params"][2, :, :0].any() and o["params"][1, :, 4:].max() == 0


def test_attention_over_pages_equals_attention_over_what_is_read():
    g = rng(4)
    H, G, n = 2, 3, 37
    lens, table = [n], np.array([[2, 0, 1]])
    cache = empty(3, H, 16, 4)
    k, v = (g.standard_normal((n, H, 128)).astype(np.float16) for _ in range(2))
    o = opg.rope_kv_write(np.zeros((n, H * G, 128), np.float16), k, v, cache, [0, n], lens, table, None)
    kk, vv, _ = opg.kv_read(o, [0, n], lens, table, n)
    q = g.standard_normal((1, H * G, 128)).astype(np.float16)
    a, _ = opg.attn_paged(q, o, lens, table, 64)
    b, _, _ = opg.attn_prompt(q, kk, vv, [0, 1], [0, n])
    assert np.allclose(a, b, atol=1e-12)
    assert not opg.attn_paged(q, o, [0], table, 64)[0].any()


def test_causal_rows():
    g = rng(5)
    q, k, v = (g.standard_normal((6, 1, 128)) for _ in range(3))
    out, _, rows = opg.attn_prompt(q, k, v, [0, 4, 5], [0, 2, 6])
    assert rows.tolist() == [True] * 5 + [False]
    assert not out[:2].any() and np.allclose(out[2, 0], v[0, 0])  # 4 queries, 2 keys: the first two see none
    s = np.exp(k[2:6, 0] @ q[4, 0] / math.sqrt(128))
    assert np.allclose(out[4, 0], (s / s.sum()) @ v[2:6, 0])


@pytest.mark.parametrize("bits", [4, 8])
def test_smallest_value_scale(bits):
    """fp16 values differ by 2^-24 or not at all: clipped to 2^-28 of the range, alpha is 2^-60 or more."""
    x = np.zeros((3, 128), dtype=np.float16)
    x[0, 5] = 2.0 ** -24
    x[1, :] = np.float16(0.5)
    x[1, 7] = np.nextafter(np.float16(0.5), np.float16(0))
    _, alpha, _ = quant_asym(x.astype(np.float32), bits=bits, group=128, clip=2.0 ** -28)
    assert alpha.min() >= 2.0 ** -60 and alpha[2] == 1
