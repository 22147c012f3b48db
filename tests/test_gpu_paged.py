"""The paged cache on the GPU against oracle/paged.py: write, read back, decode and prompt attention.

Tolerances, from the arithmetic (fp16 rounds by 2^-11 of the value or 2^-25, fp32 by 2^-24):
  rotated queries (fp16)  2^-11 |y| + 2^-25, and 2e-6 of the row's norm for 32-bit angles, seven
                          butterflies and two products
  keys                    rotated in 64 bits and rounded once to fp32: alpha and beta within two fp32
                          roundings of the group's range (one more fp16 step where stored so);
                          codes as the oracle's except within 1e-4 of a border
  values                  parameters and codes bit for bit
  read back               2^-11 |v| + 2^-25 and two fp32 roundings of |alpha c| + |beta|; plain basis:
                          10 roundings of the row's norm
  attention               weights rounded to fp16: 2^-11 sum p |v|, the output's own rounding, and the
                          weights' relative error from fp32 scores: the given `scores` bound
"""

import numpy as np
import pytest
import torch

from oracle import paged as opg
from oracle import quant as oq
from paper_2405_16406_amd import sq

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def rng(seed):
    return np.random.Generator(np.random.PCG64(seed))


def up(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def ints(a):
    return torch.tensor(np.asarray(a, dtype=np.int64).tolist(), dtype=torch.int32, device=DEV)


def f64(t):
    return t.cpu().numpy().astype(np.float64)


def spread_table(g, lens, page, spare=1):
    """A block table of distinct pages in random order, and the number of pages."""
    need = [max(1, -(-n // page)) for n in lens]
    order = g.permutation(sum(need) + spare)
    table = np.zeros((len(lens), max(need)), dtype=np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, sum(need) + spare


def filled(g, pages, heads, page, bits, dt, std=1.5):
    """A cache of normal vectors."""
    out = {}
    ab = []
    for n in ("k_q", "v_q"):
        x = (g.standard_normal((pages, heads, page, 128)) * std).astype(np.float32)
        c, a, b = oq.quant_asym(x, bits=bits, group=128, param_fp16=dt == np.float16)
        out[n] = oq.store_codes(c, bits)
        ab += [a, b]
    out["params"] = np.concatenate(ab, axis=-1).astype(dt)
    return out


def device_cache(c):
    return up(c["k_q"]), up(c["v_q"]), up(c["params"])


def heads_of(g, rows, h, std=1.0):
    return (g.standard_normal((rows, h, 128)) * std).astype(np.float16)


def check_write(o, q_rot, cache, q, bits, live):
    """cache: the device's after the call."""
    norm = np.linalg.norm(o["q_rot"], axis=-1, keepdims=True)
    got = f64(q_rot)
    bad = np.abs(got - o["q_rot"]) > 2.0 ** -11 * np.abs(o["q_rot"]) + 2.0 ** -25 + 2e-6 * norm
    assert not bad[live].any()
    k_q, v_q, params = (t.cpu().numpy() for t in cache)
    assert np.array_equal(v_q, o["v_q"])
    assert np.array_equal(params[..., 2:], o["params"][..., 2:])
    ga, oa = params[..., :2].astype(np.float64), o["params"][..., :2].astype(np.float64)
    top = 2.0 ** bits - 1
    if params.dtype == np.float32:
        scale = np.abs(oa[..., :1]) * top + np.abs(oa[..., 1:])
        assert np.all(np.abs(ga - oa) <= 2.0 ** -23 * scale)
    else:
        assert np.all(np.abs(ga - oa) <= 2.0 ** -10 * np.abs(oa) + 2.0 ** -24)
        assert np.mean(ga != oa) <= 1e-3
    a = oq.unpack_nibbles(k_q, signed=False) if bits == 4 else k_q.astype(np.int64)
    b = oq.unpack_nibbles(o["k_q"], signed=False) if bits == 4 else o["k_q"].astype(np.int64)
    for t in np.nonzero(o["where"] >= 0)[0]:
        at = (o["where"][t], slice(None), o["pos"][t] % k_q.shape[2])
        d = a[at] - b[at]
        if d.any():
            al, be = (o["params"][at][:, i, None].astype(np.float64) for i in (0, 1))
            x = (o["k32"][t].astype(np.float64) - be) / al
            same = np.array_equal(ga[at], oa[at])
            assert np.all(np.abs(d) <= 1) and (not same or np.all(np.abs(x - np.floor(x) - 0.5)[d != 0] <= 1e-4))
            a[at] = b[at]
    assert np.array_equal(a, b)  # nothing else was touched


WRITE = [  # Hq, Hkv, page, bits, params, rotary, interleaved, clip, rows of each sequence, tokens before
    (8, 2, 16, 4, np.float32, 128, False, 1.0, [5, 1, 40], [11, 0, 100000]),
    (4, 4, 64, 8, np.float32, 128, True, 1.0, [1], [70]),
    (64, 8, 32, 4, np.float16, 64, False, 0.95, [3, 0, 2], [0, 4, 31]),
    (5, 1, 16, 8, np.float16, 96, False, 0.9, [17, 16], [15, 16]),
    (32, 8, 128, 4, np.float32, 32, True, 1.0, [2, 7], [126, 1000000]),
    (32, 32, 16, 4, np.float16, 16, False, 1.0, [9], [3]),
    (3, 3, 16, 8, np.float32, 0, False, 1.0, [33], [0]),
    (300, 100, 16, 4, np.float32, 128, False, 1.0, [2], [14]),
]


@pytest.mark.parametrize("case", WRITE, ids=lambda c: f"{c[0]}x{c[1]}-p{c[2]}-b{c[3]}-{np.dtype(c[4]).name}-r{c[5]}{'i' if c[6] else 'h'}")
@pytest.mark.parametrize("form", ["packed", "fused", "k_out"])
def test_write(case, form):
    Hq, H, page, bits, dt, rotary, inter, clip, new, past = case
    g = rng(Hq + page)
    lens = [n + p for n, p in zip(new, past)]
    T = sum(new) + 2  # two rows behind the last sequence
    cu = np.concatenate([[0], np.cumsum(new)])
    used = [min(n, 400) if n > 400 else n for n in lens]
    # long histories: a table that maps only the last positions (others have no page here)
    cols = max(-(-n // page) for n in lens)
    table = np.full((len(lens), cols), -1, dtype=np.int32)
    pages = 0
    for b, n in enumerate(lens):
        for c in range(max(0, (n - used[b]) // page), -(-n // page)):
            table[b, c] = pages
            pages += 1
    pages = max(pages, 1)
    q, k, v = (heads_of(g, T, h) for h in (Hq, H, H))
    freq = opg.rope_frequencies(rotary, 10000.0) if rotary else None
    cache = filled(g, pages, H, page, bits, dt)
    o = opg.rope_kv_write(q, k, v, cache, cu, lens, table, freq, inter, 1.0, clip, clip)
    dc = device_cache(cache)
    if form == "fused":
        fused = torch.empty((T, Hq + 2 * H, 128), dtype=torch.float16, device=DEV)
        fused[:, :Hq], fused[:, Hq:Hq + H], fused[:, Hq + H:] = up(q), up(k), up(v)
        dq, dk, dv = fused[:, :Hq], fused[:, Hq:Hq + H], fused[:, Hq + H:]
    else:
        dq, dk, dv = up(q), up(k), up(v)
    out = torch.full((T, Hq, 128), 7.0, dtype=torch.float16, device=DEV)
    k_out = torch.full((T, H, 128), 7.0, dtype=torch.float16, device=DEV) if form == "k_out" else None
    sq.rope_kv_write(dq, dk, dv, dc, ints(table), ints(lens), None if freq is None else up(freq), cu=ints(cu), interleaved=inter,
                     k_clip=clip, v_clip=clip, out=out, k_out=k_out)
    torch.cuda.synchronize()
    check_write(o, out, dc, q, bits, o["rows"])
    assert torch.all(out[sum(new):] == 7.0)
    if k_out is not None:
        kr = o["k_rot"]
        assert np.all(np.abs(f64(k_out) - kr)[o["rows"]] <= (2.0 ** -11 * 1.001 * np.abs(kr) + 2.0 ** -25)[o["rows"]])
        assert torch.all(k_out[sum(new):] == 7.0)


def test_write_one_token_per_sequence_and_bad_pages():
    g = rng(5)
    B, Hq, H, page = 70, 4, 2, 16
    lens = [int(x) for x in g.integers(1, 60, B)]
    lens[3] = 0      # no position
    lens[4] = 200    # past the table
    table, pages = spread_table(g, [min(n, 64) for n in lens], page)
    table[7, (lens[7] - 1) // page] = pages          # not in the pool
    table[8, (lens[8] - 1) // page] = -5
    table[9, (lens[9] - 1) // page] = 2 ** 31 - 1
    q, k, v = (heads_of(g, B, h) for h in (Hq, H, H))
    freq = opg.rope_frequencies(128, 500000.0, "by parts", 8.0)
    cache = filled(g, pages, H, page, 4, np.float32)
    o = opg.rope_kv_write(q, k, v, cache, np.arange(B + 1), lens, table, freq, magnitude=1.25)
    dc = device_cache(cache)
    out = torch.full((B, Hq, 128), 7.0, dtype=torch.float16, device=DEV)
    sq.rope_kv_write(up(q), up(k), up(v), dc, ints(table), ints(lens), up(freq), magnitude=1.25, out=out)
    torch.cuda.synchronize()
    assert list(np.nonzero(~o["rows"])[0]) == [3] and (o["where"] < 0).sum() == 5
    check_write(o, out, dc, q, 4, o["rows"])
    assert torch.all(out[3] == 7.0)
    # the same through cu, many sequences
    dc2 = device_cache(cache)
    out2 = sq.rope_kv_write(up(q), up(k), up(v), dc2, ints(table), ints(lens), up(freq), cu=ints(np.arange(B + 1)), magnitude=1.25)
    live = torch.tensor(o["rows"], device=DEV)
    assert torch.equal(out[live], out2[live]) and all(torch.equal(a, b) for a, b in zip(dc, dc2))


@pytest.mark.parametrize("plain", [False, True])
@pytest.mark.parametrize("H,page,bits,dt", [(8, 16, 4, np.float32), (32, 64, 8, np.float16), (1, 16, 8, np.float32), (3, 32, 4, np.float16),
                                            (100, 16, 4, np.float32)])
def test_read(H, page, bits, dt, plain):
    g = rng(H)
    lens, new = [50, 3, 17, 130], [50, 0, 9, 70]
    cu = np.concatenate([[2], 2 + np.cumsum(new)])  # two rows before the first sequence, one behind
    T = int(cu[-1]) + 1
    table, pages = spread_table(g, lens, page)
    table[0, 1] = -1
    cache = filled(g, pages, H, page, bits, dt)
    k, v, rows = opg.kv_read(cache, cu, lens, table, T, plain)
    wide = torch.full((T, H + 3, 128), 7.0, dtype=torch.float16, device=DEV)
    out = torch.full((T, H, 128), 7.0, dtype=torch.float16, device=DEV), wide[:, :H]
    sq.kv_read(device_cache(cache), ints(table), ints(lens), ints(cu), T, plain, out=out)
    torch.cuda.synchronize()
    norm = np.linalg.norm(k, axis=-1, keepdims=True)
    size = lambda x: 2.0 ** -11 * np.abs(x) + 2.0 ** -25 + 2.0 ** -22 * np.abs(x).max(-1, keepdims=True)  # noqa: E731
    assert np.all(np.abs(f64(out[0]) - k)[rows] <= (size(k) + (10 * 2.0 ** -24 * norm if plain else 0))[rows])
    assert np.all(np.abs(f64(out[1]) - v)[rows] <= size(v)[rows])
    for t in out:
        assert torch.all(t[torch.tensor(~rows, device=DEV)] == 7.0)
    assert torch.all(wide[:, H:] == 7.0)


def attention_close(got, want, weight, scores):
    got, want = f64(got), np.asarray(want)
    assert np.all(np.isfinite(got))
    tol = (2.0 ** -11 + scores) * weight + 2.0 ** -11 * np.abs(want) + 2.0 ** -25
    worst = (np.abs(got - want) / tol).max()
    assert worst <= 1.0, f"{worst:.3g} times the tolerance"


PAGED = [  # Hq, Hkv, page, bits, params, lens, max_len
    (8, 2, 16, 4, np.float32, [1, 2, 15, 16, 17, 63, 64, 65, 0, 200], 200),
    (4, 4, 16, 8, np.float32, [257, 31, 1], 300),
    (32, 1, 32, 4, np.float16, [100, 513], 513),       # 32 query heads on one: two tiles
    (17, 1, 64, 8, np.float16, [300], 300),
    (16, 2, 128, 4, np.float32, [1030, 7], 5000),
    (6, 2, 16, 4, np.float16, [0, 0, 3], 1 << 20),     # far fewer tokens than max_len
    (64, 8, 32, 4, np.float32, [90] * 40, 90),
]


@pytest.mark.parametrize("case", PAGED, ids=lambda c: f"{c[0]}x{c[1]}-p{c[2]}-b{c[3]}-{np.dtype(c[4]).name}-{max(c[5])}of{c[6]}")
def test_paged_attention(case):
    Hq, H, page, bits, dt, lens, most = case
    g = rng(Hq + bits)
    B = len(lens)
    table, pages = spread_table(g, lens, page)
    cache = filled(g, pages, H, page, bits, dt)
    q = heads_of(g, B, Hq)
    out = torch.full((B, Hq, 128), 7.0, dtype=torch.float16, device=DEV)
    n = sq.attn_paged_workspace_bytes(B, most, Hq, H)
    ws = torch.full((n + 16,), 255, dtype=torch.uint8, device=DEV)  # NaN wherever it is read unwritten
    got = sq.attn_paged(up(q), device_cache(cache), ints(table), ints(lens), most, out=out, workspace=ws)
    torch.cuda.synchronize()
    want, weight = opg.attn_paged(q, cache, lens, table, most)
    attention_close(got, want, weight, 2e-5)
    assert torch.all(got[[b for b in range(B) if lens[b] == 0]] == 0)
    again = sq.attn_paged(up(q), device_cache(cache), ints(table), ints(lens), most)
    assert torch.equal(got, again)


def test_paged_attention_strides_scale_lengths_and_missing_pages():
    g = rng(11)
    B, Hq, H, page = 5, 8, 2, 16
    lens = [80, 80, 75, 40, 100]
    table, pages = spread_table(g, lens, page)
    table[0, 2] = -1           # a hole
    table[1, :] = pages + 3    # nothing at all
    table[2, 4] = 2 ** 31 - 1
    cache = filled(g, pages, H, page, 4, np.float32)
    q = heads_of(g, B, Hq)
    wide = torch.zeros((B, Hq + 4, 128), dtype=torch.float16, device=DEV)
    wide[:, 2:Hq + 2] = up(q)
    out = torch.full((B, Hq + 1, 128), 7.0, dtype=torch.float16, device=DEV)
    tw = torch.full((B, table.shape[1] + 5), 10 ** 6, dtype=torch.int32, device=DEV)
    tw[:, :table.shape[1]] = ints(table)
    got = sq.attn_paged(wide[:, 2:Hq + 2], device_cache(cache), tw[:, :table.shape[1]], ints(lens), 90, scale=0.3, out=out[:, :Hq])
    torch.cuda.synchronize()
    want, weight = opg.attn_paged(q, cache, lens, table, 90, 0.3)  # the last sequence counts as 90 tokens
    attention_close(got, want, weight, 1e-4)
    assert torch.all(got[1] == 0) and torch.all(out[:, Hq:] == 7.0)


@pytest.mark.parametrize("scale_v", [1e-5, 4e3])
def test_paged_attention_of_small_and_large_values(scale_v):
    """Values of any size keep their precision, and parameters behind the last token have no part."""
    g = rng(12)
    lens, page = [150], 16
    table, pages = spread_table(g, lens, page)
    cache = filled(g, pages, 2, page, 4, np.float32)
    cache["params"][..., 2:] *= scale_v
    behind = cache["params"][table[0, 9], :, 6:]
    behind[...] = np.nan
    q = heads_of(g, 1, 8)
    got = sq.attn_paged(up(q), device_cache(cache), ints(table), ints(lens), 150)
    want, weight = opg.attn_paged(q, cache, lens, table, 150)
    attention_close(got, want, weight, 2e-5)


@pytest.mark.parametrize("bits", [4, 8])
def test_paged_attention_of_values_that_cancel(bits):
    """Sums of the codes are as exact as fp32 beside a much larger weight: values whose mean is 0 give 0.

    Of four tokens one has weight 2^12 and value 1 - 1, two a far smaller weight w, the same for all, and
    opposite values; the last one's code and value are 0.  w has 11 bits and is at least 2^k = 8, so a
    multiple of 2^(k - 10).  A wave has one block of 64 tokens of a chunk: its sums of w and codes, whose
    mean is 2^(bits - 1), are at most 32 2^(bits - 1) 2^(k + 1) + 16 2^12, with 8 bits 2^24 units.  fp32
    holds them all, so no sum is rounded.
    """
    g = rng(14)
    n, page, heads = 1024, 16, 16
    middle = 2 ** (bits - 1)
    table, pages = spread_table(g, [n], page, spare=0)
    at = np.arange(n) % 4
    paired = (at == 1) | (at == 2)
    codes = np.zeros((n, 128), dtype=np.int64)
    codes[at == 0] = 1
    half = g.integers(1, 2 * middle, size=(paired.sum() // 2, 128))
    codes[paired] = np.stack([half, 2 * middle - half], axis=1).reshape(-1, 128)
    params = np.zeros((n, 4), dtype=np.float32)
    params[at > 0, 1] = -8
    params[:, 2] = 1
    params[at == 0, 3], params[paired, 3] = -1, -middle
    cache = {"k_q": np.zeros((pages, 1, page, 16 * bits), dtype=np.uint8), "v_q": np.empty((pages, 1, page, 16 * bits), dtype=np.uint8),
             "params": np.empty((pages, 1, page, 4), dtype=np.float32)}
    for c, where in enumerate(table[0]):
        cache["v_q"][where, 0] = oq.store_codes(codes[c * page:(c + 1) * page].astype(np.uint8), bits)
        cache["params"][where, 0] = params[c * page:(c + 1) * page]
    q = np.zeros((1, heads, 128), dtype=np.float16)
    q[0, :, 0] = np.linspace(7.1, 8.9, heads) * np.log(2) / 8  # pairs of weight 2^(12 - 7.1) .. 2^(12 - 8.9)
    want, _ = opg.attn_paged(q, cache, [n], table, n, 1.0)
    assert np.abs(want).max() < 1e-12
    got = sq.attn_paged(up(q), device_cache(cache), ints(table), ints([n]), n, scale=1.0)
    assert torch.all(got == 0), got.abs().max()


@pytest.mark.parametrize("scale", [-0.1, 0.0])
def test_paged_attention_of_scales_not_positive(scale):
    g = rng(15)
    lens, page = [150, 1, 0], 16
    table, pages = spread_table(g, lens, page)
    cache = filled(g, pages, 2, page, 4, np.float32)
    q = heads_of(g, 3, 8)
    got = sq.attn_paged(up(q), device_cache(cache), ints(table), ints(lens), 150, scale=scale)
    want, weight = opg.attn_paged(q, cache, lens, table, 150, scale)
    attention_close(got, want, weight, 2e-5)


@pytest.mark.parametrize("bits", [4, 8])
def test_paged_attention_of_value_scales_far_apart(bits):
    """Tokens whose values are 2^-18 of the others' keep their part in the softmax's sum.

    Their fp16 factor, weight times v_alpha, is 2^12 at the largest product: with scores within 4 of
    each other in base 2, and v_alpha within 2^2 of each other but for the 2^-18, it is 2^-12 or
    more, a normal number.
    """
    g = rng(16)
    lens, page = [600], 16
    table, pages = spread_table(g, lens, page)
    cache = filled(g, pages, 2, page, bits, np.float32)
    cache["params"][:, :, ::3, 2:] *= 2.0 ** -18
    q = heads_of(g, 1, 8, 0.2)
    got = sq.attn_paged(up(q), device_cache(cache), ints(table), ints(lens), 600)
    want, weight = opg.attn_paged(q, cache, lens, table, 600)
    attention_close(got, want, weight, 2e-5)


PROMPT = [  # Hq, Hkv, queries, keys
    (2, 2, [1], [1]),
    (4, 1, [5, 0, 1, 64, 65], [5, 0, 1, 64, 65]),
    (8, 2, [33, 70], [40, 300]),
    (3, 3, [257], [257]),
    (16, 2, [100, 3], [100, 2]),            # more queries than keys: rows that see nothing
    (17, 1, [20], [700]),
    (8, 8, [129, 31], [129, 63]),
    (4, 4, [3, 2], [0, 9]),                 # no keys at all
    (8, 1, [2], [9000]),                    # few rows, many keys: split
    (8, 2, [1, 7], [3000, 5000]),
    (64, 32, [70, 1, 130, 5, 0, 64, 20, 33, 257], [70, 1, 140, 5, 0, 300, 20, 20, 257]),  # tiles of 256 rows
    (20, 4, [3, 60], [7000, 2000]),         # tokens whose heads lie in two tiles of rows, in parts
]


def prompt_scores(q, k, scale):
    """Relative error of the weights: 128 fp32 accumulations of q k, and the exponent's own rounding."""
    big = np.linalg.norm(q.astype(np.float64), axis=-1).max() * np.linalg.norm(k.astype(np.float64), axis=-1).max() if k.size else 0.0
    return 140 * 2.0 ** -24 * big * scale + 2.0 ** -18


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("case", PROMPT, ids=lambda c: f"{c[0]}x{c[1]}-{'_'.join(map(str, c[2]))}of{'_'.join(map(str, c[3]))}")
def test_prompt_attention(case, causal):
    Hq, H, nq, nk = case
    g = rng(sum(nq) + Hq)
    cu_q, cu_k = (np.concatenate([[1], 1 + np.cumsum(n)]) for n in (nq, nk))
    Tq, Tk = int(cu_q[-1]) + 2, int(cu_k[-1]) + 1
    q, k, v = heads_of(g, Tq, Hq), heads_of(g, Tk, H), heads_of(g, Tk, H)
    for x in (k, v):  # rows of no sequence
        x[0] = x[-1] = np.nan
    out = torch.full((Tq, Hq, 128), 7.0, dtype=torch.float16, device=DEV)
    n = sq.attn_prompt_workspace_bytes(len(nq), Tq, Tk, Hq, H)
    ws = torch.full((n + 16,), 255, dtype=torch.uint8, device=DEV)
    got = sq.attn_prompt(up(q), up(k), up(v), ints(cu_q), ints(cu_k), causal=causal, out=out, workspace=ws)
    torch.cuda.synchronize()
    want, weight, rows = opg.attn_prompt(q, k, v, cu_q, cu_k, causal=causal)
    attention_close(got[torch.tensor(rows, device=DEV)], want[rows], weight[rows], prompt_scores(q, k[1:-1], 128 ** -0.5))
    assert torch.all(got[torch.tensor(~rows, device=DEV)] == 7.0)
    assert torch.equal(sq.attn_prompt(up(q), up(k), up(v), ints(cu_q), ints(cu_k), causal=causal)[1:-2], got[1:-2])


def test_prompt_attention_of_a_fused_projection():
    g = rng(21)
    T, Hq, H = 150, 8, 2
    x = heads_of(g, T, Hq + 2 * H, 2.0)  # sharper scores
    fused = up(x)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + H], x[:, Hq + H:]
    cu = [0, 90, 150]
    wide = torch.full((T, Hq + 1, 128), 7.0, dtype=torch.float16, device=DEV)
    got = sq.attn_prompt(fused[:, :Hq], fused[:, Hq:Hq + H], fused[:, Hq + H:], ints(cu), ints(cu), scale=0.2, out=wide[:, 1:])
    torch.cuda.synchronize()
    want, weight, _ = opg.attn_prompt(q, k, v, cu, cu, 0.2)
    attention_close(got, want, weight, prompt_scores(q, k, 0.2))
    assert torch.all(wide[:, 0] == 7.0)


@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("n,m,H,at", [(200, 200, 2, 77), (90, 90, 300, 77), (40, 3000, 2, 2970), (40, 3000, 2, 100)],
                         ids=["halves", "whole", "parts", "parts_early"])
def test_prompt_values_that_a_row_does_not_see(n, m, H, at, value, which):
    """A key or value that is not finite reaches the rows that see it and no other."""
    g = rng(22)
    q, k, v = heads_of(g, n, H), heads_of(g, m, H), heads_of(g, m, H)
    (k if which == "k" else v)[at, 1, 5] = value
    got = f64(sq.attn_prompt(up(q), up(k), up(v), ints([0, n]), ints([0, m])))
    clean = k if which == "k" else v
    clean[at, 1, 5] = 0
    want, weight, _ = opg.attn_prompt(q, k, v, [0, n], [0, m])
    ok = np.ones((n, H), dtype=bool)
    first = max(0, at - (m - n))  # the first row that sees it
    ok[first:, 1] = False
    tol = (2.0 ** -11 + prompt_scores(q, k, 128 ** -0.5)) * weight + 2.0 ** -11 * np.abs(want) + 2.0 ** -25
    assert np.all((np.abs(got - want) <= tol)[ok])
    hit = got[first:, 1]
    if which == "v":
        assert np.all(np.isnan(hit[:, 5])) if np.isnan(value) else np.all(hit[:, 5] == value)
        others = np.arange(128) != 5
        assert np.all((np.abs(got - want) <= tol)[first:, 1][:, others])
    elif np.isnan(value):
        assert np.all(np.isnan(hit))


def test_prompt_attention_of_extreme_scores():
    """Scores of thousands, and of the type's lowest value, keep a softmax."""
    g = rng(23)
    T = 130
    q, k, v = (heads_of(g, T, 1) for _ in range(3))
    q[:, 0, 0], k[:, 0, 0] = 60000, np.where(np.arange(T) % 3 == 0, -60000, -59000)
    got = sq.attn_prompt(up(q), up(k), up(v), ints([0, T]), ints([0, T]), scale=1e-6)
    want, weight, _ = opg.attn_prompt(q, k, v, [0, T], [0, T], 1e-6)
    attention_close(got, want, weight, 140 * 2.0 ** -24 * 3600)


def test_a_conversation():
    """A prompt in two chunks, then tokens: each call's input is the one before's output."""
    g = rng(31)
    Hq, H, page, bits = 8, 2, 16, 4
    B = 3
    first, second, steps = [40, 9, 70], [33, 1, 20], 3
    total = [a + b + steps for a, b in zip(first, second)]
    table, pages = spread_table(g, total, page)
    cache = {n: np.zeros_like(a) for n, a in filled(g, pages, H, page, bits, np.float32).items()}
    freq = opg.rope_frequencies(128, 500000.0, "by parts", 8.0)
    dfreq = sq.rope_frequencies(128, 500000.0, "by parts", 8.0, device=DEV)
    dc, dt = device_cache(cache), ints(table)
    assert [tuple(t.shape) for t in sq.kv_cache(pages, page, H, bits)] == [tuple(t.shape) for t in dc]

    lens = np.zeros(B, dtype=np.int64)
    for new in (first, second):
        lens = lens + np.array(new)
        cu = np.concatenate([[0], np.cumsum(new)])
        cu_k = np.concatenate([[0], np.cumsum(lens)])
        T = int(cu[-1])
        q, k, v = heads_of(g, T, Hq), heads_of(g, T, H), heads_of(g, T, H)
        o = opg.rope_kv_write(q, k, v, cache, cu, lens, table, freq)
        qr = sq.rope_kv_write(up(q), up(k), up(v), dc, dt, ints(lens), dfreq, cu=ints(cu))
        check_write(o, qr, dc, q, bits, o["rows"])
        cache = {n: t.cpu().numpy() for n, t in zip(("k_q", "v_q", "params"), dc)}
        kk, vv = sq.kv_read(dc, dt, ints(lens), ints(cu_k), int(cu_k[-1]))
        out = sq.attn_prompt(qr, kk, vv, ints(cu), ints(cu_k))
        ok, ov, _ = opg.kv_read(cache, cu_k, lens, table, int(cu_k[-1]))
        want, weight, _ = opg.attn_prompt(qr.cpu().numpy(), ok, ov, cu, cu_k)
        # keys and values rounded to fp16 on the way: 2^-11 of them, scores 2^-11 sum |q k| scale
        attention_close(out, want, weight, 2.0 ** -11 + prompt_scores(qr.cpu().numpy(), ok, 128 ** -0.5) + 2.0 ** -11 * 16)
    most = max(total)
    ws = torch.empty(sq.attn_paged_workspace_bytes(B, most, Hq, H), dtype=torch.uint8, device=DEV)
    # the step is captured once; its replays see longer lengths and new rows
    bufs = [torch.zeros((B, h, 128), dtype=torch.float16, device=DEV) for h in (Hq, H, H)]
    dl = ints(lens)
    qr, out = torch.empty_like(bufs[0]), torch.empty_like(bufs[0])

    def step():
        sq.rope_kv_write(*bufs, dc, dt, dl, dfreq, out=qr)
        sq.attn_paged(qr, dc, dt, dl, most, out=out, workspace=ws)

    saved = [t.clone() for t in dc]
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for t, s in zip(dc, saved):
        t.copy_(s)
    for _ in range(steps):
        lens = lens + 1
        q, k, v = heads_of(g, B, Hq), heads_of(g, B, H), heads_of(g, B, H)
        for t, x in zip(bufs, (q, k, v)):
            t.copy_(up(x))
        dl.copy_(ints(lens))
        before = [t.clone() for t in dc]
        graph.replay()
        torch.cuda.synchronize()
        o = opg.rope_kv_write(q, k, v, cache, np.arange(B + 1), lens, table, freq)
        check_write(o, qr, dc, q, bits, o["rows"])
        cache = {n: t.cpu().numpy() for n, t in zip(("k_q", "v_q", "params"), dc)}
        want, weight = opg.attn_paged(qr.cpu().numpy(), cache, lens, table, most)
        attention_close(out, want, weight, 2e-5)
        replayed = [t.clone() for t in (qr, out, *dc)]
        for t, s in zip(dc, before):
            t.copy_(s)
        step()  # the same step eagerly
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, (qr, out, *dc)))


def test_another_stream_and_two_workspaces():
    g = rng(41)
    lens = [700, 90]
    table, pages = spread_table(g, lens, 16)
    cache = filled(g, pages, 2, 16, 4, np.float32)
    q = up(heads_of(g, 2, 8))
    dc, dt, dl = device_cache(cache), ints(table), ints(lens)
    want = sq.attn_paged(q, dc, dt, dl, 700)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = sq.attn_paged(q, dc, dt, dl, 700)
    other = sq.attn_paged(q, dc, dt, dl, 700)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(other, want)


def test_two_graphs_that_share_a_workspace():
    """Replayed in any order on one stream, with lengths that change and other work between them."""
    g = rng(42)
    page, most, Hq, H = 16, 2000, 16, 2
    n = max(sq.attn_paged_workspace_bytes(b, most, Hq, H) for b in (1, 3))
    pq, pk = [5, 20], [1500, 1900]
    n = max(n, sq.attn_prompt_workspace_bytes(2, sum(pq), sum(pk), Hq, H))
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    calls = []
    for B, bits in ((1, 4), (3, 8)):
        table, pages = spread_table(g, [most] * B, page)
        dc, dt, dl = device_cache(filled(g, pages, H, page, bits, np.float32)), ints(table), ints([most] * B)
        q, out = up(heads_of(g, B, Hq)), torch.empty((B, Hq, 128), dtype=torch.float16, device=DEV)
        calls.append((dl, out, lambda q=q, dc=dc, dt=dt, dl=dl, out=out, ws=ws: sq.attn_paged(q, dc, dt, dl, most, out=out, workspace=ws)))
    q, k, v = up(heads_of(g, sum(pq), Hq)), up(heads_of(g, sum(pk), H)), up(heads_of(g, sum(pk), H))
    cq, ck = ints([0, *np.cumsum(pq)]), ints([0, *np.cumsum(pk)])
    out = torch.empty_like(q)
    calls.append((None, out, lambda: sq.attn_prompt(q, k, v, cq, ck, out=out, workspace=ws)))
    assert sq.attn_prompt_workspace_bytes(2, sum(pq), sum(pk), Hq, H) > 0
    graphs = []
    for _, _, call in calls:
        call()
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call()
    for step in range(4):
        for dl, out, _ in calls:
            out.fill_(7.0)
            if dl is not None:
                dl.copy_(ints([[1, 700, most, 64][(step + b) % 4] for b in range(dl.numel())]))
        for i in ((0, 1, 2), (2, 1, 0), (1, 0, 2), (0, 2, 1))[step]:
            graphs[i].replay()
        torch.cuda.synchronize()
        got = [out.clone() for _, out, _ in calls]
        for (_, out, call), have in zip(calls, got):
            assert torch.equal(call(), have)


@pytest.mark.parametrize("bits", [4, 8])
def test_pages_beyond_32_bits(bits):
    """Codes and parameters that lie behind the pool's first 4 GiB of each."""
    g = rng(43)
    H, page, n = 2, 64, 300
    table, used = spread_table(g, [n], page)
    small = filled(g, used, H, page, bits, np.float32)
    pages = (1 << 32) // (H * page * 16) + 3 * used  # 4 GiB of parameters, 16 or 32 of codes
    dc = [torch.empty((pages, *small[x].shape[1:]), dtype=t, device=DEV) for x, t in
          (("k_q", torch.uint8), ("v_q", torch.uint8), ("params", torch.float32))]
    for t, x in zip(dc, ("k_q", "v_q", "params")):
        t[-used:] = up(small[x])
    far = ints(table + pages - used)
    near = device_cache(small)
    q, k, v = up(heads_of(g, 1, 4)), up(heads_of(g, 1, H)), up(heads_of(g, 1, H))
    results = []
    for cache, dt in ((near, ints(table)), (dc, far)):
        qr = sq.rope_kv_write(q, k, v, cache, dt, ints([n]), sq.rope_frequencies(device=DEV))
        out = sq.attn_paged(qr, cache, dt, ints([n]), n)
        kk, vv = sq.kv_read(cache, dt, ints([n]), ints([0, n]), n)
        results.append([qr, out, kk, vv, *(t[-used:] for t in cache)])
    torch.cuda.synchronize()
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_prompt_rows_beyond_32_bits():
    """Sequences of q, k, v and out whose rows lie behind 4 GiB."""
    g = rng(44)
    Hq, H, n, m, wide = 4, 2, 40, 150, 1 << 15
    rows = (1 << 32) // (2 * wide) + 200
    q, k, v = (heads_of(g, x, h) for x, h in ((n, Hq), (m, H), (m, H)))
    # (the division of the keys goes by the rows of all k: not the bits of a call on the rows alone)
    want, weight, _ = opg.attn_prompt(q, k, v, [0, n], [0, m])
    # the four tensors are columns of one each, so that a row is 64 KiB
    far = []
    for x, h in ((q, Hq), (k, H), (v, H)):
        t = torch.empty((rows, wide), dtype=torch.float16, device=DEV)[:, :h * 128].unflatten(1, (h, 128))
        t[rows - len(x):] = up(x)
        far.append(t)
    out = torch.full((rows, wide), 7.0, dtype=torch.float16, device=DEV)[:, :Hq * 128].unflatten(1, (Hq, 128))
    sq.attn_prompt(*far, ints([rows - n, rows]), ints([rows - m, rows]), out=out)
    torch.cuda.synchronize()
    attention_close(out[-n:], want, weight, prompt_scores(q, k, 128 ** -0.5))
    assert torch.all(out[:-n] == 7.0)


def test_empty_calls():
    cache, dt = sq.kv_cache(1, 16, 2), torch.zeros((0, 1), dtype=torch.int32, device=DEV)
    none = torch.empty((0, 2, 128), dtype=torch.float16, device=DEV)
    z = torch.zeros((0,), dtype=torch.int32, device=DEV)
    one = torch.zeros((1,), dtype=torch.int32, device=DEV)
    assert sq.rope_kv_write(none, none, none, cache, dt, z).shape == (0, 2, 128)
    assert sq.kv_read(cache, dt, z, one, 0)[0].shape == (0, 2, 128)
    assert sq.attn_paged(none, cache, dt, z, 16).shape == (0, 2, 128)
    assert sq.attn_prompt(none, none, none, one, one).shape == (0, 2, 128)
    q = torch.zeros((3, 2, 128), dtype=torch.float16, device=DEV)
    out = sq.attn_prompt(q, none, none, ints([0, 3]), ints([0, 0]))
    assert torch.all(out == 0)


def test_binding_refusals():
    q = torch.zeros((4, 8, 128), dtype=torch.float16, device=DEV)
    k = torch.zeros((4, 2, 128), dtype=torch.float16, device=DEV)
    cache, lens, cu = sq.kv_cache(4, 16, 2), ints([4]), ints([0, 4])
    table = ints([[0, 1]])
    freq = sq.rope_frequencies(device=DEV)
    for bad in (lambda: sq.rope_kv_write(q, k[:3], k, cache, table, lens, freq, cu=cu),
                lambda: sq.rope_kv_write(q, k, k, sq.kv_cache(4, 16, 4), table, lens, freq, cu=cu),
                lambda: sq.rope_kv_write(q, k, k, cache, table, lens, freq, cu=ints([0, 2, 4])),
                lambda: sq.rope_kv_write(q.transpose(0, 1), k, k, cache, table, lens, freq, cu=cu),
                lambda: sq.rope_kv_write(q[..., :64], k, k, cache, table, lens, freq, cu=cu),
                lambda: sq.kv_read(cache, table[:, 0], lens, cu, 4),
                lambda: sq.kv_read((cache[0], cache[1], cache[2][:2]), table, lens, cu, 4),
                lambda: sq.kv_read(cache, table, lens, cu, 4, out=(k[:2], k[2:])),
                lambda: sq.attn_paged(q[:1], cache, table.t(), lens, 16),
                lambda: sq.attn_prompt(q, k, k[:3], cu, cu),
                lambda: sq.attn_prompt(q, k, k, cu, ints([0, 1, 4]))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: sq.rope_kv_write(q.float(), k, k, cache, table, lens, freq, cu=cu),
                lambda: sq.rope_kv_write(q, k, k, cache, table, lens, freq.float(), cu=cu),
                lambda: sq.attn_paged(q[:1], cache, table.long(), lens, 16),
                lambda: sq.attn_prompt(q, k, k, cu.long(), cu)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: sq.rope_kv_write(q, k, k, cache, table, lens, freq),            # four rows, one sequence
                lambda: sq.attn_paged(q[:1, :3], cache, table, lens, 16),
                lambda: sq.attn_paged(q[:1], cache, table, lens, 0),
                lambda: sq.attn_paged(q[:1], cache, table, lens, 4096, workspace=torch.empty(16, dtype=torch.uint8, device=DEV)),
                lambda: sq.attn_prompt(q, k, k, cu, cu, out=q)):
        with pytest.raises(sq.SqError):
            bad()
