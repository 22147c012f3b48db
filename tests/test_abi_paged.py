"""Refusals of the paged-cache entry points on the host, before anything is enqueued (fake,
never-dereferenced pointers), and the binding's own checks."""

import ctypes
import os

import numpy as np
import pytest
import torch

from paper_2405_16406_amd import sq

BASE = 0x1000000000


def fake(i, off=0):
    return ctypes.c_void_p(BASE * (i + 1) + off)


@pytest.fixture(scope="module")
def L():
    if os.environ.get("SQ_TEST_LIBRARY"):
        sq._lib = sq.load(os.environ["SQ_TEST_LIBRARY"])
    return sq.lib()


def cache_args(kw):
    return (kw.get("table", fake(4)), kw.get("ldt", 8), kw.get("cols", 8), kw.get("kq", fake(5)), kw.get("vq", fake(6)),
            kw.get("params", fake(7)), kw.get("pages", 16), kw.get("page", 16), kw.get("Hkv", 2))


def write(L, **kw):
    f32 = ctypes.c_float
    return L.sq_rope_kv_write(kw.get("q", fake(0)), kw.get("ldq", 1024), kw.get("k", fake(1)), kw.get("ldk", 256),
                              kw.get("v", fake(2)), kw.get("ldv", 256), kw.get("T", 4), kw.get("Hq", 8), kw.get("D", 128),
                              kw.get("cu", fake(3)), kw.get("lens", fake(8)), kw.get("B", 3), *cache_args(kw), kw.get("bits", 4),
                              kw.get("pbits", 32), kw.get("freq", fake(9)), kw.get("rotary", 128), kw.get("inter", 0),
                              f32(kw.get("mag", 1.0)), f32(kw.get("kc", 1.0)), f32(kw.get("vc", 1.0)), kw.get("qr", fake(10)),
                              kw.get("kr", None), None)


def read(L, **kw):
    return L.sq_kv_read(kw.get("cu", fake(3)), kw.get("lens", fake(8)), kw.get("B", 3), kw.get("T", 4), *cache_args(kw),
                        kw.get("D", 128), kw.get("bits", 4), kw.get("pbits", 32), kw.get("plain", 0), kw.get("k", fake(1)),
                        kw.get("ldk", 256), kw.get("v", fake(2)), kw.get("ldv", 256), None)


def paged(L, **kw):
    return L.sq_attn_paged(kw.get("q", fake(0)), kw.get("ldq", 1024), kw.get("lens", fake(8)), kw.get("B", 3), *cache_args(kw),
                           kw.get("Hq", 8), kw.get("D", 128), kw.get("bits", 4), kw.get("pbits", 32), kw.get("max_len", 128),
                           ctypes.c_float(kw.get("scale", 0.1)), kw.get("out", fake(10)), kw.get("ldo", 1024),
                           kw.get("ws", fake(11)), kw.get("wsb", 1 << 20), None)


def prompt(L, **kw):
    return L.sq_attn_prompt(kw.get("q", fake(0)), kw.get("ldq", 1024), kw.get("k", fake(1)), kw.get("ldk", 256),
                            kw.get("v", fake(2)), kw.get("ldv", 256), kw.get("cuq", fake(3)), kw.get("cuk", fake(4)),
                            kw.get("B", 3), kw.get("Tq", 4), kw.get("Tk", 9), kw.get("Hq", 8), kw.get("Hkv", 2),
                            kw.get("D", 128), ctypes.c_float(kw.get("scale", 0.1)), kw.get("causal", 1), kw.get("out", fake(10)),
                            kw.get("ldo", 1024), kw.get("ws", fake(11)), kw.get("wsb", 1 << 20), None)


CACHE = [(dict(page=24), "SHAPE"), (dict(page=8), "SHAPE"), (dict(page=1 << 21), "SHAPE"), (dict(pages=0), "SHAPE"),
         (dict(pages=1 << 37, page=16), "SHAPE"), (dict(cols=0), "SHAPE"), (dict(cols=9), "SHAPE"), (dict(bits=6), "UNSUPPORTED"),
         (dict(pbits=8), "UNSUPPORTED"), (dict(D=64), "UNSUPPORTED"), (dict(B=-1), "SHAPE"), (dict(table=None), "NULL"),
         (dict(lens=None), "NULL"), (dict(params=None), "NULL"), (dict(kq=fake(5, 8)), "ALIGN"), (dict(params=fake(7, 8)), "ALIGN"),
         (dict(pbits=16, params=fake(7, 4)), "ALIGN"), (dict(table=fake(4, 2)), "ALIGN"), (dict(lens=fake(8, 2)), "ALIGN")]


@pytest.mark.parametrize("kw,status", CACHE)
def test_cache_arguments(L, kw, status):
    for call in (write, read, paged):
        assert call(L, **kw) == getattr(sq, "SQ_ERR_" + status), (call, kw)


def test_write_refusals(L):
    for n in ("q", "k", "v", "qr", "freq"):
        assert write(L, **{n: None}) == sq.SQ_ERR_NULL
    for kw in (dict(T=-1), dict(T=1 << 31), dict(cu=None), dict(Hq=7), dict(Hq=1), dict(Hq=1 << 17, ldq=1 << 24), dict(ldq=1016),
               dict(ldk=128), dict(ldv=1 << 24), dict(rotary=120), dict(rotary=144), dict(rotary=-16), dict(rotary=0),
               dict(mag=float("nan")), dict(kc=0.0), dict(vc=1.5)):
        assert write(L, **kw) == sq.SQ_ERR_SHAPE, kw
    assert write(L, inter=2) == sq.SQ_ERR_UNSUPPORTED
    for kw in (dict(ldq=1028), dict(q=fake(0, 8)), dict(qr=fake(10, 4)), dict(kr=fake(12, 2)), dict(freq=fake(9, 4)), dict(cu=fake(3, 1))):
        assert write(L, **kw) == sq.SQ_ERR_ALIGN, kw
    for kw in (dict(qr=fake(0, 1024)), dict(kr=fake(10, 1024)), dict(vq=fake(5, 1024)), dict(params=fake(6, 16)), dict(qr=fake(4)),
               dict(kr=fake(8)), dict(qr=fake(9, 496))):
        assert write(L, **kw) == sq.SQ_ERR_ALIAS, kw
    # q, k and v may share rows of one projection's output; nothing to do is fine
    assert write(L, T=0, k=fake(0, 2048), ldq=1536, ldk=1536) == sq.SQ_OK
    assert write(L, T=0, B=0, cu=None, freq=None, rotary=0) == sq.SQ_OK


def test_read_refusals(L):
    for n in ("cu", "k", "v"):
        assert read(L, **{n: None}) == sq.SQ_ERR_NULL
    assert read(L, T=-1) == sq.SQ_ERR_SHAPE
    assert read(L, ldk=248) == sq.SQ_ERR_SHAPE
    assert read(L, Hkv=0) == sq.SQ_ERR_SHAPE
    assert read(L, plain=3) == sq.SQ_ERR_UNSUPPORTED
    assert read(L, ldv=260) == sq.SQ_ERR_ALIGN
    assert read(L, v=fake(2, 8)) == sq.SQ_ERR_ALIGN
    assert read(L, k=fake(5)) == sq.SQ_ERR_ALIAS
    assert read(L, v=fake(1, 512)) == sq.SQ_ERR_ALIAS
    assert read(L, T=0) == sq.SQ_OK


def test_paged_attention_refusals(L):
    for n in ("q", "out"):
        assert paged(L, **{n: None}) == sq.SQ_ERR_NULL
    for kw in (dict(Hq=9), dict(B=1 << 21), dict(max_len=0), dict(max_len=1 << 30), dict(ldq=1000), dict(ldo=1 << 24),
               dict(scale=float("inf")), dict(scale=float("nan"))):
        assert paged(L, **kw) == sq.SQ_ERR_SHAPE, kw
    for kw in (dict(q=fake(0, 8)), dict(out=fake(10, 8)), dict(ws=fake(11, 8)), dict(ldo=1028)):
        assert paged(L, **kw) == sq.SQ_ERR_ALIGN, kw
    for kw in (dict(out=fake(0)), dict(ws=fake(7)), dict(ws=fake(10, 16)), dict(out=fake(4))):
        assert paged(L, **kw) == sq.SQ_ERR_ALIAS, kw
    assert paged(L, B=0) == sq.SQ_OK
    n = ctypes.c_uint64(3)
    assert L.sq_attn_paged_workspace(1, 64, 8, 2, 128, None) == sq.SQ_ERR_NULL
    assert L.sq_attn_paged_workspace(1, 0, 8, 2, 128, ctypes.byref(n)) == sq.SQ_ERR_SHAPE
    assert L.sq_attn_paged_workspace(1, 64, 8, 3, 128, ctypes.byref(n)) == sq.SQ_ERR_SHAPE
    assert L.sq_attn_paged_workspace(1, 64, 8, 2, 64, ctypes.byref(n)) == sq.SQ_ERR_UNSUPPORTED
    assert n.value == 3


def test_prompt_refusals(L):
    for n in ("q", "out", "cuq", "cuk", "k"):
        assert prompt(L, **{n: None}) == sq.SQ_ERR_NULL
    for kw in (dict(Tq=-1), dict(Tk=1 << 31), dict(B=-1), dict(Hkv=3), dict(Hkv=0), dict(Tq=1 << 28), dict(B=1 << 22, Tq=4),
               dict(ldk=248), dict(scale=float("inf")), dict(ldo=8)):
        assert prompt(L, **kw) == sq.SQ_ERR_SHAPE, kw
    assert prompt(L, causal=2) == sq.SQ_ERR_UNSUPPORTED
    assert prompt(L, D=256) == sq.SQ_ERR_UNSUPPORTED
    for kw in (dict(ldq=1028), dict(k=fake(1, 2)), dict(cuq=fake(3, 2)), dict(ws=fake(11, 4))):
        assert prompt(L, **kw) == sq.SQ_ERR_ALIGN, kw
    for kw in (dict(out=fake(0, 16)), dict(out=fake(2)), dict(ws=fake(10)), dict(out=fake(3))):
        assert prompt(L, **kw) == sq.SQ_ERR_ALIAS, kw
    assert prompt(L, Tq=0) == sq.SQ_OK
    assert prompt(L, B=0, k=None, v=None, Tk=0) == sq.SQ_OK
    n = ctypes.c_uint64(3)
    assert L.sq_attn_prompt_workspace(1, 4, 4, 8, 2, 128, None) == sq.SQ_ERR_NULL
    assert L.sq_attn_prompt_workspace(1, -4, 4, 8, 2, 128, ctypes.byref(n)) == sq.SQ_ERR_SHAPE
    assert n.value == 3


def test_frequency_refusals(L):
    buf = np.full(64, 7.0)
    f = lambda *a: L.sq_rope_frequencies(a[0], ctypes.c_double(a[1]), a[2], *(ctypes.c_double(x) for x in a[3:]),  # noqa: E731
                                         buf.ctypes.data_as(ctypes.c_void_p))
    assert L.sq_rope_frequencies(128, ctypes.c_double(1e4), 0, *(ctypes.c_double(1.0),) * 4, None) == sq.SQ_ERR_NULL
    inf, nan = float("inf"), float("nan")
    for bad in ((24, 1e4, 0, 1, 1, 4, 8), (0, 1e4, 0, 1, 1, 4, 8), (144, 1e4, 0, 1, 1, 4, 8), (128, 0, 0, 1, 1, 4, 8),
                (128, nan, 0, 1, 1, 4, 8), (128, inf, 0, 1, 1, 4, 8), (128, 1e4, 1, 0.5, 1, 4, 8), (128, 1e4, 2, nan, 1, 4, 8),
                (128, 1e4, 2, 8, 4, 4, 8), (128, 1e4, 2, 8, 1, inf, 8), (128, 1e4, 2, 8, 1, 4, 0)):
        assert f(*bad) == sq.SQ_ERR_SHAPE, bad
    assert f(128, 1e4, 3, 1, 1, 4, 8) == sq.SQ_ERR_UNSUPPORTED
    assert np.all(buf == 7.0)
    with pytest.raises(sq.SqError):
        sq.rope_frequencies(24)
    with pytest.raises(ValueError):
        sq.rope_frequencies(128, scaling="other")


@pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="a GPU driver is present: the calls below would "
                    "launch kernels on fake pointers")
def test_no_device_is_a_hip_error(L):
    for call in (write, read, paged, prompt):
        assert call(L) == sq.SQ_ERR_HIP, call
    n = ctypes.c_uint64(0)
    assert L.sq_attn_paged_workspace(1, 64, 8, 2, 128, ctypes.byref(n)) == sq.SQ_ERR_HIP


@pytest.mark.parametrize("call,kw,ok", [
    (paged, dict(scale=2.0 ** 40 * 1.001), False), (paged, dict(scale=-2.0 ** 41), False), (paged, dict(scale=3e38), False),
    (paged, dict(scale=-0.1, B=0), True), (paged, dict(scale=0.0, B=0), True), (paged, dict(scale=2.0 ** 40, B=0), True),
    (prompt, dict(scale=0.0), False), (prompt, dict(scale=-0.1), False), (prompt, dict(scale=-0.0), False),
    (prompt, dict(scale=2.0 ** 40 * 1.001), False), (prompt, dict(scale=2.0 ** 40, B=0), True)])
def test_scales(L, call, kw, ok):
    """Scales whose base-2 factor overflows, and those that turn the order of a prompt's scores around."""
    assert call(L, **kw) == (sq.SQ_OK if ok else sq.SQ_ERR_SHAPE)


def test_read_into_one_tensor(L):
    """Two outputs in one tensor's rows: their spans overlap."""
    assert read(L, k=fake(1), ldk=512, v=fake(1, 512), ldv=512) == sq.SQ_ERR_ALIAS


def test_binding_refuses_host_tensors():
    x = torch.zeros((2, 4, 128), dtype=torch.float16)
    lens = torch.ones(2, dtype=torch.int32)
    cache = sq.kv_cache(1, 16, 4, device="cpu")
    with pytest.raises(TypeError):
        sq.rope_kv_write(x, x, x, cache, lens[:, None], lens)
    with pytest.raises(TypeError):
        sq.kv_read(cache, lens[:, None], lens, lens, 2)
    with pytest.raises(TypeError):
        sq.attn_paged(x, cache, lens[:, None], lens, 16)
    with pytest.raises(TypeError):
        sq.attn_prompt(x, x, x, lens, lens)


@pytest.mark.parametrize("bad", [lambda t: t[::2], lambda t: t[:1].expand(64), lambda t: t.view(8, 8).t()], ids=["strided", "expanded", "transposed"])
def test_workspaces_are_contiguous(bad):
    """A workspace whose bytes are not side by side is refused before anything else is looked at."""
    t = torch.zeros(64, dtype=torch.uint8)
    with pytest.raises(ValueError):
        sq._workspace_bytes(bad(t))
    with pytest.raises(TypeError):  # on the host
        sq._workspace_bytes(t)


def test_frequencies_that_overflow(L):
    """theta^(-126 / 128) of the smallest doubles is infinite; nothing is written then."""
    buf = np.full(64, 7.0)
    ptr = buf.ctypes.data_as(ctypes.c_void_p)
    rest = (ctypes.c_double(1.0), ctypes.c_double(1.0), ctypes.c_double(4.0), ctypes.c_double(8192.0))
    for theta, scaling in ((5e-324, 0), (5e-324, 1), (1e-320, 2)):
        assert L.sq_rope_frequencies(128, ctypes.c_double(theta), scaling, *rest, ptr) == sq.SQ_ERR_SHAPE
    assert np.all(buf == 7.0)
    assert L.sq_rope_frequencies(128, ctypes.c_double(1e-300), 0, *rest, ptr) == sq.SQ_OK and np.all(np.isfinite(buf))
