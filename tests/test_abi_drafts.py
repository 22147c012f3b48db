"""Refusals of the calls on drafts, windows and page tables on the host, before anything is enqueued (fake,
never-dereferenced pointers), and the binding's own checks."""

import ctypes
import os

import pytest
import torch

from paper_2405_16406_amd import sq
from test_abi_paged import CACHE, L, cache_args, fake  # noqa: F401

F32 = ctypes.c_float


def mask(L, **kw):
    return L.sq_tree_mask(kw.get("parents", fake(0)), kw.get("cu", fake(1)), kw.get("lens", fake(2)), kw.get("B", 3), kw.get("T", 9),
                          kw.get("window", 0), kw.get("sinks", 0), kw.get("mask", fake(3)), kw.get("ldm", 4), kw.get("words", 2),
                          kw.get("depth", fake(4)), None)


def write_ex(L, **kw):
    return L.sq_rope_kv_write_ex(kw.get("q", fake(0)), kw.get("ldq", 1024), kw.get("k", fake(1)), kw.get("ldk", 256),
                                 kw.get("v", fake(2)), kw.get("ldv", 256), kw.get("T", 4), kw.get("Hq", 8), kw.get("D", 128),
                                 kw.get("cu", fake(3)), kw.get("lens", fake(8)), kw.get("B", 3), kw.get("depth", fake(13)),
                                 *cache_args(kw), kw.get("bits", 4), kw.get("pbits", 32), kw.get("freq", fake(9)),
                                 kw.get("rotary", 128), kw.get("inter", 0), F32(kw.get("mag", 1.0)), F32(1.0), F32(1.0),
                                 kw.get("qr", fake(10)), kw.get("kr", None), None)


def tree(L, **kw):
    return L.sq_attn_tree(kw.get("q", fake(0)), kw.get("ldq", 1024), kw.get("cu", fake(1)), kw.get("lens", fake(8)), kw.get("B", 3),
                          kw.get("T", 9), kw.get("mask", fake(2)), kw.get("ldm", 2), kw.get("words", 1), kw.get("depth", fake(3)),
                          kw.get("window", 0), kw.get("sinks", 0), *cache_args(kw), kw.get("Hq", 8), kw.get("D", 128),
                          kw.get("bits", 4), kw.get("pbits", 32), kw.get("max_len", 128), F32(kw.get("scale", 0.1)),
                          kw.get("out", fake(10)), kw.get("ldo", 1024), kw.get("ws", fake(11)), kw.get("wsb", 1 << 20), None)


def paged(L, **kw):
    return L.sq_attn_paged_window(kw.get("q", fake(0)), kw.get("ldq", 1024), kw.get("lens", fake(8)), kw.get("B", 3),
                                  kw.get("window", 16), kw.get("sinks", 2), *cache_args(kw), kw.get("Hq", 8), kw.get("D", 128),
                                  kw.get("bits", 4), kw.get("pbits", 32), kw.get("max_len", 128), F32(kw.get("scale", 0.1)),
                                  kw.get("out", fake(10)), kw.get("ldo", 1024), kw.get("ws", fake(11)), kw.get("wsb", 1 << 20), None)


def prompt(L, **kw):
    return L.sq_attn_prompt_window(kw.get("q", fake(0)), kw.get("ldq", 1024), kw.get("k", fake(1)), kw.get("ldk", 256),
                                   kw.get("v", fake(2)), kw.get("ldv", 256), kw.get("cuq", fake(3)), kw.get("cuk", fake(4)),
                                   kw.get("B", 3), kw.get("Tq", 4), kw.get("Tk", 9), kw.get("Hq", 8), kw.get("Hkv", 2),
                                   kw.get("D", 128), F32(kw.get("scale", 0.1)), kw.get("window", 16), kw.get("sinks", 2),
                                   kw.get("out", fake(10)), kw.get("ldo", 1024), kw.get("ws", fake(11)), kw.get("wsb", 1 << 20), None)


def release(L, **kw):
    return L.sq_paged_release(kw.get("first", fake(0)), kw.get("end", fake(1)), kw.get("held", fake(2)), kw.get("B", 3),
                              kw.get("table", fake(3)), kw.get("ldt", 8), kw.get("cols", 8), kw.get("page", 16), kw.get("pool", fake(4)),
                              kw.get("count", fake(5)), kw.get("pages", 16), None)


def grow(L, **kw):
    return L.sq_paged_grow(kw.get("have", fake(0)), kw.get("add", fake(1)), kw.get("held", fake(2)), kw.get("B", 3), kw.get("T", 9),
                           kw.get("table", fake(3)), kw.get("ldt", 8), kw.get("cols", 8), kw.get("page", 16), kw.get("pool", fake(4)),
                           kw.get("count", fake(5)), kw.get("pages", 16), kw.get("lens", fake(6)), kw.get("cu", fake(7)),
                           kw.get("pos", fake(8)), kw.get("slots", fake(9)), kw.get("missing", fake(10)), None)


def keep(L, **kw):
    return L.sq_kv_keep(kw.get("cu", fake(0)), kw.get("lens", fake(8)), kw.get("B", 3), kw.get("path", fake(1)), kw.get("ldp", 8),
                        kw.get("most", 8), kw.get("kept", fake(2)), *cache_args(kw), kw.get("D", 128), kw.get("bits", 4),
                        kw.get("pbits", 32), kw.get("out", fake(10)), None)


@pytest.mark.parametrize("kw,status", CACHE)
def test_cache_arguments(L, kw, status):  # noqa: F811
    for call in (tree, paged, keep, write_ex):
        assert call(L, **kw) == getattr(sq, "SQ_ERR_" + status), (call, kw)


def test_tree_mask_refusals(L):  # noqa: F811
    for n in ("parents", "cu", "mask", "depth"):
        assert mask(L, **{n: None}) == sq.SQ_ERR_NULL
    assert mask(L, lens=None, window=4, sinks=1) == sq.SQ_ERR_NULL
    for kw in (dict(T=-1), dict(B=-1), dict(T=1 << 31), dict(words=0), dict(words=5), dict(words=(1 << 16) + 1, ldm=1 << 20), dict(ldm=1 << 24),
               dict(window=-1), dict(sinks=-1), dict(window=1 << 30), dict(sinks=1 << 30)):
        assert mask(L, **kw) == sq.SQ_ERR_SHAPE, kw
    for n in ("parents", "cu", "mask", "depth", "lens"):
        assert mask(L, **{n: fake(7, 2)}) == sq.SQ_ERR_ALIGN
    for kw in (dict(mask=fake(0)), dict(depth=fake(1)), dict(depth=fake(3, 4 * (8 * 4 + 1))), dict(mask=fake(2), window=1, sinks=1)):
        assert mask(L, **kw) == sq.SQ_ERR_ALIAS, kw
    for kw in (dict(T=0), dict(B=0), dict(T=0, lens=None), dict(T=0, lens=None, window=5)):
        assert mask(L, **kw) == sq.SQ_OK, kw


def test_tree_mask_refuses_more_words_than_it_writes(L):  # noqa: F811
    assert mask(L, T=0, words=1 << 9, ldm=1 << 9) == sq.SQ_OK
    assert mask(L, T=0, words=(1 << 9) + 1, ldm=1 << 10) == sq.SQ_ERR_SHAPE


def test_write_refusals(L):  # noqa: F811
    assert write_ex(L, depth=fake(13, 2)) == sq.SQ_ERR_ALIGN
    assert write_ex(L, qr=fake(13)) == write_ex(L, kr=fake(13)) == sq.SQ_ERR_ALIAS
    assert write_ex(L, freq=None) == sq.SQ_ERR_NULL
    assert write_ex(L, T=0) == write_ex(L, T=0, depth=None) == sq.SQ_OK


def test_tree_attention_refusals(L):  # noqa: F811
    for n in ("q", "out", "cu"):
        assert tree(L, **{n: None}) == sq.SQ_ERR_NULL
    for kw in (dict(Hq=9), dict(T=1 << 21), dict(T=-1), dict(max_len=0), dict(max_len=1 << 30), dict(ldq=1000), dict(ldo=1 << 24),
               dict(scale=float("inf")), dict(scale=float("nan")), dict(words=0), dict(words=3), dict(ldm=1 << 24), dict(window=-1),
               dict(sinks=1 << 30), dict(mask=None), dict(T=(1 << 21) - 3)):
        assert tree(L, **kw) == sq.SQ_ERR_SHAPE, kw
    for kw in (dict(q=fake(0, 8)), dict(out=fake(10, 8)), dict(ws=fake(11, 8)), dict(ldo=1028), dict(cu=fake(1, 2)), dict(mask=fake(2, 2)),
               dict(depth=fake(3, 1))):
        assert tree(L, **kw) == sq.SQ_ERR_ALIGN, kw
    for kw in (dict(out=fake(0)), dict(ws=fake(7)), dict(ws=fake(10, 16)), dict(out=fake(4)), dict(out=fake(1)), dict(ws=fake(2)), dict(out=fake(3))):
        assert tree(L, **kw) == sq.SQ_ERR_ALIAS, kw
    for kw in (dict(B=0), dict(T=0), dict(T=0, mask=None, depth=None, words=0, ldm=0)):
        assert tree(L, **kw) == sq.SQ_OK, kw
    n = ctypes.c_uint64(3)
    assert L.sq_attn_tree_workspace(1, 4, 64, 0, 0, 8, 2, 128, None) == sq.SQ_ERR_NULL
    for a in ((1, 4, 0, 0, 0, 8, 2, 128), (1, 4, 64, -1, 0, 8, 2, 128), (1, 4, 64, 0, 0, 8, 3, 128), (1, 1 << 21, 64, 0, 0, 8, 2, 128)):
        assert L.sq_attn_tree_workspace(*a, ctypes.byref(n)) == sq.SQ_ERR_SHAPE
    assert L.sq_attn_tree_workspace(1, 4, 64, 0, 0, 8, 2, 64, ctypes.byref(n)) == sq.SQ_ERR_UNSUPPORTED
    assert n.value == 3


def test_window_refusals(L):  # noqa: F811
    for call in (paged, prompt):
        for kw in (dict(window=-1), dict(sinks=-1), dict(window=1 << 30), dict(sinks=1 << 30), dict(Hq=9), dict(scale=float("nan"))):
            assert call(L, **kw) == sq.SQ_ERR_SHAPE, (call, kw)
        assert call(L, q=None) == call(L, out=None) == sq.SQ_ERR_NULL
        assert call(L, out=fake(0)) == sq.SQ_ERR_ALIAS
        assert call(L, q=fake(0, 8)) == sq.SQ_ERR_ALIGN
        assert call(L, B=0) == sq.SQ_OK
    assert paged(L, B=1 << 20) == sq.SQ_ERR_SHAPE and prompt(L, Tq=0) == sq.SQ_OK
    n = ctypes.c_uint64(3)
    assert L.sq_attn_paged_window_workspace(1, 64, 16, 2, 8, 2, 128, None) == sq.SQ_ERR_NULL
    assert L.sq_attn_paged_window_workspace(1, 64, -16, 2, 8, 2, 128, ctypes.byref(n)) == sq.SQ_ERR_SHAPE
    assert L.sq_attn_prompt_window_workspace(1, 4, 4, 16, 2, 8, 2, 128, None) == sq.SQ_ERR_NULL
    assert L.sq_attn_prompt_window_workspace(1, 4, 4, 16, -2, 8, 2, 128, ctypes.byref(n)) == sq.SQ_ERR_SHAPE
    assert n.value == 3


def test_table_refusals(L):  # noqa: F811
    for call, names in ((release, ("first", "end")), (grow, ("have", "add", "lens", "cu", "pos", "slots", "missing"))):
        for n in names + ("held", "table", "pool", "count"):
            assert call(L, **{n: None}) == sq.SQ_ERR_NULL, n
            assert call(L, **{n: fake(20, 2)}) == sq.SQ_ERR_ALIGN, n
        for kw in (dict(B=-1), dict(B=(1 << 20) + 1), dict(page=24), dict(page=8), dict(page=1 << 21), dict(pages=0), dict(pages=1 << 31),
                   dict(cols=0), dict(cols=9), dict(cols=1 << 24, ldt=1 << 24), dict(ldt=1 << 41)):
            assert call(L, **kw) == sq.SQ_ERR_SHAPE, kw
        for kw in (dict(held=fake(3)), dict(pool=fake(3, 4 * 23)), dict(count=fake(4, 4 * 15)), dict(table=fake(0)), dict(held=fake(1))):
            assert call(L, **kw) == sq.SQ_ERR_ALIAS, kw
    assert release(L, B=0) == sq.SQ_OK
    assert grow(L, T=-1) == grow(L, T=1 << 31) == sq.SQ_ERR_SHAPE
    assert grow(L, slots=fake(9, 4)) == sq.SQ_ERR_ALIGN
    for kw in (dict(lens=fake(0)), dict(cu=fake(6, 8)), dict(pos=fake(9, 64)), dict(missing=fake(5)), dict(lens=fake(2))):
        assert grow(L, **kw) == sq.SQ_ERR_ALIAS, kw


def test_keep_refusals(L):  # noqa: F811
    for n in ("cu", "path", "kept", "out"):
        assert keep(L, **{n: None}) == sq.SQ_ERR_NULL
        assert keep(L, **{n: fake(20, 2)}) == sq.SQ_ERR_ALIGN
    for kw in (dict(most=0), dict(most=9), dict(ldp=1 << 24)):
        assert keep(L, **kw) == sq.SQ_ERR_SHAPE, kw
    for kw in (dict(out=fake(8)), dict(out=fake(0, 12)), dict(path=fake(5)), dict(out=fake(7)), dict(kq=fake(6))):
        assert keep(L, **kw) == sq.SQ_ERR_ALIAS, kw
    assert keep(L, B=0) == sq.SQ_OK


@pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="a GPU driver is present: the calls below would "
                    "launch kernels on fake pointers")
def test_no_device_is_a_hip_error(L):  # noqa: F811
    for call in (mask, write_ex, tree, paged, prompt, release, grow, keep):
        assert call(L) == sq.SQ_ERR_HIP, call


def test_binding_refuses():
    """Host tensors, wrong types and shapes."""
    x = torch.zeros((2, 4, 128), dtype=torch.float16)
    i = torch.ones(2, dtype=torch.int32)
    cache = sq.kv_cache(1, 16, 4, device="cpu")
    for call in (lambda: sq.tree_mask(i, i, 4), lambda: sq.attn_tree(x, cache, i[:, None], i, i, 16),
                 lambda: sq.paged_release(i[:, None], 16, i, i, i, i, i[:1]), lambda: sq.paged_grow(i, i, i, i[:, None], 16, i, i[:1], 2),
                 lambda: sq.kv_keep(cache, i[:, None], i, i, i[:, None], i), lambda: sq.attn_paged(x, cache, i[:, None], i, 16, window=4),
                 lambda: sq.attn_prompt(x, x, x, i, i, window=4)):
        with pytest.raises(TypeError):
            call()


def test_every_call_has_its_argument_types():
    """As many types in the binding as arguments in the header."""
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "sq.h")).read()
    for name in ("sq_tree_mask", "sq_rope_kv_write_ex", "sq_attn_tree", "sq_attn_tree_workspace", "sq_attn_paged_window",
                 "sq_attn_paged_window_workspace", "sq_attn_prompt_window", "sq_attn_prompt_window_workspace", "sq_paged_release",
                 "sq_paged_grow", "sq_kv_keep"):
        at = text.index("sq_status %s(" % name)
        args = text[at:text.index(";", at)].split("(", 1)[1].rsplit(")", 1)[0].split(",")
        kinds = [ctypes.c_void_p if "*" in a else {"int64_t": ctypes.c_int64, "int32_t": ctypes.c_int32, "float": ctypes.c_float,
                                                  "uint64_t": ctypes.c_uint64}[a.split()[0]] for a in args]
        assert getattr(sq.lib(), name).argtypes == kinds, name
