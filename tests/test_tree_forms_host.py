"""Which forms of the attention of several rows the sizes of the GPU tests reach (csrc/paged_plan.h compiled alone, no GPU)."""

import ctypes

import numpy as np
import pytest

from test_drafts_host import I64, host, plan_of  # noqa: F401


def forms(host, cases, window=None):  # noqa: F811
    out = {}
    for name, (hq, h, dt, new, past, *w) in cases.items():
        args = (len(new), sum(new), max(n + p for n, p in zip(new, past)), *(w or [0]), 2 if w else 0, hq, h)
        rb, _, chunks, _ = plan_of(host, *args)
        out[name] = (rb, host.tree_waves(I64(args[0]), I64(args[1]), 0, I64(args[2]), *args[3:], 256), chunks > 1)
    return out


def test_hidden_parameters_reach_every_form(host):  # noqa: F811
    t = pytest.importorskip("test_gpu_tree_hidden")
    assert forms(host, t.FORMS) == {"one column": (1, 4, False), "eight waves": (1, 8, False), "two columns": (2, 4, True),
                                    "two columns, joined": (2, 4, True), "one column, joined": (1, 4, True)}


def test_queries_of_different_sizes_reach_every_form(host):  # noqa: F811
    t = pytest.importorskip("test_gpu_tree_queries")
    got = forms(host, t.FORMS)
    assert got == {"one": (1, 4, False), "eight": (1, 8, False), "two": (2, 4, True), "two, fp16": (2, 4, True), "joined": (1, 4, True)}
    assert {c[2] for n, c in t.FORMS.items() if n.startswith("two")} == {np.float16, np.float32}
