"""Workspaces that do not lie in one piece are refused by every call that takes one."""

import pytest
import torch

from paper_2405_16406_amd import sq

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("bad", [lambda n: torch.empty(2 * n, dtype=torch.uint8, device=DEV)[::2],
                                 lambda n: torch.empty(1, dtype=torch.uint8, device=DEV).expand(n)], ids=["strided", "expanded"])
def test_workspaces_are_contiguous(bad):
    q = torch.zeros((1, 8, 128), dtype=torch.float16, device=DEV)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    cache = sq.kv_cache(256, 16, 2)
    table = torch.arange(256, dtype=torch.int32, device=DEV)[None]
    kv = torch.zeros((9000, 2, 128), dtype=torch.float16, device=DEV)
    codes = torch.zeros((1, 4096, 8, 64), dtype=torch.uint8, device=DEV)
    ab = torch.ones((1, 4096, 8, 1), dtype=torch.float32, device=DEV)
    calls = [(sq.attn_paged_workspace_bytes(1, 4096, 8, 2), lambda w: sq.attn_paged(q, cache, table, ints([4096]), 4096, workspace=w)),
             (sq.attn_prompt_workspace_bytes(1, 1, 9000, 8, 2), lambda w: sq.attn_prompt(q, kv, kv, ints([0, 1]), ints([0, 9000]), workspace=w)),
             (sq.attn_decode_workspace_bytes(1, 4096, 8), lambda w: sq.attn_decode_kv4_split(q, codes, ab, ab, codes, ab, ab, workspace=w))]
    for n, call in calls:
        assert n > 0
        with pytest.raises(ValueError):
            call(bad(n))
