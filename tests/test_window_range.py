"""Windows and first tokens beyond 32 bits are refused by the binding, not cut down to what is left of them."""

import pytest
import torch

from paper_2405_16406_amd import sq

BEYOND = [(2 ** 32 + 8, 2), (8, 2 ** 32 + 2), (2 ** 31, 0), (2 ** 32, 0), (-2 ** 32 + 8, 2), (8, -2 ** 32), (2 ** 63, 2), (1 << 30, 0), (-1, 0), (8, -1)]


@pytest.mark.parametrize("window,sinks", BEYOND)
def test_workspaces(window, sinks):
    for call in (lambda: sq.attn_paged_workspace_bytes(4, 1000, 8, 2, window, sinks),
                 lambda: sq.attn_tree_workspace_bytes(1, 4, 1000, 8, 2, window, sinks),
                 lambda: sq.attn_prompt_workspace_bytes(1, 4, 1000, 8, 2, window, sinks)):
        with pytest.raises(sq.SqError) as e:
            call()
        assert e.value.status == sq.SQ_ERR_SHAPE and str(window) in str(e.value)


@pytest.mark.gpu
@pytest.mark.parametrize("window,sinks", BEYOND)
def test_calls(window, sinks):
    ints = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda:0")  # noqa: E731
    q = torch.zeros((4, 8, 128), dtype=torch.float16, device="cuda:0")
    cache, table, lens, cu = sq.kv_cache(2, 16, 2, device="cuda:0"), ints(0, 1)[None], ints(20), ints(0, 4)
    space = torch.empty(1 << 20, dtype=torch.uint8, device="cuda:0")
    args = dict(window=window, sinks=sinks)
    for call in (lambda: sq.tree_mask(ints(-1, 0, 1, 2), cu, 4, lens, **args),
                 lambda: sq.attn_tree(q, cache, table, lens, cu, 20, workspace=space, **args),
                 lambda: sq.attn_paged(q[:1], cache, table, lens, 20, workspace=space, **args),
                 lambda: sq.attn_prompt(q, q[:, :2], q[:, :2], cu, cu, workspace=space, **args)):
        with pytest.raises(sq.SqError) as e:
            call()
        assert e.value.status == sq.SQ_ERR_SHAPE
