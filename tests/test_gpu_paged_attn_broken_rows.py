"""A query row that is not finite has no result: NaN in out and in lse, which says -infinity of rows without a key only."""
import math

import pytest
import torch

from paged_util import i32
from test_gpu_paged_attn import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,cache", [("bf16", None), ("f16", None), ("bf16", "e4m3")])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("workspace", [False, True])
@pytest.mark.parametrize("heads,kv_heads", [(10, 2), (3, 3), (24, 1)])
def test_rows_that_are_not_finite(kind, cache, bad, workspace, heads, kv_heads):
    import paper_2604_17397_amd as P
    # (the last request has two more new tokens than keys: those rows see nothing)
    c = Case([(700, 3), (65, 4), (3001, 8), (2, 2)], heads, kv_heads, 16, kind, cache)
    c.requests[3] = (2, 4)
    c.q_start = i32([0, 3, 7, 15, 19])
    c.q = torch.randn((19, heads, 128), device="cuda").to(c.q.dtype)
    broken = [1, 8, 18]
    c.q[broken] = bad
    ws = torch.empty(P.paged_attn_workspace_bytes(c.q, c.handle(), c.table), dtype=torch.uint8, device="cuda") if workspace else None
    lse = torch.full(c.q.shape[:2], 3.0, device="cuda")
    out = P.paged_attn(c.q, c.handle(), c.table, c.q_start, c.kv_lens, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    for t in range(19):
        if t in broken:
            assert torch.isnan(out[t]).all() and torch.isnan(lse[t]).all(), t
        elif t in (15, 16):
            assert (out[t] == 0).all() and (lse[t] == -math.inf).all(), t
        else:
            assert torch.isfinite(out[t]).all() and torch.isfinite(lse[t]).all(), t
