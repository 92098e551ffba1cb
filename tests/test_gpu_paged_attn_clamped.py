"""What the numbers in q_start and kv_lens mean when they are out of range: they are clamped, and nothing but the rows they
then name is written. With and without a split, whose workspace is not left either."""
import math

import pytest
import torch

from paged_util import i32
from test_gpu_paged_attn import HALF_STEP, Case

pytestmark = pytest.mark.gpu
BIG = 2**31 - 1


def requests(*sizes):
    """(out, size, lse) of the two tokens for requests of the given (length, new tokens), by the definition."""
    c = Case([(4800, 1), (80, 1)], 2, 1, 16)
    c.requests = list(sizes)
    return c.want()


@pytest.mark.parametrize("starts,lens,means", [
    ([0, 1, 2], [4800, 80], [(4800, 1), (80, 1)]),
    ([-3, 1, 900], [4800, 80], [(4800, 1), (80, 1)]),
    ([-2**31, 1, BIG], [4800, 80], [(4800, 1), (80, 1)]),
    ([0, 1, 2], [BIG, BIG], [(4800, 1), (80, 1)]),              # keys without a page are not there
    ([0, 2, 1], [-5, 80], [(0, 2), (80, 0)]),                   # an end ahead of its start: no token
    ([0, 2, 2], [4800, 80], [(4800, 2), (80, 0)]),
    ([0, 0, 2], [4800, 80], [(4800, 0), (80, 2)]),
    ([0, 1, 2], [-2**31, 1], [(0, 1), (1, 1)]),
    ([0, 1, 2], [4800, 0], [(4800, 1), (0, 1)]),
    ([5, 6, 7], [4800, 80], None),                              # every token past the last row: nothing is written
    ([BIG, -5, 0], [4800, 80], None),
])
@pytest.mark.parametrize("split", [False, True])
def test_clamped(starts, lens, means, split):
    import paper_2604_17397_amd as P
    c = Case([(4800, 1), (80, 1)], 2, 1, 16)
    rows = torch.full((6, 2, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    all_lse = torch.full((6, 2), 7.0, device="cuda")
    n = P.paged_attn_workspace_bytes(c.q, c.handle(), c.table)
    ws = torch.full((n + 8192,), 201, dtype=torch.uint8, device="cuda")
    P.paged_attn(c.q, c.handle(), c.table, i32(starts), i32(lens), out=rows[2:4], lse=all_lse[2:4], workspace=ws[4096:4096 + n] if split else None)
    torch.cuda.synchronize()
    assert (rows[:2] == 7).all() and (rows[4:] == 7).all() and (all_lse[:2] == 7).all() and (all_lse[4:] == 7).all()
    assert (ws[:4096] == 201).all() and (ws[4096 + n:] == 201).all()
    if means is None:
        assert (rows == 7).all() and (all_lse == 7).all()
        return
    want, size, lse = requests(*means)
    h = HALF_STEP["bf16"]
    excess = (rows[2:4].double() - want).abs() - ((h + 2.0**-12) * size + h * want.abs())
    assert not torch.isnan(excess).any() and excess.max().item() <= 0
    empty = torch.isinf(lse)
    assert torch.equal(torch.isinf(all_lse[2:4]), empty) and (rows[2:4][empty] == 0).all()
    assert ((all_lse[2:4].double() - lse).abs()[~empty] <= 2.0**-12).all()


@pytest.mark.parametrize("split", [False, True])
def test_a_window_past_the_table(split):
    """A length far beyond its table whose window holds no key that has a page: a row without any key."""
    import paper_2604_17397_amd as P
    c = Case([(4800, 1), (80, 1)], 2, 1, 16)
    ws = torch.empty(P.paged_attn_workspace_bytes(c.q, c.handle(), c.table), dtype=torch.uint8, device="cuda") if split else None
    lse = torch.zeros((2, 2), device="cuda")
    out = P.paged_attn(c.q, c.handle(), c.table, c.q_start, i32([BIG, 80]), lse=lse, window=100, workspace=ws)
    torch.cuda.synchronize()
    assert (out[0] == 0).all() and (lse[0] == -math.inf).all() and (out[1] != 0).any() and torch.isfinite(lse[1]).all()
