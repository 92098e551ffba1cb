"""What out-of-range numbers in q_start and kv_lens mean to sdvg_paged_prefix_attn: they are clamped, as sdvg_paged_attn has it, for the shared
keys as for the requests' own ones. Out and lse are those of the clamped numbers in 64 bits, with and without a workspace, and nothing
beside the rows that they name and the workspace is written. Bounds as in test_gpu_paged_prefix."""
import pytest
import torch

from paged_util import i32
from test_gpu_paged_attn import HALF_STEP
from test_gpu_paged_prefix import GROUPS, Shared

pytestmark = pytest.mark.gpu
BIG = 2**31 - 1
LENS = [1008, 720]           # whole pages of 16, the first 700 keys shared


def case(cache=None):
    return Shared([(700, [(308, 1), (20, 1)])], 4, 2, 16, cache=cache)


@pytest.mark.parametrize("starts,lens,means", [
    ([0, 1, 2], LENS, [(1008, 1), (720, 1)]),
    ([-3, 1, 900], LENS, [(1008, 1), (720, 1)]),
    ([-2**31, 1, BIG], LENS, [(1008, 1), (720, 1)]),
    ([-2**31, 1, 3], LENS, [(1008, 1), (720, 1)]),
    ([0, 1, 2], [BIG, BIG], [(1008, 1), (720, 1)]),            # keys without a page are not there
    ([0, 2, 1], [-5, 720], [(0, 2), (720, 0)]),                # an end ahead of its start: no token
    ([-9, 2, 2], LENS, [(1008, 2), (720, 0)]),
    ([0, 0, 70], LENS, [(1008, 0), (720, 2)]),
    ([0, 1, 2], [-2**31, 701], [(0, 1), (701, 1)]),
    ([0, 2, 2], [-2**31, 720], [(0, 2), (720, 0)]),            # a length and a number of rows whose difference leaves 32 bits
    ([0, 0, BIG], [3, -2**31], [(3, 0), (0, 2)]),
    ([0, 1, 2], [1008, 0], [(1008, 1), (0, 1)]),
    ([5, 6, 7], LENS, None),                                   # every token past the last row: nothing is written
    ([BIG, -5, 0], LENS, None),
])
@pytest.mark.parametrize("window", [0, 50, 500])
@pytest.mark.parametrize("workspace", [False, True])
@pytest.mark.parametrize("groups", ["one", "two", "none named"])
@pytest.mark.parametrize("cache", [None, "e4m3"])
def test_clamped(starts, lens, means, window, workspace, groups, cache):
    import paper_2604_17397_amd as P
    if window and lens == [BIG, BIG]:
        means = [(0, 1), (0, 1)]                               # a window past all pages: no key
    c = case(cache)
    c.group_start, c.prefix_lens = (i32([0, 1, 2]), i32([700, 700])) if groups == "two" else (i32([0, 2]), i32([700]))
    rows = torch.full((6, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    all_lse = torch.full((6, 4), 7.0, device="cuda")
    n = c.need(len(c.prefix_lens))
    ws = torch.full((n + 8192,), 201, dtype=torch.uint8, device="cuda")
    P.paged_prefix_attn(c.q, c.handle(), c.table, i32(starts), i32(lens), c.prefix_lens, group_start=None if groups == "none named" else c.group_start,
                        out=rows[2:4], lse=all_lse[2:4], window=window, workspace=ws[4096:4096 + n] if workspace else None)
    torch.cuda.synchronize()
    assert (rows[:2] == 7).all() and (rows[4:] == 7).all() and (all_lse[:2] == 7).all() and (all_lse[4:] == 7).all()
    assert (ws[:4096] == 201).all() and (ws[4096 + n:] == 201).all()
    if means is None:
        assert (rows == 7).all() and (all_lse == 7).all()
        return
    c.requests = means
    want, size, lse = c.want(window)
    h = HALF_STEP["bf16"]
    excess = (rows[2:4].double() - want).abs() - ((h + 2.0**-12) * size + h * want.abs())
    assert not torch.isnan(excess).any() and excess.max().item() <= 0, excess.max().item()
    empty = torch.isinf(lse)
    assert torch.equal(torch.isinf(all_lse[2:4]), empty) and (rows[2:4][empty] == 0).all()
    assert ((all_lse[2:4].double() - lse).abs()[~empty] <= 2.0**-12).all()


@pytest.mark.parametrize("window", [0, 300])
@pytest.mark.parametrize("groups", ["many rows", "groups", "many groups"])
def test_ends_of_many_requests(groups, window):
    """The first start below 0 and the last end past the rows: the same bits as with the clamped ones."""
    c = Shared(GROUPS[groups], 6, 2, 16)
    c.n_tokens = c.q.shape[0]
    lse = [torch.empty(c.q.shape[:2], device="cuda") for _ in range(2)]
    want = c.run(window=window, lse=lse[0])
    c.q_start = c.q_start.clone()
    c.q_start[c.q_start == 0] = -2**31
    c.q_start[c.q_start == c.n_tokens] = BIG
    got = c.run(window=window, lse=lse[1])
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(lse[0], lse[1])
