"""The attention's workspace: none where no request can be split, ignored when too small, never left."""
import pytest
import torch

from test_gpu_paged_attn import Case

pytestmark = pytest.mark.gpu


def attn(c, ws):
    import paper_2604_17397_amd as P
    out = P.paged_attn(c.q, c.handle(), c.table, c.q_start, c.kv_lens, workspace=ws)
    torch.cuda.synchronize()
    return out


def need(c):
    import paper_2604_17397_amd as P
    return P.paged_attn_workspace_bytes(c.q, c.handle(), c.table)


@pytest.mark.parametrize("heads,kv_heads", [(4, 4), (40, 2), (5, 1)])
@pytest.mark.parametrize("lengths", [[(256, 1)], [(1, 1), (250, 8), (256, 3)]])
def test_none_for_requests_that_are_not_split(heads, kv_heads, lengths):
    c = Case(lengths, heads, kv_heads, 16)
    c.table = c.table[:, :16].contiguous()      # 256 keys
    assert need(c) == 0
    c.check()
    wider = Case(lengths, heads, kv_heads, 16)
    assert wider.table.shape[1] == 17 and need(wider) > 0
    assert torch.equal(attn(c, None), attn(wider, torch.empty(need(wider), dtype=torch.uint8, device="cuda")))


@pytest.mark.parametrize("heads,kv_heads,cache", [(10, 2, None), (40, 8, "e4m3"), (3, 3, None)])
@pytest.mark.parametrize("lengths", [[(9000, 1), (400, 1)], [(2000, 8)] * 5])
def test_too_small_and_exact(heads, kv_heads, cache, lengths):
    c = Case(lengths, heads, kv_heads, 16, cache=cache)
    n = need(c)
    whole = attn(c, None)
    small = torch.full((n - 16,), 201, dtype=torch.uint8, device="cuda")
    assert torch.equal(attn(c, small), whole) and (small == 201).all()
    for at in (0, 16):
        guarded = torch.full((n + 4096,), 201, dtype=torch.uint8, device="cuda")
        split = attn(c, guarded[at:at + n])
        assert (guarded[:at] == 201).all() and (guarded[at + n:] == 201).all() and (guarded != 201).any()
        assert torch.equal(split, attn(c, torch.empty(n + 64, dtype=torch.uint8, device="cuda")))
