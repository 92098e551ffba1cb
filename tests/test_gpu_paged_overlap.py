"""Rows right beside the pools, in one allocation with them, are none of theirs: taken, and nothing else is written."""
import pytest
import torch

from paged_util import i32

pytestmark = pytest.mark.gpu


def test_commit_of_rows_right_beside_the_pools():
    import paper_2604_17397_amd as P
    n, pool = 4 * 2 * 128, 4 * 8 * 2 * 128
    torch.manual_seed(2)
    # q | k pool | k rows | v pool | q_out
    one = torch.randn(3 * n + 2 * pool, device="cuda").bfloat16()
    q, kp, k, vp, q_out = one.split([n, pool, n, pool, n])
    q, k, q_out = (t.view(4, 2, 128) for t in (q, k, q_out))
    kp, vp = (t.view(4, 8, 2, 128) for t in (kp, vp))
    freqs, _ = P.rope_frequencies(64)
    pos, slots = i32([3, 9, 0, 70]), torch.tensor([5, 31, 0, 12], device="cuda")
    want = one.clone()
    turned = [P.rope_positions(t, pos, freqs) for t in (q, k)]
    assert P.paged_commit(P.PagedKV(kp, vp), k, k, slots, positions=pos, freqs=freqs, q=q, q_out=q_out) is q_out
    torch.cuda.synchronize()
    _, wk, _, wv, wq = want.split([n, pool, n, pool, n])
    wk.view(32, 2, 128)[slots], wv.view(32, 2, 128)[slots] = turned[1], k
    wq.copy_(turned[0].flatten())
    assert torch.equal(one, want)
