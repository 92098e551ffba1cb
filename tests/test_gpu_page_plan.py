"""sdvg_page_plan against plain Python integers: pages, slots, positions and row ranges from lengths."""
import numpy as np
import pytest
import torch

from paged_util import i32, plan_oracle

pytestmark = pytest.mark.gpu


def check(cached, new, table, P, max_tokens, held=None, free=None, next_free=None, table_pad=0):
    import paper_2604_17397_amd as S
    R, W = table.shape
    want = plan_oracle(cached, new, table, P, max_tokens, held, () if free is None else free, next_free or 0)
    wide = torch.full((R, W + table_pad), 777, dtype=torch.int32, device="cuda")
    wide[:, :W] = i32(table)
    d_table = wide[:, :W]
    plan = S.PagePlan(R, max_tokens)
    for t in (plan.q_start, plan.kv_lens, plan.positions, plan.slots):
        t.fill_(-99)
    kw = {} if held is None else dict(held=i32(held), free_pages=None if free is None else i32(free),
                                      next_free=None if next_free is None else i32([next_free]))
    for _ in range(2):   # the same call again gives the same answer
        got = S.page_plan(i32(cached), i32(new), d_table, P, out=plan, **kw)
        torch.cuda.synchronize()
        assert got is plan
        assert np.array_equal(d_table.cpu().numpy(), want["table"])
        assert (wide[:, W:] == 777).all()
        for name in ("q_start", "kv_lens", "positions", "slots"):
            assert np.array_equal(getattr(plan, name).cpu().numpy(), want[name]), name
        if held is not None:
            assert np.array_equal(plan.held.cpu().numpy(), want["held"])
            assert plan.next_free.item() == want["next_free"]
    return want


@pytest.mark.parametrize("R,longest,new,P", [(1, 1, 1, 8), (1, 5000, 1, 16), (7, 90, 8, 24), (64, 300, 1, 64),
                                             (200, 4000, 9, 16), (3, 40, 5000, 256), (1024, 60, 3, 8), (1025, 60, 3, 16)])
def test_lengths_to_pages(R, longest, new, P):
    rng = np.random.default_rng(R * 7 + P)
    cached, fresh = rng.integers(0, longest + 1, R), rng.integers(0, new + 1, R)
    held = -(-cached // P) + rng.integers(0, 2, R)      # some hold a page more than they need, as after a rejected draft
    W = int((-(-(cached + fresh) // P)).max()) + 2
    ids = rng.permutation(int(held.sum()) + R * (W + 1))
    table = np.full((R, W), -1)
    for r in range(R):
        table[r, :held[r]] = ids[held[:r].sum():held[:r + 1].sum()]
    check(cached, fresh, table, P, int(fresh.sum()) + 3, held, ids[held.sum() - 2 if held.sum() > 2 else 0:], 2 if held.sum() > 2 else 0,
          table_pad=R % 3)


def test_no_request_and_no_token():
    import paper_2604_17397_amd as S
    plan = S.PagePlan(0, 4)
    plan.slots.fill_(9)
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    S.page_plan(none, none, torch.empty((0, 3), dtype=torch.int32, device="cuda"), 16, held=none, free_pages=i32([4, 5]),
                next_free=i32([1]), out=plan)
    torch.cuda.synchronize()
    assert plan.q_start.tolist() == [0] and plan.slots.tolist() == [-1] * 4 and plan.next_free.item() == 1
    check(np.array([5, 9]), np.array([0, 0]), np.array([[3, -1], [1, 2]]), 8, 0, np.array([1, 2]), np.array([7]))
    check(np.array([0]), np.array([0]), np.array([[-1]]), 8, 2)


def test_pages_run_out():
    table = np.full((4, 4), -1)
    want = check([0, 0, 0, 0], [10, 20, 9, 1], table, 8, 50, [0, 0, 0, 0], [5, 9, 2, 7], 0)
    assert want["next_free"] == 8 and want["held"].tolist() == [2, 2, 0, 0]     # 4 pages short
    check([0, 0], [10, 10], table[:2], 8, 20, [0, 0], None, None)               # none at all
    check([0, 0], [10, 10], table[:2], 8, 20, [0, 0], [1, 2, 3], 7)             # the cursor stands past the list


def test_narrow_table_missing_pages_and_negative_lengths():
    check([14, 30], [6, 2], np.array([[4, 6], [1, 2]]), 8, 9, [2, 2], [8, 9], 0)       # tokens past the table
    check([3, 8, -5], [6, 1, 3], np.array([[-1, 6], [3, -1], [2, 2]]), 8, 12)          # a page that is missing
    check([-7, 4], [-2, 3], np.array([[1], [2]]), 8, 4, [-3, 1], [5], 0)
    check([2**31 - 3], [2], np.array([[1]]), 8, 2)                                      # far past the table
    want = check([9, 4], [9, 6], np.array([[3, 8, -1], [4, -1, -1]]), 8, 15, [9, 1], [5, 6], None)   # more held than the table has
    assert want["held"].tolist() == [9, 2]


def test_tokens_past_the_room_have_no_row():
    want = check([4, 4, 4], [5, 5, 5], np.full((3, 2), -1), 8, 7, [0, 0, 0], np.arange(10), 1)
    assert want["q_start"].tolist() == [0, 5, 7, 7] and want["kv_lens"].tolist() == [9, 6, 4]


def test_steps_in_a_graph_take_pages_one_after_the_other():
    """A captured step whose results become the next step's state: every replay goes on where the last one ended."""
    import paper_2604_17397_amd as S
    P, R = 8, 3
    state = dict(cached=np.array([6, 0, 15]), held=np.array([1, 0, 2]), next_free=0)
    table0 = np.full((R, 6), -1)
    table0[0, 0], table0[2, :2] = 40, (41, 42)
    free = np.arange(20, 30)
    new = np.array([3, 1, 2])
    cached, held, cursor, table = i32(state["cached"]), i32(state["held"]), i32([0]), i32(table0)
    d_new, d_free = i32(new), i32(free)
    plan = S.PagePlan(R, 6)

    def step():
        S.page_plan(cached, d_new, table, P, free_pages=d_free, held=held, next_free=cursor, out=plan)
        cached.copy_(plan.kv_lens)
        held.copy_(plan.held)
        cursor.copy_(plan.next_free)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    want_table = table0
    with torch.cuda.stream(side):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step()
        for rep in range(4):
            g.replay()
            torch.cuda.synchronize()
            w = plan_oracle(state["cached"], new, want_table, P, 6, state["held"], free, state["next_free"])
            want_table = w["table"]
            state = dict(cached=w["kv_lens"], held=w["held"], next_free=w["next_free"])
            assert np.array_equal(table.cpu().numpy(), want_table), rep
            assert np.array_equal(plan.slots.cpu().numpy(), w["slots"]) and np.array_equal(plan.positions.cpu().numpy(), w["positions"])
            torch.zeros(1000, device="cuda").sum().item()       # eager work between the replays


def test_new_plan_on_another_stream_than_the_busy_current_one():
    import paper_2604_17397_amd as S
    cached, new, table = np.array([5, 31, 0]), np.array([1, 4, 17]), np.array([[3, 4, 9], [7, 1, 8], [2, 0, -1]])
    want = plan_oracle(cached, new, table, 16, 24, None, (), 0)
    args = [i32(cached), i32(new), i32(table)]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    torch.cuda._sleep(20_000_000)   # some ms of the current stream's time
    plan = S.page_plan(*args, 16, max_tokens=24, stream=s)
    torch.cuda.synchronize()
    for name in ("q_start", "kv_lens", "positions", "slots"):
        assert np.array_equal(getattr(plan, name).cpu().numpy(), want[name]), name


def test_numbers_beyond_32_bits_are_refused():
    import paper_2604_17397_amd as S
    with pytest.raises(ValueError, match="32 bits"):
        S.page_plan(i32([1]), i32([1]), i32([[0]]), 2**32 + 16, max_tokens=1)
