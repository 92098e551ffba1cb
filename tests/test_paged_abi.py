"""Refusals of the paged cache's entry points: on the host, before anything is launched (no GPU needed)."""
import ctypes

import pytest
import torch

FAKE = 0x100000  # aligned, never dereferenced: validation fails first


@pytest.fixture(scope="module")
def b():
    import paper_2604_17397_amd.binding as binding
    binding.lib()
    return binding


def plan_args(b, **kw):
    at = iter(range(FAKE, FAKE + (1 << 20), 1 << 14))
    names = ("cached", "new_tokens", "free_pages", "held", "next_free", "block_table", "q_start", "kv_lens", "positions",
             "held_out", "next_free_out", "slots")
    a = b.sdvg_page_plan_args(n_requests=4, page_tokens=16, table_width=8, n_free=10, table_stride=8, max_tokens=40,
                              **{n: next(at) for n in names})
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("kw,expect", [
    (dict(n_requests=-1), -2), (dict(max_tokens=-1), -2), (dict(page_tokens=0), -2), (dict(table_width=0), -2),
    (dict(n_free=-1), -2), (dict(table_stride=7), -2), (dict(max_tokens=1 << 31), -5), (dict(page_tokens=12), -4),
    (dict(cached=None), -1), (dict(new_tokens=None), -1), (dict(block_table=None), -1), (dict(q_start=None), -1),
    (dict(kv_lens=None), -1), (dict(positions=None), -1), (dict(slots=None), -1), (dict(held_out=None), -1),
    (dict(next_free_out=None), -1), (dict(free_pages=None), -1), (dict(slots=FAKE + (1 << 19) + 4), -4), (dict(cached=FAKE + 2), -4),
    (dict(held_out=FAKE + 3 * (1 << 14)), -3),          # held in place
    (dict(kv_lens=FAKE), -3),                           # cached in place
    (dict(next_free_out=FAKE + 4 * (1 << 14)), -3),
    (dict(positions=FAKE + 11 * (1 << 14) + 8), -3),    # positions inside slots
    (dict(block_table=FAKE + 8), -3),
])
def test_page_plan_rejects_bad_arguments(b, kw, expect):
    assert b.lib().sdvg_page_plan(ctypes.byref(plan_args(b, **kw)), None) == expect
    assert b.lib().sdvg_page_plan(None, None) == -1


def test_page_plan_binding_checks(b, monkeypatch):
    monkeypatch.setattr(b, "_check_here", lambda *a: None)
    monkeypatch.setattr(b, "_LIB", type("Trap", (), {"__getattr__": lambda s, n: pytest.fail("the C library must not be reached")})())
    n = torch.zeros(3, dtype=torch.int32)
    table = torch.zeros((3, 5), dtype=torch.int32)
    plan = b.PagePlan(3, 7, device="cpu")
    bad = [dict(new_tokens=n[:2]), dict(cached=n.long()), dict(block_table=table.long()), dict(block_table=table[:2]),
           dict(block_table=table.t().contiguous().t()), dict(held=n[:1]), dict(free_pages=n), dict(next_free=n[:1]),
           dict(held=n, free_pages=n.float()), dict(held=n, next_free=n), dict(out=None), dict(max_tokens=3),
           dict(out=b.PagePlan(2, 7, device="cpu"))]
    for kw in bad:
        a = dict(cached=n, new_tokens=n, block_table=table, page_tokens=16, out=plan)
        a.update(kw)
        with pytest.raises(ValueError):
            b.page_plan(**a)
    with pytest.raises(ValueError):
        b.PagePlan(-1, 4, device="cpu")
