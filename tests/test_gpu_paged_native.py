"""The C++ marshalling of the paged cache's calls: it takes them, gives what the Python code gives, and leaves the
rest (subclasses, wrong sizes, other types) to it."""
import pytest
import torch

from paged_util import i32
from test_gpu_native_binding import both

pytestmark = pytest.mark.gpu


def pools(dtype=torch.bfloat16):
    torch.manual_seed(4)
    return [torch.randn((9, 16, 2, 128), device="cuda").to(dtype) for _ in range(2)]


def x(n, heads, dtype=torch.bfloat16, seed=0):
    torch.manual_seed(seed)
    return torch.randn((n, heads, 128), device="cuda").to(dtype)


def same(a, b):
    a, b = ([t] if torch.is_tensor(t) else list(t) for t in (a, b))
    assert len(a) == len(b) and all(torch.equal(s.view(torch.uint8), t.view(torch.uint8)) for s, t in zip(a, b))


@pytest.mark.parametrize("form", ["pages", "given pages", "stream", "new plan"])
def test_page_plan(monkeypatch, form):
    kw = dict(held=i32([1, 0]), free_pages=i32([5, 6, 7]), next_free=i32([1])) if form != "given pages" else {}
    if form == "stream":
        kw["stream"] = torch.cuda.current_stream()

    def call(P):
        table = i32([[3, 4, 2], [1, 0, 8]])
        plan = P.page_plan(i32([14, 0]), i32([4, 2]), table, 16, max_tokens=8, out=None if form == "new plan" else P.PagePlan(2, 8), **kw)
        return [table, plan.q_start, plan.kv_lens, plan.positions, plan.slots, plan.held, plan.next_free]
    got, want, taken = both(monkeypatch, call)
    same(got, want)
    assert taken == [True]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("form", ["one", "two", "out", "stream"])
def test_rope_positions(monkeypatch, dtype, form):
    def call(P):
        freqs, gain = P.rope_frequencies(64)
        kw = dict(y=x(5, 2, dtype, 1)) if form != "one" else {}
        if form == "out":
            kw.update(out=torch.empty((5, 3, 128), dtype=dtype, device="cuda"), y_out=torch.empty((5, 2, 128), dtype=dtype, device="cuda"))
        if form == "stream":
            kw["stream"] = torch.cuda.current_stream()
        r = P.rope_positions(x(5, 3, dtype), i32([1, 2, 9, 0, 4]), freqs, gain=gain, layout="interleaved", **kw)
        assert form != "out" or (r[0] is kw["out"] and r[1] is kw["y_out"])
        return r
    got, want, taken = both(monkeypatch, call)
    same(got, want)
    assert taken == [True]


@pytest.mark.parametrize("dtype,cache", [(torch.bfloat16, torch.bfloat16), (torch.float16, torch.float8_e4m3fn)])
@pytest.mark.parametrize("form", ["plain", "k", "q", "q_out"])
def test_paged_commit(monkeypatch, dtype, cache, form):
    def call(P):
        k, v = pools(cache)
        c = P.PagedKV(k, v, *[torch.full((2,), 0.02, device="cuda")] * (2 if cache == torch.float8_e4m3fn else 0))
        freqs, _ = P.rope_frequencies(128)
        kw = {} if form == "plain" else dict(positions=i32([1, 2, 9, 0, 4]), freqs=freqs)
        if form.startswith("q"):
            kw["q"] = x(5, 4, dtype, 3)
        if form == "q_out":
            kw["q_out"] = kw["q"]
        r = P.paged_commit(c, x(5, 2, dtype, 1), x(5, 2, dtype, 2), torch.tensor([3, 140, -1, 7, 90], device="cuda"), **kw)
        assert (r is None) == (not form.startswith("q")) and (form != "q_out" or r is kw["q"])
        return [k.view(torch.uint8), v.view(torch.uint8)] + ([] if r is None else [r])
    got, want, taken = both(monkeypatch, call)
    same(got, want)
    assert taken == [True]


@pytest.mark.parametrize("form", ["plain", "all", "stream", "e4m3"])
def test_paged_attn(monkeypatch, form):
    def call(P):
        c = P.PagedKV(*pools(torch.float8_e4m3fn if form == "e4m3" else torch.bfloat16))
        q, table = x(3, 6), i32([[3, 4, 2], [1, 0, 8]])
        kw, lse = {}, torch.zeros((3, 6), device="cuda")
        if form == "all":
            kw = dict(out=torch.empty_like(q), lse=lse, scale=0.1, window=20,
                      workspace=torch.empty(P.paged_attn_workspace_bytes(q, c, table), dtype=torch.uint8, device="cuda"))
        if form == "stream":
            kw["stream"] = torch.cuda.current_stream()
        return [P.paged_attn(q, c, table, i32([0, 2, 3]), i32([40, 17]), **kw), lse]
    got, want, taken = both(monkeypatch, call)
    same(got, want)
    assert taken == [True]


def test_what_the_marshalling_leaves_is_still_checked():
    import paper_2604_17397_amd as P
    c = P.PagedKV(*pools())
    q, table = x(3, 6), i32([[3, 4, 2], [1, 0, 8]])
    freqs, _ = P.rope_frequencies(64)
    for kw in (dict(q=x(3, 6, torch.float16)), dict(q=x(3, 6).cpu()), dict(q_start=i32([0, 1])), dict(lse=torch.zeros((3, 5), device="cuda")),
               dict(block_table=table.cpu()), dict(kv_lens=i32([1, 2, 3]))):
        with pytest.raises(ValueError):
            P.paged_attn(**{**dict(q=q, cache=c, block_table=table, q_start=i32([0, 2, 3]), kv_lens=i32([40, 17])), **kw})
    with pytest.raises(P.SdvgError) as e:
        P.paged_attn(x(3, 5), c, table, i32([0, 2, 3]), i32([40, 17]))      # 5 heads over 2 key heads
    assert e.value.status == -2
    with pytest.raises(P.SdvgError) as e:
        P.page_plan(i32([1, 2]), i32([1, 1]), table, 12, max_tokens=2)
    assert e.value.status == -4
    with pytest.raises(P.SdvgError) as e:
        P.rope_positions(q, i32([0, 1, 2]), freqs[:4])
    assert e.value.status == -2
    with pytest.raises(ValueError):
        P.paged_commit(c, q[:, :2], q[:, :2], torch.zeros(2, dtype=torch.int64, device="cuda"))
    cached = i32([1, 2])
    plan = P.PagePlan(2, 4)
    plan.kv_lens = cached
    with pytest.raises(P.SdvgError) as e:       # a length that is read and written
        P.page_plan(cached, i32([1, 1]), table, 16, out=plan)
    assert e.value.status == -3


def test_other_forms():
    """A tensor subclass, an integer scale and a strided table go through the Python code."""
    import paper_2604_17397_amd as P
    c = P.PagedKV(*pools())
    q, table = x(3, 6), i32([[3, 4, 2], [1, 0, 8]])
    args = (table, i32([0, 2, 3]), i32([40, 17]))
    want = P.paged_attn(q, c, *args, scale=1.0)

    class Sub(torch.Tensor):
        pass
    same(P.paged_attn(q.as_subclass(Sub), c, *args, scale=1).as_subclass(torch.Tensor), want)
    wide = torch.full((2, 7), -1, dtype=torch.int32, device="cuda")
    wide[:, :3] = table
    same(P.paged_attn(q, c, wide[:, :3], *args[1:], scale=1.0), want)
