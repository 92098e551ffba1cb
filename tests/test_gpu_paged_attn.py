"""sdvg_paged_attn against the definition in 64 bits, element by element.

With h = half a step of the 16-bit type relative to the value and A = sum p |v|: every probability is rounded once
(h A), the result once (h |o|), and the scores have fp32 sums of 128 products, at most 128 x 2^-24 x scale x sum |q k| off,
here below 2^-12 of a probability (2^-12 A). lse has the scores' error alone."""
import math

import numpy as np
import pytest
import torch

from paged_util import i32

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f16": torch.float16}
HALF_STEP = {"bf16": 2.0**-8, "f16": 2.0**-11}


class Case:
    """Requests of the given (length, new tokens) over a pool whose unused places hold NaN (16 bit) or the largest number."""

    def __init__(self, requests, heads, kv_heads, page, kind="bf16", cache=None, pool="token", spare=2, seed=1, q_how="plain"):
        self.requests, self.heads, self.kv_heads, self.page, self.kind = requests, heads, kv_heads, page, kind
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        dt = DT[kind]
        ct = torch.float8_e4m3fn if cache == "e4m3" else dt
        used = [-(-n // page) for n, _ in requests]
        width = max(max(used), 1) + 1
        pages = sum(used) + spare
        ids = torch.randperm(pages, generator=gen, device="cuda").cpu().numpy()
        table = np.full((len(requests), width), -1)
        at = 0
        for r, u in enumerate(used):
            table[r, :u] = ids[at:at + u]
            at += u
        self.table = i32(table)
        starts = np.concatenate([[0], np.cumsum([n for _, n in requests])])
        self.q_start, self.kv_lens = i32(starts), i32([n for n, _ in requests])
        self.n_tokens = int(starts[-1])
        q = torch.randn((self.n_tokens + 1, heads + 2, 128), generator=gen, device="cuda").to(dt)
        self.q = q[:-1, 1:-1] if q_how == "wide" else q[:-1, :heads].contiguous()
        shape = {"token": (pages, page, kv_heads, 128), "head": (kv_heads, pages, page, 128),
                 "padded": (pages, page + 1, kv_heads, 144)}[pool]
        self.k_scale = self.v_scale = None
        if cache == "e4m3":
            self.k_scale, self.v_scale = ((0.5 + torch.rand(kv_heads, generator=gen, device="cuda")) / 64 for _ in range(2))

        def storage():
            t = torch.randn(shape, generator=gen, device="cuda")
            t = (t * 48).clamp(-400, 400).to(ct) if cache == "e4m3" else t.to(ct)
            return t.permute(1, 2, 0, 3) if pool == "head" else t[:, :page, :, :128] if pool == "padded" else t
        self.k, self.v = storage(), storage()
        # what no request has is poison
        mine = torch.zeros((pages, page), dtype=torch.bool, device="cuda")
        for r, (n, _) in enumerate(requests):
            for j in range(used[r]):
                mine[table[r, j], :min(page, n - j * page)] = True
        poison = torch.tensor(float("nan"), device="cuda").to(ct).view(torch.uint8 if cache == "e4m3" else torch.int16)
        for t in (self.k, self.v):
            raw = t.view(torch.uint8 if cache == "e4m3" else torch.int16)
            raw[~mine] = poison

    def handle(self):
        import paper_2604_17397_amd as P
        return P.PagedKV(self.k, self.v, self.k_scale, self.v_scale)

    def want(self, window=0, scale=None, gone=()):
        """(out, A, lse) in 64 bits; `gone`: pages (request, index) that are not there."""
        scale = 1 / math.sqrt(128) if scale is None else scale
        group = self.heads // self.kv_heads
        out = torch.zeros(self.q.shape, dtype=torch.float64, device="cuda")
        size, lse = torch.zeros_like(out), torch.full(self.q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
        t = 0
        for r, (n, new) in enumerate(self.requests):
            j = torch.arange(n, device="cuda")
            page = self.table[r].long()[j // self.page]
            there = torch.ones(n, dtype=torch.bool, device="cuda")
            for rr, i in gone:
                if rr == r:
                    there &= j // self.page != i
            sees = torch.arange(n - new + 1, n + 1, device="cuda")[:, None]
            ok = there & (j < sees)
            if window:
                ok &= j >= sees - window
            for h in range(self.kv_heads):
                if n == 0 or new == 0:
                    continue
                k, v = (c[page.clamp(0, c.shape[0] - 1), j % self.page, h].double() for c in (self.k, self.v))
                k, v = (torch.where(there[:, None], x, 0.0) for x in (k, v))
                ks = 1.0 if self.k_scale is None else self.k_scale[h].double()
                vs = 1.0 if self.v_scale is None else self.v_scale[h].double()
                for g in range(group):
                    s = (self.q[t:t + new, h * group + g].double() @ k.t().contiguous()) * (scale * ks)
                    s = torch.where(ok, s, -math.inf)
                    some = ok.any(1)
                    p = torch.where(some[:, None], torch.softmax(s, 1), 0.0)
                    out[t:t + new, h * group + g] = p @ v * vs
                    size[t:t + new, h * group + g] = p @ v.abs() * vs
                    lse[t:t + new, h * group + g] = torch.logsumexp(s, 1)
            t += new
        return out, size, lse

    def check(self, window=0, scale=None, gone=(), workspace=True, out=None, **kw):
        import paper_2604_17397_amd as P
        handle = self.handle()
        ws = None
        if workspace:
            ws = torch.full((P.paged_attn_workspace_bytes(self.q, handle, self.table),), 255, dtype=torch.uint8, device="cuda")
        lse = torch.full(self.q.shape[:2], 55.0, device="cuda")
        want, size, want_lse = self.want(window, scale, gone)
        got = P.paged_attn(self.q, handle, self.table, self.q_start, self.kv_lens, out=out, lse=lse, scale=scale, window=window,
                           workspace=ws, **kw)
        torch.cuda.synchronize()
        h = HALF_STEP[self.kind]
        tiny = 2.0**-25 if self.kind == "f16" else 0.0       # half a step below f16's smallest normal number
        excess = (got.double() - want).abs() - ((h + 2.0**-12) * size + h * want.abs() + tiny)
        assert not torch.isnan(excess).any() and excess.max().item() <= 0, excess.max().item()
        empty = torch.isinf(want_lse)
        assert torch.equal(torch.isinf(lse), empty) and (got[empty] == 0).all()
        assert ((lse.double() - want_lse).abs()[~empty] <= 2.0**-12).all()
        return got


LENGTHS = {
    "one": [(1, 1)], "tile": [(32, 1)], "past a tile": [(33, 1)], "odd": [(1037, 1)], "long": [(40001, 1)],
    "ragged": [(5, 1), (700, 1), (64, 1), (1, 1), (3001, 1), (129, 1), (255, 1)],
    "verify": [(5, 5), (700, 3), (64, 1), (9, 0), (0, 0), (3001, 8), (33, 2)],
    "many": [(1 + 37 * i % 300, i % 3) for i in range(150)],
    "drafts": [(2000 + i, 9) for i in range(5)],
}


@pytest.mark.parametrize("lengths", list(LENGTHS))
@pytest.mark.parametrize("heads,kv_heads,page", [(1, 1, 8), (12, 12, 16), (5, 1, 24), (12, 4, 64), (32, 2, 256), (40, 1, 16)])
@pytest.mark.parametrize("workspace", [True, False])
def test_lengths_and_heads(lengths, heads, kv_heads, page, workspace):
    Case(LENGTHS[lengths], heads, kv_heads, page, seed=heads + page).check(workspace=workspace)


@pytest.mark.parametrize("kind,cache", [("bf16", None), ("f16", None), ("bf16", "e4m3"), ("f16", "e4m3")])
@pytest.mark.parametrize("pool,q_how", [("token", "wide"), ("head", "plain"), ("padded", "plain")])
@pytest.mark.parametrize("window", [0, 1, 40, 100000])
@pytest.mark.parametrize("lengths,heads,kv_heads,page", [("verify", 10, 2, 16), ("drafts", 8, 1, 24), ("long", 6, 3, 64)])
def test_types_layouts_and_windows(kind, cache, pool, q_how, window, lengths, heads, kv_heads, page):
    Case(LENGTHS[lengths], heads, kv_heads, page, kind, cache, pool, q_how=q_how).check(window=window)


def test_in_place_scale_stream_and_rows_behind_the_last():
    import paper_2604_17397_amd as P
    c = Case([(300, 1), (5000, 2)], 4, 2, 16)
    c.check(scale=0.02)
    c.check(scale=0.5)
    q = torch.randn((6, 4, 128), device="cuda").bfloat16()
    q[:3] = c.q
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    want = c.check()
    h = c.handle()
    ws = torch.empty(P.paged_attn_workspace_bytes(q, h, c.table), dtype=torch.uint8, device="cuda")
    out = torch.full_like(q, 9.0)
    side.wait_stream(torch.cuda.current_stream())
    assert P.paged_attn(q, h, c.table, c.q_start, c.kv_lens, out=out, workspace=ws, stream=side) is out
    side.synchronize()
    assert torch.equal(out[:3], want) and (out[3:] == 9).all()
    keep = q.clone()
    P.paged_attn(q, h, c.table, c.q_start, c.kv_lens, out=q, workspace=ws)
    torch.cuda.synchronize()
    assert torch.equal(q[:3], want) and torch.equal(q[3:], keep[3:])


def test_pages_that_are_not_there():
    c = Case([(200, 2), (64, 1), (24, 1)], 4, 2, 8, spare=4)
    pages = c.k.shape[0]
    c.table[0, 3], c.table[0, 7], c.table[0, 24], c.table[2, 0], c.table[2, 1], c.table[2, 2] = -1, pages, -7, -1, 2**31 - 1, -1
    got = c.check(gone=[(0, 3), (0, 7), (0, 24), (2, 0), (2, 1), (2, 2)])
    assert (got[3] == 0).all()
    # a table that is shorter than the request
    c = Case([(200, 1)], 4, 2, 8)
    c.table = c.table[:, :10].contiguous()
    d = Case([(200, 1)], 4, 2, 8)
    want, size, _ = d.want(gone=[(0, i) for i in range(10, 25)])
    import paper_2604_17397_amd as P
    got = P.paged_attn(c.q, c.handle(), c.table, c.q_start, c.kv_lens)
    assert ((got.double() - want).abs() <= 2.0**-7 * (size + want.abs())).all()


def test_more_new_tokens_than_keys_and_empty_rows():
    """A length that is shorter than its new tokens: the first ones lie before the start and see nothing."""
    c = Case([(3, 3), (50, 2)], 6, 3, 16)
    c.requests = [(3, 5), (50, 2)]
    c.q_start, c.n_tokens = i32([0, 5, 7]), 7
    c.q = torch.randn((7, 6, 128), device="cuda").bfloat16()
    got = c.check()
    assert (got[:2] == 0).all() and (got[2:] != 0).any()


def test_numbers_out_of_range_are_clamped():
    import paper_2604_17397_amd as P
    c = Case([(40, 1), (70, 1)], 2, 1, 16)
    out = torch.full_like(c.q, 7.0)
    for starts, lens in [([-3, 1, 900], [40, 70]), ([0, 2, 1], [-5, 70]), ([5, 6, 7], [40, 70]), ([0, 1, 2], [2**31 - 1, 2**31 - 1]),
                         ([0, 1, 2], [-2**31, 1])]:
        out.fill_(7.0)
        P.paged_attn(c.q, c.handle(), c.table, i32(starts), i32(lens), out=out)
        torch.cuda.synchronize()
    e = torch.empty((0, 2, 128), dtype=torch.bfloat16, device="cuda")
    assert P.paged_attn(e, c.handle(), c.table, i32([0, 0, 0]), c.kv_lens).shape == (0, 2, 128)
    none = P.paged_attn(c.q, c.handle(), c.table[:0], i32([0]), i32([]), out=out.fill_(7.0))
    torch.cuda.synchronize()
    assert (none == 7).all()


@pytest.mark.parametrize("kind,cache", [("bf16", None), ("f16", "e4m3")])
@pytest.mark.parametrize("window", [1, 37, 64, 500])
def test_what_lies_ahead_of_the_window_may_be_anything(kind, cache, window):
    """A rolling cache: pages ahead of the first token's window are gone, and the rest of the page it begins in is no number."""
    requests = [(700, 3), (41, 2), (2000, 1), (1111, 8)]
    c = Case(requests, 6, 2, 16, kind, cache)
    want = c.check(window=window).clone()
    poison = torch.tensor(float("nan"), device="cuda").to(c.k.dtype)
    for r, (n, new) in enumerate(requests):
        first = max(0, n - new + 1 - window)
        for j in range(first // 16 * 16, first):
            for t in (c.k, c.v):
                raw = t.view(torch.uint8 if cache else torch.int16)
                raw[c.table[r, j // 16], j % 16] = poison.view(torch.uint8 if cache else torch.int16)
        c.table[r, :first // 16] = torch.tensor([-1, 2**31 - 1], dtype=torch.int32, device="cuda").repeat(400)[:first // 16]
    import paper_2604_17397_amd as P
    for ws in (None, torch.empty(P.paged_attn_workspace_bytes(c.q, c.handle(), c.table), dtype=torch.uint8, device="cuda")):
        got = P.paged_attn(c.q, c.handle(), c.table, c.q_start, c.kv_lens, window=window, workspace=ws)
        torch.cuda.synchronize()
        if ws is not None:
            assert torch.equal(got, want)
        assert not torch.isnan(got).any()


def test_pools_past_32_bits():
    """Offsets of pages, heads and slots beyond 2^32 bytes and 2^31 elements: token-major and head-major pools of 5 GiB."""
    import paper_2604_17397_amd as P
    H, page = 8, 16
    pages = (5 << 30) // (page * H * 256)
    for how in ("token", "head"):
        shape = (pages, page, H, 128) if how == "token" else (H, pages, page, 128)
        pools = [torch.empty(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        k, v = pools if how == "token" else [t.permute(1, 2, 0, 3) for t in pools]
        c = P.PagedKV(k, v)
        n = 200
        table = i32([[pages - 1 - 7 * i for i in range(13)]])
        x, y = (torch.randn((n, H, 128), device="cuda").bfloat16() for _ in range(2))
        j = torch.arange(n, device="cuda")
        slots = table[0].long()[j // page] * page + j % page
        P.paged_commit(c, x, y, slots)
        torch.cuda.synchronize()
        assert torch.equal(k[table[0].long()[j // page], j % page], x) and torch.equal(v[table[0].long()[j // page], j % page], y)
        q = torch.randn((1, H, 128), device="cuda").bfloat16()
        got = P.paged_attn(q, c, table, i32([0, 1]), i32([n])).double()
        torch.cuda.synchronize()
        for h in range(H):
            p = torch.softmax(x[:, h].double() @ q[0, h].double() / math.sqrt(128), 0)
            assert ((got[0, h] - p @ y[:, h].double()).abs() <= 2.0**-7 * (p @ y[:, h].double().abs())).all()
        del pools, k, v, c
        torch.cuda.empty_cache()


def test_two_streams_at_once_and_strided_output():
    """Calls that overlap, each with a workspace of its own, and rows ahead of the first request's left as they are."""
    import paper_2604_17397_amd as P
    cases = [Case([(30000, 1), (5, 1)], 8, 2, 16, seed=s) for s in (1, 2)]
    want = [c.check().clone() for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    outs = [torch.full((c.n_tokens + 1, 12, 128), 3.0, dtype=torch.bfloat16, device="cuda") for c in cases]
    ws = [torch.empty(P.paged_attn_workspace_bytes(c.q, c.handle(), c.table), dtype=torch.uint8, device="cuda") for c in cases]
    torch.cuda.synchronize()
    for _ in range(20):
        for c, s, o, w in zip(cases, streams, outs, ws):
            P.paged_attn(c.q, c.handle(), c.table, c.q_start, c.kv_lens, out=o[1:, 2:10], workspace=w, stream=s)
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert torch.equal(o[1:, 2:10], w) and (o[0] == 3).all() and (o[:, :2] == 3).all() and (o[:, 10:] == 3).all()
    c = cases[0]
    q = torch.cat([c.q[:1] * 0 + 7, c.q])
    out = torch.full_like(q, 3.0)
    P.paged_attn(q, c.handle(), c.table, c.q_start + 1, c.kv_lens, out=out, workspace=ws[0])
    torch.cuda.synchronize()
    assert torch.equal(out[1:], want[0]) and (out[0] == 3).all()


def test_split_and_whole_agree_and_repeat():
    """With and without the split the same result up to rounding; the same bits every time."""
    c = Case([(9000, 1), (100, 1), (20000, 1)], 10, 2, 16, "f16")
    a, b, d = c.check(), c.check(), c.check(workspace=False)
    assert torch.equal(a, b) and (a.float() - d.float()).abs().max() <= 2.0**-10 * d.float().abs().max()


def test_peaked_and_growing_scores():
    """Scores that rise from tile to tile, and one key that outweighs all others, wherever it is."""
    for kind in ("bf16", "f16"):
        for at in (0, 31, 32, 500, 2047):
            c = Case([(2048, 1)], 2, 1, 16, kind)
            place = c.table[0, at // 16], at % 16
            c.k[place[0], place[1], 0] = c.q[0, 0] * 3
            c.check()
        c = Case([(2048, 1)], 2, 1, 16, kind)
        for j in range(0, 2048, 16):
            c.k[c.table[0, j // 16], :, 0] = (c.q[0, 0].float() * (j / 2048.0) * 2).to(c.k.dtype)
        c.check()


def test_graph_with_other_lengths():
    """A captured call follows the lengths, tables and queries that are in the arrays when it is replayed."""
    import paper_2604_17397_amd as P
    c = Case([(5000, 2), (40, 1), (4999, 3)], 8, 2, 16)
    h = c.handle()
    ws = torch.empty(P.paged_attn_workspace_bytes(c.q, h, c.table), dtype=torch.uint8, device="cuda")
    out, lens = torch.empty_like(c.q), c.kv_lens.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        P.paged_attn(c.q, h, c.table, c.q_start, lens, out=out, workspace=ws)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            P.paged_attn(c.q, h, c.table, c.q_start, lens, out=out, workspace=ws)
        for a, b, d in [(5000, 40, 4999), (7, 33, 3), (5000, 1, 200), (900, 40, 4999)]:
            lens.copy_(i32([a, b, d]))
            torch.cuda.synchronize()
            want = P.paged_attn(c.q, h, c.table, c.q_start, lens, workspace=ws)
            out.fill_(float("nan"))
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want), (a, b, d)


def test_window_beyond_32_bits_is_refused():
    import paper_2604_17397_amd as P
    cache = P.PagedKV(*[torch.zeros((1, 16, 1, 128), device="cuda").bfloat16() for _ in range(2)])
    q = torch.zeros((1, 1, 128), device="cuda").bfloat16()
    with pytest.raises(ValueError, match="32 bits"):
        P.paged_attn(q, cache, i32([[0]]), i32([0, 1]), i32([1]), window=2**32 + 5)


@pytest.mark.parametrize("kv_heads", [1, 2])
@pytest.mark.parametrize("lengths", [[256], [257], [8 * 32] * 5, [1] * 70 + [3000], [255, 256, 257, 1000], [9 * 32] * 40, [64] * 300])
def test_around_the_shortest_request_that_is_split(lengths, kv_heads):
    """Tables as wide as the longest request needs: up to 256 keys no request is split and nothing joined."""
    c = Case([(n, 1) for n in lengths], 2 * kv_heads, kv_heads, 16, seed=len(lengths))
    c.table = c.table[:, :-1].contiguous()
    c.check()


@pytest.mark.parametrize("cache", [None, "e4m3"])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_row_that_is_not_finite_stays_by_itself(cache, bad):
    """A padded or broken token's q shares a tile with other rows; they do not see it."""
    import paper_2604_17397_amd as P
    c = Case([(700, 3), (65, 4), (3001, 8)], 10, 2, 16, cache=cache)
    ws = torch.empty(P.paged_attn_workspace_bytes(c.q, c.handle(), c.table), dtype=torch.uint8, device="cuda")
    args = c.handle(), c.table, c.q_start, c.kv_lens
    good = P.paged_attn(c.q, *args, workspace=ws)
    broken = c.q.clone()
    broken[1], broken[8] = bad, bad
    got = P.paged_attn(broken, *args, workspace=ws)
    want, size, _ = c.want()
    rest = [t for t in range(c.n_tokens) if t not in (1, 8)]
    # the maximum that a row is shifted by may be raised at another step than without them: each result holds the bound
    h = HALF_STEP["bf16"]
    for x in (good, got):
        excess = ((x.double() - want).abs() - ((h + 2.0**-12) * size + h * want.abs()))[rest]
        assert not torch.isnan(excess).any() and excess.max().item() <= 0
