"""sdvg_paged_prefix_attn against the definition in 64 bits, element by element.

The bounds are those of sdvg_paged_attn: with h = half a step of the 16-bit type relative to the value and A = sum p |v|, the result is
rounded once (h |o|), a probability enters the product as two 16-bit numbers (well below h A), and the scores have fp32 sums of 128 products, at
most 128 x 2^-24 x scale x sum |q k| off, here below 2^-12 of a probability (2^-12 A). lse has the scores' error alone."""
import math

import numpy as np
import pytest
import torch

from paged_util import i32
from test_gpu_paged_attn import HALF_STEP, Case

pytestmark = pytest.mark.gpu


class Shared(Case):
    """groups: (shared keys, [(keys behind them, new tokens), ...]). The shared pages of all but a group's first request are the first one's;
    the pages that they would have had hold poison."""

    def __init__(self, groups, heads, kv_heads, page, kind="bf16", cache=None, pool="token", seed=1, q_how="plain"):
        requests = [(n + own, new) for n, rest in groups for own, new in rest]
        super().__init__(requests, heads, kv_heads, page, kind, cache, pool, seed=seed, q_how=q_how)
        self.groups = groups
        starts = np.concatenate([[0], np.cumsum([len(rest) for _, rest in groups])]).astype(int)
        self.group_start, self.prefix_lens = i32(starts), i32([n for n, _ in groups])
        raw = [t.view(torch.uint8 if cache == "e4m3" else torch.int16) for t in (self.k, self.v)]
        poison = torch.tensor(float("nan"), device="cuda").to(self.k.dtype).view(raw[0].dtype)
        for g, (n, rest) in enumerate(groups):
            for r in range(starts[g] + 1, starts[g + 1]):
                whole = n // page
                for t in raw:
                    t[self.table[r, :whole].long()] = poison
                    if n % page:
                        t[self.table[r, whole], :n % page] = t[self.table[starts[g], whole], :n % page]
                self.table[r, :whole] = self.table[starts[g], :whole]

    def need(self, n_groups=None):
        import paper_2604_17397_amd as P
        return P.paged_prefix_attn_workspace_bytes(self.q, self.handle(), self.table, len(self.groups) if n_groups is None else n_groups)

    def run(self, workspace=True, window=0, **kw):
        import paper_2604_17397_amd as P
        ws = torch.full((self.need(),), 255, dtype=torch.uint8, device="cuda") if workspace is True else workspace
        args = dict(group_start=self.group_start)
        args.update(kw)
        return P.paged_prefix_attn(self.q, self.handle(), self.table, self.q_start, self.kv_lens, self.prefix_lens, window=window,
                                   workspace=ws, **args)

    def check(self, window=0, scale=None, workspace=True, **kw):
        want, size, want_lse = self.want(window, scale)
        lse = torch.full(self.q.shape[:2], 55.0, device="cuda")
        got = self.run(workspace, window, scale=scale, lse=lse, **kw)
        torch.cuda.synchronize()
        h = HALF_STEP[self.kind]
        tiny = 2.0**-25 if self.kind == "f16" else 0.0
        excess = (got.double() - want).abs() - ((h + 2.0**-12) * size + h * want.abs() + tiny)
        assert not torch.isnan(excess).any() and excess.max().item() <= 0, excess.max().item()
        empty = torch.isinf(want_lse)
        assert torch.equal(torch.isinf(lse), empty) and (got[empty] == 0).all()
        assert ((lse.double() - want_lse).abs()[~empty] <= 2.0**-12).all()
        return got


GROUPS = {
    "one request": [(100, [(1, 1)])],
    "one key": [(1, [(1, 1), (5, 1)])],
    "a tile": [(64, [(1, 1), (33, 1), (2, 2)])],
    "past a tile": [(65, [(1, 1)] * 9)],
    "odd": [(1037, [(1 + 7 * i, 1) for i in range(11)])],
    "nothing shared": [(0, [(40, 1), (3, 2)])],
    "long": [(20011, [(50, 1), (1000, 2), (1, 1)])],
    "many rows": [(700, [(1 + 37 * i % 300, 1 + i % 3) for i in range(90)])],
    "groups": [(130, [(5, 1), (700, 2)]), (0, [(64, 1)]), (3001, [(1, 1)] * 6), (7, [(255, 8), (9, 0), (0, 0)]), (64, [])],
    "many groups": [(11 * i % 200, [(3 + i, 1), (1, 1)]) for i in range(70)],
    "no new token": [(500, [(9, 0), (4, 1), (0, 0)])],
}


@pytest.mark.parametrize("groups", list(GROUPS))
@pytest.mark.parametrize("heads,kv_heads,page", [(1, 1, 8), (12, 12, 16), (5, 1, 24), (12, 4, 64), (32, 2, 256), (40, 8, 16)])
def test_groups_and_heads(groups, heads, kv_heads, page):
    Shared(GROUPS[groups], heads, kv_heads, page, seed=heads + page).check()


@pytest.mark.parametrize("kind,cache", [("bf16", None), ("f16", None), ("bf16", "e4m3"), ("f16", "e4m3")])
@pytest.mark.parametrize("pool,q_how", [("token", "wide"), ("head", "plain"), ("padded", "plain")])
@pytest.mark.parametrize("window", [0, 1, 40, 600, 100000])
@pytest.mark.parametrize("groups,heads,kv_heads,page", [("groups", 10, 2, 16), ("many rows", 8, 1, 24), ("long", 6, 3, 64), ("a tile", 48, 1, 8)])
def test_types_layouts_and_windows(kind, cache, pool, q_how, window, groups, heads, kv_heads, page):
    Shared(GROUPS[groups], heads, kv_heads, page, kind, cache, pool, q_how=q_how).check(window=window)


def test_one_group_without_starts_and_requests_outside_of_groups():
    c = Shared(GROUPS["odd"], 6, 2, 16)
    a = c.check()
    assert torch.equal(a, c.check(group_start=None))
    # the first and the last two requests belong to no group
    c = Shared([(0, [(300, 1)]), (517, [(9, 1), (1, 2), (40, 1)]), (0, [(64, 1), (5, 1)])], 6, 2, 16)
    c.groups, c.group_start, c.prefix_lens = c.groups[1:2], i32([1, 4]), i32([517])
    c.check()


@pytest.mark.parametrize("cache", [None, "e4m3"])
@pytest.mark.parametrize("n", [203, 206, 240, 10**6])
def test_prefix_that_reaches_into_the_new_tokens(cache, n):
    """A row sees no key behind its own position, whatever the prefix's length says."""
    c = Shared([(200, [(6, 6)])], 6, 2, 16, cache=cache)
    c.prefix_lens = i32([n])
    c.check()


def test_negative_and_odd_numbers_are_clamped():
    c = Shared([(70, [(3, 1), (8, 2)])], 4, 2, 16)
    want = c.check()
    for starts, lens in [([0, 2], [-5]), ([0, 2], [0])]:
        c.group_start, c.prefix_lens = i32(starts), i32(lens)
        assert (c.check() - want).abs().max() <= 2.0**-6
    out = torch.empty_like(c.q)
    for starts, lens in [([-4, 900], [70]), ([2, 0], [70]), ([0, 2], [2**31 - 1]), ([1, 1], [70]), ([-2**31, 2**31 - 1], [-2**31])]:
        c.group_start, c.prefix_lens = i32(starts), i32(lens)
        c.run(out=out)
        torch.cuda.synchronize()
    c.group_start, c.prefix_lens = i32([0, 2]), i32([70])
    for starts, lens in [([-3, 1, 900], [73, 78]), ([0, 2, 1], [-5, 78]), ([5, 6, 7], [73, 78]), ([0, 1, 2], [2**31 - 1, 2**31 - 1])]:
        c.q_start, c.kv_lens = i32(starts), i32(lens)
        c.run(out=out)
        torch.cuda.synchronize()


@pytest.mark.parametrize("cache", [None, "e4m3"])
def test_pages_that_are_not_there(cache):
    c = Shared([(200, [(2, 2), (30, 1), (1, 1)])], 4, 2, 8, cache=cache)
    pages = c.k.shape[0]
    want_gone = []
    for j, bad in ((3, -1), (7, pages), (24, 2**31 - 1)):
        c.table[:, j] = bad
        want_gone += [(r, j) for r in range(3)]
    want, size, _ = c.want(gone=want_gone)
    got = c.run()
    torch.cuda.synchronize()
    h = HALF_STEP["bf16"]
    excess = (got.double() - want).abs() - ((h + 2.0**-12) * size + h * want.abs())
    assert not torch.isnan(excess).any() and excess.max().item() <= 0
    c.table[:] = -1
    lse = torch.empty(c.q.shape[:2], device="cuda")
    assert (c.run(lse=lse) == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("kind,cache", [("bf16", None), ("f16", "e4m3")])
@pytest.mark.parametrize("window", [1, 37, 64, 500])
def test_what_lies_ahead_of_the_windows_may_be_anything(kind, cache, window):
    groups = [(700, [(3, 1), (9, 2), (300, 1)]), (64, [(1, 1)])]
    c = Shared(groups, 6, 2, 16, kind, cache)
    want = c.check(window=window)
    poison = torch.tensor(float("nan"), device="cuda").to(c.k.dtype).view(torch.uint8 if cache else torch.int16)
    for g, (n, rest) in enumerate(groups):
        s = int(c.group_start[g])
        first = max(0, min(n + own - new + 1 - window for own, new in rest))
        for j in range(first // 16 * 16, first):
            for r in range(s, s + len(rest)):
                for t in (c.k, c.v):
                    t.view(poison.dtype)[c.table[r, j // 16], j % 16] = poison
        c.table[s:s + len(rest), :first // 16] = torch.tensor([-1, 2**31 - 1], dtype=torch.int32, device="cuda").repeat(100)[:first // 16]
    got = c.run(window=window)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_without_a_workspace_it_is_paged_attn():
    import paper_2604_17397_amd as P
    c = Shared(GROUPS["many rows"], 6, 2, 16)
    args = c.q, c.handle(), c.table, c.q_start, c.kv_lens
    assert torch.equal(c.run(None), P.paged_attn(*args))
    small = torch.full((c.need() - 16,), 201, dtype=torch.uint8, device="cuda")
    assert torch.equal(c.run(small), P.paged_attn(*args, workspace=small))
    empty = c.prefix_lens[:0]
    ws = torch.empty(c.need(0), dtype=torch.uint8, device="cuda")
    assert torch.equal(P.paged_prefix_attn(*args, empty, group_start=c.group_start[:1], workspace=ws), P.paged_attn(*args, workspace=ws))
    guarded = torch.full((c.need() + 4096,), 201, dtype=torch.uint8, device="cuda")
    want = c.check()
    assert torch.equal(c.run(guarded[16:16 + c.need()]), want) and (guarded[:16] == 201).all() and (guarded[16 + c.need():] == 201).all()


def test_in_place_streams_and_rows_of_nobody():
    import paper_2604_17397_amd as P
    cases = [Shared([(5000, [(30, 1), (5, 2)]), (77, [(1, 1)])], 8, 2, 16, seed=s) for s in (1, 2)]
    want = [c.check().clone() for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    outs = [torch.full((c.n_tokens + 2, 12, 128), 3.0, dtype=torch.bfloat16, device="cuda") for c in cases]
    ws = [torch.empty(c.need(), dtype=torch.uint8, device="cuda") for c in cases]
    torch.cuda.synchronize()
    for _ in range(20):
        for c, s, o, w in zip(cases, streams, outs, ws):
            c.run(w, out=o[1:-1, 2:10], stream=s)
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert torch.equal(o[1:-1, 2:10], w) and (o[0] == 3).all() and (o[-1] == 3).all() and (o[:, :2] == 3).all() and (o[:, 10:] == 3).all()
    c = cases[0]
    q = torch.cat([c.q[:1] * 0 + 7, c.q, c.q[:1] * 0 + 7])
    keep = q.clone()
    ws = torch.empty(P.paged_prefix_attn_workspace_bytes(q, c.handle(), c.table, 2), dtype=torch.uint8, device="cuda")
    P.paged_prefix_attn(q, c.handle(), c.table, c.q_start + 1, c.kv_lens, c.prefix_lens, c.group_start, out=q, workspace=ws)
    torch.cuda.synchronize()
    got, h = q[1:-1].double(), HALF_STEP["bf16"]
    exact, size, _ = c.want()
    assert ((got - exact).abs() <= (h + 2.0**-12) * size + h * exact.abs()).all() and torch.equal(q[0], keep[0]) and torch.equal(q[-1], keep[-1])
    e = c.q[:0]
    assert P.paged_prefix_attn(e, c.handle(), c.table, i32([0] * 4), c.kv_lens, c.prefix_lens, c.group_start).shape == (0, 8, 128)


@pytest.mark.parametrize("cache", [None, "e4m3"])
def test_graphs_with_other_numbers(cache):
    """Two captured calls that share a workspace, replayed in turn with other lengths, prefixes and groups in the arrays."""
    import paper_2604_17397_amd as P
    cases = [Shared([(4000, [(30, 1), (5, 2), (600, 3)])], 8, 2, 16, cache=cache, seed=s) for s in (1, 2)]
    for c in cases:
        c.group_start, c.prefix_lens = i32([0, 2, 3]), i32([4000, 4000])
        c.groups = c.groups * 2
    ws = torch.empty(max(c.need() for c in cases), dtype=torch.uint8, device="cuda")
    outs = [torch.empty_like(c.q) for c in cases]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graphs = []
        for c, o in zip(cases, outs):
            c.run(ws, out=o)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                c.run(ws, out=o)
            graphs.append(g)
        for starts, lens, own in [([0, 2, 3], [4000, 4000], [30, 5, 600]), ([0, 3, 3], [100, 5], [1, 2, 3]), ([0, 1, 3], [0, 3999], [7, 2, 60]),
                                  ([0, 2, 3], [4000, 64], [30, 5, 600])]:
            for c, g, o in zip(cases, graphs, outs):
                c.group_start.copy_(i32(starts))
                c.prefix_lens.copy_(i32(lens))
                of = [0 if r < starts[1] else 1 for r in range(3)]
                c.kv_lens.copy_(i32([lens[of[r]] + own[r] for r in range(3)]))
                torch.cuda.synchronize()
                want = c.run(torch.empty(c.need(), dtype=torch.uint8, device="cuda"))
                o.fill_(float("nan"))
                g.replay()
                torch.cuda.synchronize()
                assert torch.equal(o, want), (starts, lens, own)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_row_that_is_not_finite_stays_by_itself(bad):
    c = Shared([(700, [(3, 3), (65, 4), (30, 8)])], 10, 2, 16)
    want, size, _ = c.want()
    c.q = c.q.clone()
    c.q[1], c.q[8] = bad, bad
    lse = torch.empty(c.q.shape[:2], device="cuda")
    got = c.run(lse=lse)
    torch.cuda.synchronize()
    rest = [t for t in range(c.n_tokens) if t not in (1, 8)]
    h = HALF_STEP["bf16"]
    excess = ((got.double() - want).abs() - ((h + 2.0**-12) * size + h * want.abs()))[rest]
    assert not torch.isnan(excess).any() and excess.max().item() <= 0
    assert torch.isnan(got[[1, 8]]).all() and torch.isnan(lse[[1, 8]]).all()


def test_peaked_and_growing_scores():
    for kind in ("bf16", "f16"):
        for at in (0, 31, 63, 64, 500, 2047):
            c = Shared([(2048, [(5, 1), (1, 1), (9, 1)])], 2, 1, 16, kind)
            c.k[c.table[0, at // 16], at % 16, 0] = c.q[0, 0] * 3
            c.check()
        c = Shared([(2048, [(5, 1), (1, 1)])], 2, 1, 16, kind)
        for j in range(0, 2048, 16):
            c.k[c.table[0, j // 16], :, 0] = (c.q[0, 0].float() * (j / 2048.0) * 2).to(c.k.dtype)
        c.check()


def test_same_bits_every_time():
    c = Shared(GROUPS["many rows"], 10, 2, 16, "f16")
    a = c.check()
    for _ in range(3):
        assert torch.equal(a, c.run())


@pytest.mark.parametrize("kind,cache", [("bf16", None), ("f16", None), ("bf16", "e4m3"), ("f16", "e4m3")])
@pytest.mark.parametrize("groups", [[(7, [(3, 1), (1, 1)])], [(40, [(20, 1), (30, 3)])], [(64, [(5, 1)]), (50, [(9, 2), (14, 1)])]])
@pytest.mark.parametrize("heads,kv_heads", [(4, 2), (3, 1), (24, 2)])
def test_what_is_lost_beside_the_last_rounding(kind, cache, groups, heads, kv_heads):
    """Elements that are small beside A, where the result's own rounding leaves the rest to be seen: scores of one exact product each, from -4 to
    4. In units of A: a probability as two 16-bit numbers 2^-16 (bf16) or 2^-22; its exponent, of up to 17 with three roundings to 32 bits,
    2^-18; fp32 sums over up to 64 keys of a wave, twice (product and sum), and up to 4 pieces, 136 roundings, 2^-16.9: below 2^-15 (bf16) and
    2^-16 (fp16)."""
    c = Shared(groups, heads, kv_heads, 16, kind, cache, seed=len(groups) + heads)
    if cache:
        c.k_scale.fill_(1.0)
        c.v_scale.fill_(1.0)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(7)
    as_bytes = (lambda t: t.view(torch.uint8)) if cache else (lambda t: t)
    k = torch.zeros(c.k.shape, device="cuda")
    k[..., 0] = (torch.rand(k.shape[:3], generator=gen, device="cuda") * 8 - 4).to(torch.float8_e4m3fn).float()
    as_bytes(c.k).copy_(as_bytes(k.to(c.k.dtype)))
    for g, (n, rest) in enumerate(groups):      # (the part of a page that a prefix ends in is everybody's alike)
        s = int(c.group_start[g])
        for r in range(s + 1, s + len(rest)):
            if n % 16:
                as_bytes(c.k)[c.table[r, n // 16], :n % 16] = as_bytes(c.k)[c.table[s, n // 16], :n % 16]
    c.q = torch.zeros_like(c.q)
    c.q[..., 0] = 1
    want, size, _ = c.want(scale=1.0)
    got = c.run(scale=1.0).double()
    torch.cuda.synchronize()
    tiny = 2.0**-25 if kind == "f16" else 0.0
    assert (want.abs() < 2.0**-4 * size).any()
    excess = (got - want).abs() - ({"bf16": 2.0**-15, "f16": 2.0**-16}[kind] * size + HALF_STEP[kind] * want.abs() + tiny)
    assert excess.max().item() <= 0, (excess / size).max().item()


def test_pool_past_32_bits():
    import paper_2604_17397_amd as P
    H, page = 8, 16
    pages = (5 << 30) // (page * H * 256)
    for how in ("token", "head"):
        shape = (pages, page, H, 128) if how == "token" else (H, pages, page, 128)
        pools = [torch.empty(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        k, v = pools if how == "token" else [t.permute(1, 2, 0, 3) for t in pools]
        n = 200
        table = i32([[pages - 1 - 7 * i for i in range(12)] + [pages - 100 - r] for r in range(3)])
        j = torch.arange(n, device="cuda")
        x, y = (torch.randn((3, n, H, 128), device="cuda").bfloat16() for _ in range(2))
        x[1:, :192], y[1:, :192] = x[:1, :192], y[:1, :192]
        for r in range(3):
            k[table[r].long()[j // page], j % page], v[table[r].long()[j // page], j % page] = x[r], y[r]
        q = torch.randn((3, H, 128), device="cuda").bfloat16()
        c = P.PagedKV(k, v)
        ws = torch.empty(P.paged_prefix_attn_workspace_bytes(q, c, table), dtype=torch.uint8, device="cuda")
        got = P.paged_prefix_attn(q, c, table, i32([0, 1, 2, 3]), i32([n] * 3), i32([192]), workspace=ws).double()
        torch.cuda.synchronize()
        for r in range(3):
            for h in range(H):
                p = torch.softmax(x[r, :, h].double() @ q[r, h].double() / math.sqrt(128), 0)
                assert ((got[r, h] - p @ y[r, :, h].double()).abs() <= 2.0**-7 * (p @ y[r, :, h].double().abs())).all()
        del pools, k, v, c
        torch.cuda.empty_cache()


@pytest.mark.parametrize("sizes", [[2] * 200, [0] * 300 + [1] + [0] * 70 + [64, 65] + [0] * 129, [1] * 64 + [3] * 64 + [0, 0, 130]],
                         ids=["many", "empty ones", "batches"])
def test_more_groups_than_a_wave_has_lanes(sizes):
    case = Shared([(11 * i % 190, [(1 + (i + j) % 40, 1) for j in range(n)]) for i, n in enumerate(sizes)], 4, 2, 16, pool="head")
    case.check()
    case.check(window=70)
