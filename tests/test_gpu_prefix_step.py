"""Plan, commit, attention over a shared prompt and the draw of the next tokens together, as a program that samples several continuations of
each prompt uses them; the C++ marshalling of the last two; and their outputs on another stream."""
import math

import numpy as np
import pytest
import torch

from paged_util import i32
from sample_util import draw
from test_gpu_native_binding import both
from test_gpu_paged_native import pools, same, x
from test_gpu_paged_step import rows

pytestmark = pytest.mark.gpu
H, HK, PAGE, VOCAB = 6, 2, 16, 6 * 128
PROMPTS, CONTINUATIONS, PADDED, STEPS = (96, 16), (4, 3), 2, 6     # shared keys (whole pages), requests that share them, requests of the batch that are none


class Job:
    """Tokens are rows of tables of q, k and v; an output row is a row of logits. So all that a step computes is the framework's."""

    def __init__(self):
        import paper_2604_17397_amd as P
        self.R = sum(CONTINUATIONS) + PADDED
        self.real = sum(CONTINUATIONS)
        self.tables = [rows(7 + i, VOCAB, n) for i, n in enumerate((H, HK, HK))]
        self.freqs, _ = P.rope_frequencies(128)
        pages = 64
        self.kc, self.vc = (torch.full((pages, PAGE, HK, 128), float("nan"), device="cuda", dtype=torch.bfloat16) for _ in range(2))
        self.cache = P.PagedKV(self.kc, self.vc)
        self.starts = np.concatenate([[0], np.cumsum(CONTINUATIONS), [self.R]]).astype(int)     # the padding is a group without shared keys
        self.group_start, self.prefix_lens = i32(self.starts), i32(list(PROMPTS) + [0])
        table = torch.full((self.R, 12), -1, dtype=torch.int32)
        gen = np.random.default_rng(5)
        self.prompt = [gen.integers(0, VOCAB, n) for n in PROMPTS]
        held, at = [0] * self.R, 0
        for g, n in enumerate(PROMPTS):
            for r in range(self.starts[g], self.starts[g + 1]):
                table[r, :n // PAGE] = torch.arange(at, at + n // PAGE)
                held[r] = n // PAGE
            at += n // PAGE
        self.table, self.held, self.first_page = table.cuda(), i32(held), at
        self.cursor, self.free = i32([0]), i32(list(range(at, pages)))
        for g, n in enumerate(PROMPTS):     # a prompt's keys are committed once
            slots = (self.table[self.starts[g], :n // PAGE].long()[:, None] * PAGE + torch.arange(PAGE, device="cuda")).flatten()
            t = torch.from_numpy(self.prompt[g]).cuda()
            P.paged_commit(self.cache, self.tables[1][t], self.tables[2][t], slots, positions=i32(range(n)), freqs=self.freqs)
        self.cached = i32([n for g, n in enumerate(PROMPTS) for _ in range(CONTINUATIONS[g])] + [0] * PADDED)
        self.new = i32([1] * self.real + [0] * PADDED)
        self.tokens = torch.zeros(self.R, dtype=torch.int32, device="cuda")
        self.u, self.lp = torch.zeros(self.R, device="cuda"), torch.zeros(self.R, device="cuda")
        self.temperature = torch.tensor([0.05 * (1 + r % 3) for r in range(self.R)], device="cuda")
        self.top_k = i32([0, 50, 7] * self.R)[:self.R].contiguous()
        self.plan = P.PagePlan(self.R, self.R)
        self.out = torch.zeros((self.R, H, 128), dtype=torch.bfloat16, device="cuda")
        q = self.tables[0][:self.R]
        self.ws = torch.empty(P.paged_prefix_attn_workspace_bytes(q, self.cache, self.table, len(PROMPTS) + 1), dtype=torch.uint8, device="cuda")
        self.sample_ws = torch.empty(P.sample_tokens_workspace_bytes(self.R, VOCAB), dtype=torch.uint8, device="cuda")

    def step(self):
        import paper_2604_17397_amd as P
        q, k, v = (t[self.tokens.long()] for t in self.tables)
        P.page_plan(self.cached, self.new, self.table, PAGE, free_pages=self.free, held=self.held, next_free=self.cursor, out=self.plan)
        q = P.paged_commit(self.cache, k, v, self.plan.slots, positions=self.plan.positions, freqs=self.freqs, q=q)
        P.paged_prefix_attn(q, self.cache, self.table, self.plan.q_start, self.plan.kv_lens, self.prefix_lens, group_start=self.group_start,
                            out=self.out, workspace=self.ws)
        P.sample_tokens(self.out.view(self.R, VOCAB), self.u, temperature=self.temperature, top_k=self.top_k, top_p=0.95, out=self.tokens,
                        logprob=self.lp, workspace=self.sample_ws)
        self.held.copy_(self.plan.held)
        self.cursor.copy_(self.plan.next_free)
        self.cached.copy_(self.plan.kv_lens)

    def attention(self, tokens):
        """The last of a request's tokens, over all of them, in 64 bits."""
        t = torch.tensor(tokens, device="cuda")

        def turn(a, pos):
            a = a.double()
            lo, hi = a[..., :64], a[..., 64:]
            ang = (pos.double()[:, None] * self.freqs)[:, None, :]
            return torch.cat([lo * torch.cos(ang) - hi * torch.sin(ang), lo * torch.sin(ang) + hi * torch.cos(ang)], -1).bfloat16().double()
        pos = torch.arange(len(tokens), device="cuda")
        q, k, v = turn(self.tables[0][t[-1:]], pos[-1:]), turn(self.tables[1][t], pos), self.tables[2][t].double()
        out = torch.zeros((H, 128), dtype=torch.float64, device="cuda")
        for h in range(H):
            s = k[:, h // (H // HK)] @ q[0, h] / math.sqrt(128)
            out[h] = torch.softmax(s, 0) @ v[:, h // (H // HK)]
        return out


def run(captured):
    job = Job()
    first = i32([3] * job.R)
    rng = np.random.default_rng(11)
    numbers = [rng.random(job.R).astype(np.float32) for _ in range(STEPS)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    record = []
    with torch.cuda.stream(side):
        graph = None
        if captured:
            new = job.new.clone()
            job.new.zero_()
            job.step()      # nothing to do: no new token
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                job.step()
            job.new.copy_(new)
        job.tokens.copy_(first)
        for s in range(STEPS):
            job.u.copy_(torch.from_numpy(numbers[s]))
            job.out.fill_(5.0)
            given = job.tokens.clone()
            torch.cuda.synchronize()
            graph.replay() if captured else job.step()
            torch.cuda.synchronize()
            record.append([t.clone() for t in (given, job.out, job.tokens, job.lp)])
    return job, numbers, record


def test_continuations_of_shared_prompts():
    job, numbers, record = run(captured=False)
    history = [list(job.prompt[g]) for g, n in enumerate(CONTINUATIONS) for _ in range(n)]
    for s, (given, out, tokens, lp) in enumerate(record):
        assert (out[job.real:] == 5).all()
        for r in range(job.real):
            history[r].append(given[r].item())
            # (as in the test of plan, commit and attention: rotated rows are rounded to bf16, a step apart where the angle's last bits decide)
            assert (out[r].double() - job.attention(history[r])).abs().max().item() <= 2e-2
            token, want = draw(out[r].flatten().double().cpu().numpy(), numbers[s][r], job.temperature[r].item(), job.top_k[r].item(), float(np.float32(0.95)))
            assert tokens[r].item() == token
            assert abs(lp[r].item() - want) <= 2.0**-24 * abs(want) * (1 + 2.0**-20) + 2.0**-34
    assert len({tuple(h) for h in history}) > 4, "continuations differ"
    assert job.held[:job.real].tolist() == [n // PAGE + 1 for g, n in enumerate(PROMPTS) for _ in range(CONTINUATIONS[g])]
    assert job.cursor.item() == job.real


def test_the_same_captured():
    eager, replayed = run(False)[2], run(True)[2]
    for a, b in zip(eager, replayed):
        for s, t in zip(a, b):
            assert torch.equal(s.view(torch.uint8), t.view(torch.uint8))


def shared(P, **kw):
    c = P.PagedKV(*pools())
    q, table = x(3, 6), i32([[3, 4, 2], [3, 0, 8]])
    return c, q, table, (i32([0, 2, 3]), i32([40, 17])), i32([16])


@pytest.mark.parametrize("form", ["plain", "all", "stream", "groups"])
def test_marshalling_of_the_attention(monkeypatch, form):
    def call(P):
        c, q, table, lens, prefix = shared(P)
        kw, lse = {}, torch.zeros((3, 6), device="cuda")
        if form == "all":
            kw = dict(out=torch.empty_like(q), lse=lse, scale=0.1, window=20, group_start=i32([0, 2]),
                      workspace=torch.empty(P.paged_prefix_attn_workspace_bytes(q, c, table), dtype=torch.uint8, device="cuda"))
        if form == "stream":
            kw["stream"] = torch.cuda.current_stream()
        if form == "groups":
            kw["group_start"], prefix = i32([0, 1, 2]), i32([16, 5])
        return [P.paged_prefix_attn(q, c, table, *lens, prefix, **kw), lse]
    got, want, taken = both(monkeypatch, call)
    same(got, want)
    assert taken == [True]


@pytest.mark.parametrize("form", ["plain", "numbers", "arrays", "out", "stream", "no workspace"])
def test_marshalling_of_the_draw(monkeypatch, form):
    def call(P):
        torch.manual_seed(2)
        logits, u = torch.randn((4, 999), device="cuda").bfloat16(), torch.rand(4, device="cuda")
        kw, lp = {}, torch.zeros(4, device="cuda")
        if form == "numbers":
            kw = dict(temperature=0.7, top_k=40, top_p=0.9, min_p=0.01)
        if form == "arrays":
            kw = dict(temperature=torch.rand(4, device="cuda"), top_k=i32([1, 0, 5, 2000]), top_p=torch.rand(4, device="cuda"),
                      min_p=torch.zeros(4, device="cuda"))
        if form == "out":
            kw = dict(out=torch.zeros(4, dtype=torch.int32, device="cuda"), logprob=lp)
        if form != "no workspace":
            kw["workspace"] = torch.empty(P.sample_tokens_workspace_bytes(4, 999), dtype=torch.uint8, device="cuda")
        if form == "stream":
            kw["stream"] = torch.cuda.current_stream()
        r = P.sample_tokens(logits, u, **kw)
        assert form != "out" or r is kw["out"]
        return [r, lp]
    got, want, taken = both(monkeypatch, call)
    same(got, want)
    assert taken == [form != "no workspace"]     # a workspace for the call is made in Python


def test_what_the_marshalling_leaves_is_still_checked():
    import paper_2604_17397_amd as P
    c, q, table, (start, lens), prefix = shared(P)
    for kw in (dict(q=q.cpu()), dict(prefix_lens=prefix.cpu()), dict(prefix_lens=prefix.long()), dict(prefix_lens=i32([1, 2])),
               dict(group_start=i32([0])), dict(kv_lens=i32([1]))):
        with pytest.raises(ValueError):
            P.paged_prefix_attn(**{**dict(q=q, cache=c, block_table=table, q_start=start, kv_lens=lens, prefix_lens=prefix), **kw})
    logits, u = torch.zeros((2, 50), device="cuda"), torch.rand(2, device="cuda")
    for kw in (dict(u=u[:1]), dict(u=u.cpu()), dict(top_k=u), dict(logits=logits.double()), dict(temperature=u.half())):
        with pytest.raises(ValueError):
            P.sample_tokens(**{**dict(logits=logits, u=u), **kw})


@pytest.mark.parametrize("name", ["paged_prefix_attn", "sample_tokens"])
@pytest.mark.parametrize("native", [True, False])
def test_given_back_block_of_a_busy_stream(monkeypatch, name, native):
    """As for the other calls that take stream=: their new outputs are not blocks that the current stream still writes to."""
    import paper_2604_17397_amd as P
    c, q, table, lens, prefix = shared(P)
    torch.manual_seed(3)
    logits, u = torch.randn((700, 333), device="cuda"), torch.rand(700, device="cuda")
    call = {"paged_prefix_attn": lambda **kw: P.paged_prefix_attn(q, c, table, *lens, prefix, **kw),
            "sample_tokens": lambda **kw: P.sample_tokens(logits, u, top_k=9, **kw)}[name]
    P.lib()
    if not native:
        monkeypatch.setattr(P.binding, "_NATIVE", P.binding._PythonOnly)
    want = call().clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)
    junk = torch.empty(want.shape, dtype=want.dtype, device="cuda")
    junk.fill_(77)
    given_back = junk.data_ptr()
    del junk
    got = call(stream=side)
    assert got.data_ptr() != given_back
    torch.cuda.synchronize()
    assert torch.equal(got.view(torch.uint8), want.view(torch.uint8))
