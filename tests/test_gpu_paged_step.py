"""Plan, commit and attention together, as a program that drafts and verifies tokens uses them: the pages a request holds
at the end give the same attention as its tokens in one piece, whatever was rejected on the way."""
import math

import numpy as np
import pytest
import torch

from paged_util import i32

pytestmark = pytest.mark.gpu
H, HK, P_, THETA = 6, 2, 16, 1e4


def rows(seed, n, heads):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.randn((n, heads, 128), generator=gen, device="cuda").bfloat16()


def attention(q, k, v, first, freqs, window):
    """Tokens `first` .. of one request, q [new, H, 128] against k, v [len, HK, 128], rotated here in 64 bits."""
    def turn(x, pos):
        x = x.double()
        a, b = x[..., :64], x[..., 64:]
        ang = (pos.double()[:, None] * freqs)[:, None, :]
        return torch.cat([a * torch.cos(ang) - b * torch.sin(ang), a * torch.sin(ang) + b * torch.cos(ang)], -1).bfloat16().double()
    n = k.shape[0]
    j = torch.arange(n, device="cuda")
    i = torch.arange(first, first + q.shape[0], device="cuda")
    qr, kr = turn(q, i), turn(k, j)
    ok = j[None] <= i[:, None]
    if window:
        ok &= j[None] > i[:, None] - window
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    for h in range(H):
        s = qr[:, h] @ kr[:, h // (H // HK)].t().contiguous() / math.sqrt(128)
        out[:, h] = torch.softmax(torch.where(ok, s, -math.inf), 1) @ v[:, h // (H // HK)].double()
    return out


@pytest.mark.parametrize("window", [0, 70])
@pytest.mark.parametrize("captured", [False, True])
def test_draft_verify_reject(window, captured):
    import paper_2604_17397_amd as P
    R, most, steps = 5, 6, 7
    rng = np.random.default_rng(3)
    freqs, _ = P.rope_frequencies(128, theta=THETA)
    pages = 60
    shape = (pages, P_, HK, 128)
    kc, vc = (torch.full(shape, float("nan"), device="cuda", dtype=torch.bfloat16) for _ in range(2))
    cache = P.PagedKV(kc, vc)
    table = torch.full((R, 12), -1, dtype=torch.int32, device="cuda")
    free = i32(rng.permutation(pages))
    cached, held, cursor, new = i32([0] * R), i32([0] * R), i32([0]), i32([0] * R)
    room = 200
    plan = P.PagePlan(R, room)
    q, k, v = rows(0, room, H), rows(0, room, HK), rows(0, room, HK)
    out = torch.zeros_like(q)
    h = P.PagedKV(kc, vc)
    ws = torch.empty(P.paged_attn_workspace_bytes(q, h, table), dtype=torch.uint8, device="cuda")

    def step():
        P.page_plan(cached, new, table, P_, free_pages=free, held=held, next_free=cursor, out=plan)
        qr = P.paged_commit(cache, k, v, plan.slots, positions=plan.positions, freqs=freqs, q=q)
        P.paged_attn(qr, cache, table, plan.q_start, plan.kv_lens, out=out, window=window, workspace=ws)
        held.copy_(plan.held)
        cursor.copy_(plan.next_free)
    graph = None
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    history = [[torch.empty((0, n, 128), dtype=torch.bfloat16, device="cuda") for n in (HK, HK)] for _ in range(R)]
    lens = [0] * R
    with torch.cuda.stream(side):
        if captured:
            step()      # nothing to do: no new token
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                step()
        for s in range(steps):
            # a prompt first, then drafts of a few tokens of which some are taken back afterwards
            n = [int(x) for x in (rng.integers(1, 41, R) if s == 0 else rng.integers(0, most + 1, R))]
            new.copy_(i32(n))
            total = sum(n)
            q.copy_(rows(10 * s + 1, room, H))
            k.copy_(rows(10 * s + 2, room, HK))
            v.copy_(rows(10 * s + 3, room, HK))
            out.fill_(5.0)
            torch.cuda.synchronize()
            graph.replay() if captured else step()
            torch.cuda.synchronize()
            assert (out[total:] == 5).all() and plan.q_start[-1].item() == total
            at = 0
            for r in range(R):
                kk = torch.cat([history[r][0], k[at:at + n[r]]])
                vv = torch.cat([history[r][1], v[at:at + n[r]]])
                want = attention(q[at:at + n[r]], kk, vv, lens[r], freqs, window)
                # as in the attention's own tests, and the rotated rows are rounded to bf16 (a step apart where the
                # angle's last bits decide): bounded by the bf16 bounds of the framework's attention
                err = (out[at:at + n[r]].double() - want).abs()
                assert n[r] == 0 or err.max().item() <= 2e-2, (s, r, err.max().item())
                kept = n[r] if s == 0 else int(rng.integers(0, n[r] + 1))       # tokens of the draft that are accepted
                history[r] = [kk[:lens[r] + kept], vv[:lens[r] + kept]]
                lens[r] += kept
                at += n[r]
            cached.copy_(i32(lens))     # undoing the rest needs nothing else
    assert cursor.item() == held.sum().item() <= pages
