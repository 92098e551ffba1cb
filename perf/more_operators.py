"""Many continuations of one prompt, as cases that can be timed: attention of a batch whose requests share a long
prefix in the paged cache, which is read once for all of them, and sampling of the next tokens from logits with
temperature, top-k, top-p and min-p and given random numbers.

A case is one pass through one operator. Head layouts are those of the other cases: 12 heads (drafter), 40 heads (target), groups
of query heads that share a key head; 128 dims; a block has 4680 tokens. Where `own` is true the operators are the package's,
otherwise their plain form.
"""
import math
import random

import numpy
import torch

own = False

D = 128                      # head_dim
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}
BYTES = {"bf16": 2, "f16": 2, "f32": 4, "e4m3": 1}


def listed():
    return [
        # four candidates of the drafter behind one short prompt: latency counts
        {"name": "prefix_few", "kind": "prefix", "requests": 4, "groups": 1, "prefix": 936, "longest": 40, "new": 1, "heads": 12,
         "kv_heads": 12, "page": 16, "type": "bf16", "cache": "bf16", "window": 0},
        # candidates for the next block behind 7 blocks: one row per head and candidate, bound by the cache's memory
        {"name": "prefix_candidates", "kind": "prefix", "requests": 16, "groups": 1, "prefix": 32760, "longest": 1000, "new": 1,
         "heads": 40, "kv_heads": 8, "page": 64, "type": "bf16", "cache": "bf16", "window": 0},
        # a serving step: many requests with one system prompt, answers of all lengths
        {"name": "prefix_serving", "kind": "prefix", "requests": 128, "groups": 1, "prefix": 8191, "longest": 2000, "new": 1,
         "heads": 32, "kv_heads": 8, "page": 16, "type": "f16", "cache": "f16", "window": 0},
        # verification of up to 8 drafted tokens per request over a cache of 8 bits
        {"name": "prefix_verify", "kind": "prefix", "requests": 24, "groups": 1, "prefix": 16384, "longest": 700, "new": 8, "heads": 40,
         "kv_heads": 8, "page": 64, "type": "bf16", "cache": "e4m3", "window": 0},
        # several prompts at once, each with its own continuations, prompts of unlike lengths, a head for every query head, a rolling window
        {"name": "prefix_groups", "kind": "prefix", "requests": 42, "groups": 6, "prefix": 14040, "longest": 333, "new": 3, "heads": 12,
         "kv_heads": 12, "page": 24, "type": "bf16", "cache": "bf16", "window": 9000},
        # the longest prompt, 14 blocks, with many candidates: bound by the matrix cores
        {"name": "prefix_long", "kind": "prefix", "requests": 64, "groups": 1, "prefix": 65520, "longest": 500, "new": 1, "heads": 40,
         "kv_heads": 8, "page": 64, "type": "bf16", "cache": "bf16", "window": 0},
        # one request's next token, all filters: latency counts
        {"name": "sample_one", "kind": "sample", "rows": 1, "vocab": 32000, "type": "bf16", "filters": "all", "masked": 0.0},
        # one request's next token from a large vocabulary in 32 bits
        {"name": "sample_large", "kind": "sample", "rows": 1, "vocab": 262144, "type": "f32", "filters": "all", "masked": 0.0},
        # a serving step: every request has its own settings, some are greedy, some have filters, some have none
        {"name": "sample_serving", "kind": "sample", "rows": 128, "vocab": 131072, "type": "bf16", "filters": "mixed", "masked": 0.0},
        # candidates drawn without filters
        {"name": "sample_open", "kind": "sample", "rows": 64, "vocab": 131072, "type": "f32", "filters": "none", "masked": 0.0},
        # drafted tokens of many requests, an odd vocabulary, most of it ruled out by a grammar
        {"name": "sample_masked", "kind": "sample", "rows": 200, "vocab": 150001, "type": "f16", "filters": "top_p", "masked": 0.7},
        # a small vocabulary, many rows
        {"name": "sample_many", "kind": "sample", "rows": 777, "vocab": 32768, "type": "f32", "filters": "mixed", "masked": 0.1},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    if rng.random() < 0.5:
        vocab = _log_int(rng, 1000, 262144)
        return {"kind": "sample", "rows": _log_int(rng, 1, min(777, 30000000 // vocab)), "vocab": vocab,
                "type": rng.choice(["bf16", "f16", "f32"]), "filters": rng.choice(["all", "mixed", "none", "top_k", "top_p", "min_p"]),
                "masked": rng.choice([0.0, 0.0, 0.1, 0.7, 0.99])}
    kv_heads = rng.choice([1, 2, 3, 4, 5, 8, 12, 16])
    group = rng.choice([1, 1, 2, 3, 4, 5, 7, 8, 16])
    kind16 = rng.choice(["bf16", "f16"])
    requests, new = _log_int(rng, 1, 128), rng.choice([1, 1, 1, 2, 4, 8])
    groups = rng.choice([1, 1, _log_int(rng, 1, min(8, requests))])
    # no more work than the largest listed case, in attention and in memory
    most = min(65520, 64 * 40 * 65520 // (2 * requests * new * kv_heads * group), 8 * 65520 // (kv_heads * groups))
    return {"kind": "prefix", "requests": requests, "groups": groups, "prefix": _log_int(rng, 1, most),
            "longest": _log_int(rng, new, 2000), "new": new, "heads": kv_heads * group, "kv_heads": kv_heads,
            "page": rng.choice([8, 16, 24, 32, 64, 128, 256]), "type": kind16, "cache": rng.choice([kind16, kind16, "e4m3"]),
            "window": rng.choice([0, 0, 0, _log_int(rng, 16, 16384)])}


# ---------------------------------------------------------------------------- inputs

def _requests(case):
    """Of the groups: first request, keys of the prefix; of the requests: own keys behind the prefix, new tokens. Part of the
    case, the same for every seed."""
    rng = random.Random(case["requests"] * 1000003 + case["prefix"])
    R, G = case["requests"], case["groups"]
    cuts = sorted(rng.sample(range(1, R), G - 1))
    start = [0] + cuts + [R]
    prefix = [case["prefix"] if g == G // 2 else _log_int(rng, max(1, case["prefix"] // 16), case["prefix"]) for g in range(G)]
    new = [case["new"] if r == R // 2 else rng.randint(1, case["new"]) for r in range(R)]
    own_keys = [case["longest"] if r == R // 2 else _log_int(rng, new[r], case["longest"]) for r in range(R)]
    return start, prefix, own_keys, new


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def _prepare_prefix(case, gen, st):
    start, prefix, own_keys, new = _requests(case)
    P, H, R = case["page"], case["kv_heads"], case["requests"]
    t, cache = TYPES[case["type"]], TYPES[case["cache"]]
    of = [g for g in range(case["groups"]) for _ in range(start[g], start[g + 1])]
    lens = [prefix[of[r]] + own_keys[r] for r in range(R)]
    # whole pages of a prefix are shared; a request has pages of its own from the first one that it writes to
    shared = [n // P for n in prefix]
    used = [-(-n // P) for n in lens]
    total = sum(shared) + sum(used[r] - shared[of[r]] for r in range(R)) + 1
    ids = torch.randperm(total, generator=gen, device="cuda").int()
    table = torch.full((R, max(used)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for g in range(case["groups"]):
        table[start[g]:start[g + 1], :shared[g]] = ids[at:at + shared[g]]
        at += shared[g]
    for r in range(R):
        n = used[r] - shared[of[r]]
        table[r, shared[of[r]]:used[r]] = ids[at:at + n]
        at += n
    for name in ("kc", "vc"):
        x = torch.randn((total, P, H, D), generator=gen, device="cuda", dtype=torch.bfloat16)
        x = (x * 48).to(cache) if case["cache"] == "e4m3" else x.to(cache)
        # where a prefix ends inside a page, every request has a copy of that page's part of it
        raw = x.view(torch.uint8)
        for g in range(case["groups"]):
            if prefix[g] % P and start[g + 1] - start[g] > 1:
                pages = table[start[g]:start[g + 1], shared[g]].long()
                raw[pages[1:], :prefix[g] % P] = raw[pages[:1], :prefix[g] % P]
        st[name] = x
    for name in ("k_scale", "v_scale"):
        st[name] = (0.5 + torch.rand(H, generator=gen, device="cuda")) / 64 if case["cache"] == "e4m3" else None
    q_start = [0]
    for n in new:
        q_start.append(q_start[-1] + n)
    st.update(table=table, q_start=_ints(q_start), kv_lens=_ints(lens), prefix_lens=_ints(prefix), group_start=_ints(start),
              q=torch.randn((q_start[-1], case["heads"], D), generator=gen, device="cuda").to(t), scale=1 / math.sqrt(D))
    if own:
        import paper_2604_17397_amd as package
        st["handle"] = package.PagedKV(st["kc"], st["vc"], st["k_scale"], st["v_scale"])
        n = package.paged_prefix_attn_workspace_bytes(st["q"], st["handle"], table, case["groups"])
        st["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")


def _prepare_sample(case, gen, st):
    n, V = case["rows"], case["vocab"]
    # probabilities that fall with the rank as words' do, and what a context does to them
    u = torch.rand((n, V), generator=gen, device="cuda")
    steep = 0.9 + 0.9 * torch.rand((n, 1), generator=gen, device="cuda")
    x = -steep * torch.log1p(u * V) + 0.5 * torch.randn((n, V), generator=gen, device="cuda") + 12.0
    if case["masked"]:
        gone = torch.rand((n, V), generator=gen, device="cuda") < case["masked"]
        gone[:, V // 3] = False                              # something is always allowed
        x = x.masked_fill_(gone, -math.inf)
    x[:, V - V // 500:] = -math.inf                          # the vocabulary's padding
    st["logits"] = x.to(TYPES[case["type"]])
    st["u"] = torch.rand(n, generator=gen, device="cuda")

    def some(low, high):
        return low + (high - low) * torch.rand(n, generator=gen, device="cuda")
    kind = torch.arange(n, device="cuda") % 6
    f = case["filters"]
    st["temperature"] = some(0.5, 1.5)
    st["top_k"] = st["top_p"] = st["min_p"] = None
    if f in ("all", "top_k"):
        st["top_k"] = torch.randint(1, min(1000, V), (n,), generator=gen, device="cuda", dtype=torch.int32)
    if f in ("all", "top_p"):
        st["top_p"] = some(0.5, 0.99)
    if f in ("all", "min_p"):
        st["min_p"] = some(0.0005, 0.05)
    if f == "mixed":
        st["temperature"] = torch.where(kind == 0, 0.0, st["temperature"])
        st["top_k"] = torch.where((kind == 1) | (kind == 2), torch.randint(1, min(200, V), (n,), generator=gen, device="cuda"), 0).int()
        st["top_p"] = torch.where((kind == 2) | (kind == 3), some(0.8, 0.99), 1.0)
        st["min_p"] = torch.where(kind == 4, some(0.01, 0.1), 0.0)
    if own:
        import paper_2604_17397_amd as package
        st["workspace"] = torch.empty(package.sample_tokens_workspace_bytes(n, V), dtype=torch.uint8, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    st = {"case": case}
    (_prepare_prefix if case["kind"] == "prefix" else _prepare_sample)(case, gen, st)
    return st


# ---------------------------------------------------------------------------- plain forms

def _gathered(cache, table, first, keys, scale):
    """Keys first .. first + keys - 1 (first: one number per row of the table): [rows, kv_heads, keys, 128] in 32 bits."""
    P = cache.shape[1]
    at = first[:, None] + torch.arange(keys, device="cuda")
    page = torch.gather(table, 1, (at // P).clamp(max=table.shape[1] - 1)).clamp(min=0).long()
    x = cache.view(torch.uint8)[page, at % P].view(cache.dtype).float()
    return (x if scale is None else x * scale[:, None]).transpose(1, 2).contiguous()


def _prefix_plain(st):
    case, q, table = st["case"], st["q"], st["table"]
    start, prefix, own_keys, new = _requests(case)
    Hk, most, window = case["kv_heads"], case["new"], case["window"] or 1 << 30
    group = case["heads"] // Hk
    outs, lses = [], []
    i = torch.arange(most, device="cuda")
    for g, L in enumerate(prefix):
        a, b = start[g], start[g + 1]
        R, n = b - a, max(own_keys[a:b])
        counts = st["q_start"][a + 1:b + 1] - st["q_start"][a:b]
        token = (st["q_start"][a:b, None] + i).clamp(max=q.shape[0] - 1)
        x = q[token].float().view(R, most, Hk, group, D).permute(2, 0, 1, 3, 4)        # [Hk, R, most, group, D]
        sees = (st["kv_lens"][a:b] - counts)[:, None] + i + 1                          # keys before this one
        # the prefix, once for all rows
        zero = torch.zeros(1, dtype=torch.int64, device="cuda")
        kp, vp = (_gathered(st[c + "c"], table[a:a + 1], zero, L, st[c + "_scale"])[0] for c in "kv")
        sp = torch.matmul(x.reshape(Hk, -1, D), kp.transpose(1, 2).contiguous()).view(Hk, R, most, group, L).mul_(st["scale"])
        if case["window"]:
            sp.masked_fill_((torch.arange(L, device="cuda") < sees[..., None] - window)[None, :, :, None], -math.inf)
        # every request's own keys
        first = torch.full((R,), L, dtype=torch.int64, device="cuda")
        ko, vo = (_gathered(st[c + "c"], table[a:b], first, n, st[c + "_scale"]) for c in "kv")
        y = x.permute(1, 0, 2, 3, 4).reshape(R, Hk, most * group, D)
        so = torch.matmul(y, ko.transpose(2, 3).contiguous()).view(R, Hk, most, group, n).mul_(st["scale"])
        key = L + torch.arange(n, device="cuda")
        seen = (key < sees[..., None]) & (key >= sees[..., None] - window)
        so = so.masked_fill(~seen[:, None, :, None], -math.inf).permute(1, 0, 2, 3, 4)
        top = torch.maximum(sp.amax(-1, keepdim=True), so.amax(-1, keepdim=True))
        pp, po = torch.exp(sp.sub_(top)), torch.exp(so - top)
        total = pp.sum(-1, keepdim=True) + po.sum(-1, keepdim=True)
        o = torch.matmul(pp.reshape(Hk, -1, L), vp).view(Hk, R, most, group, D)
        mine = torch.matmul(po.permute(1, 0, 2, 3, 4).reshape(R, Hk, most * group, n), vo).view(R, Hk, most, group, D)
        o = (o + mine.permute(1, 0, 2, 3, 4)) / total
        kept = i < counts[:, None]
        outs.append(o.permute(1, 2, 0, 3, 4).reshape(R, most, -1, D)[kept])
        lses.append((top + torch.log(total)).permute(1, 2, 0, 3, 4).reshape(R, most, -1)[kept])
    return [torch.cat(outs).to(q.dtype), torch.cat(lses)]


def _sample_plain(st):
    x, V = st["logits"].double(), st["logits"].shape[1]
    t = st["temperature"].double()[:, None]
    top, best = x.max(1, keepdim=True)
    best = torch.where(x == top, torch.arange(V, device="cuda"), V).amin(1)
    order, index = torch.sort(x, dim=1, descending=True, stable=True)     # ties: the lowest index first
    w = torch.exp((order - top) / torch.where(t > 0, t, 1.0))
    place = torch.arange(V, device="cuda")
    keep = torch.ones_like(w, dtype=torch.bool)
    if st["top_k"] is not None:
        k = st["top_k"][:, None]
        keep &= (place < k) | (k <= 0)
    if st["top_p"] is not None:
        p = st["top_p"].double()[:, None]
        some = torch.where(keep, w, 0.0)
        before = some.cumsum(1) - some
        keep &= (before < p * some.sum(1, keepdim=True)) | (p >= 1)
    if st["min_p"] is not None:
        keep &= w >= st["min_p"].double()[:, None]
    kept = torch.zeros_like(w).scatter_(1, index, torch.where(keep, w, 0.0))
    upto = kept.cumsum(1)
    total = upto[:, -1:]
    drawn = (upto <= st["u"].double()[:, None] * total).sum(1).clamp(max=V - 1)
    token = torch.where(t[:, 0] > 0, drawn, best)
    logprob = torch.log(kept.gather(1, drawn[:, None]) / total)[:, 0]
    return [token.int(), torch.where(t[:, 0] > 0, logprob, 0.0).float()]


# ---------------------------------------------------------------------------- one pass

def run(st):
    case = st["case"]
    if not own:
        return (_prefix_plain if case["kind"] == "prefix" else _sample_plain)(st)
    import paper_2604_17397_amd as package
    if case["kind"] == "prefix":
        lse = torch.empty(st["q"].shape[:2], dtype=torch.float32, device="cuda")
        out = package.paged_prefix_attn(st["q"], st["handle"], st["table"], st["q_start"], st["kv_lens"], st["prefix_lens"],
                                        group_start=st["group_start"], lse=lse, scale=st["scale"], window=case["window"],
                                        workspace=st["workspace"])
        return [out, lse]
    logprob = torch.empty(case["rows"], dtype=torch.float32, device="cuda")
    token = package.sample_tokens(st["logits"], st["u"], temperature=st["temperature"], top_k=st["top_k"], top_p=st["top_p"],
                                  min_p=st["min_p"], logprob=logprob, workspace=st["workspace"])
    return [token, logprob]


# ---------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    if case["kind"] == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * BYTES[case["type"]] + 28 * case["rows"], "flops": 2.0 * n}
    start, prefix, own_keys, new = _requests(case)
    window = case["window"] or 1 << 30
    keys, seen = 0, 0
    for g, L in enumerate(prefix):
        first = L                                              # of the prefix keys that any row sees
        for r in range(start[g], start[g + 1]):
            last = L + own_keys[r]
            lo = max(0, last - new[r] + 1 - window)
            first = min(first, lo)
            keys += last - max(lo, L)
            seen += sum(min(last - j, window) for j in range(new[r]))
        keys += L - first
    return {"bytes": 2 * keys * case["kv_heads"] * D * BYTES[case["cache"]] + 2 * sum(new) * case["heads"] * D * BYTES[case["type"]]
            + 4 * sum(new) * case["heads"] + 4 * keys // case["page"],
            "flops": 4.0 * seen * case["heads"] * D}


# ---------------------------------------------------------------------------- the same in 64 bits

def _exact_sample(case, st):
    """Log-probability of the drawn token, row by row on the host. Tokens are whole numbers and have no other value."""
    x, u = st["logits"].double().cpu().numpy(), st["u"].double().cpu().numpy()

    def of(name, off):
        return [off] * len(u) if st[name] is None else st[name].double().cpu().numpy()
    out = numpy.zeros(len(u))
    for r, (t, k, p, m) in enumerate(zip(of("temperature", 1.0), of("top_k", 0), of("top_p", 1.0), of("min_p", 0.0))):
        if t == 0:
            continue
        there = numpy.flatnonzero(x[r] > -numpy.inf)
        order = there[numpy.argsort(-x[r][there], kind="stable")]
        w = numpy.exp((x[r][order] - x[r][order[0]]) / t)
        if k > 0:
            order, w = order[:int(k)], w[:int(k)]
        if p < 1:
            n = int(numpy.searchsorted(numpy.cumsum(w), p * w.sum())) + 1
            order, w = order[:n], w[:n]
        n = int((w >= m).sum())
        order, w = order[:n], w[:n]
        by_index = numpy.argsort(order)
        total = math.fsum(w)
        at = int(numpy.searchsorted(numpy.cumsum(w[by_index]), u[r] * total, side="right"))
        out[r] = math.log(w[by_index[min(at, n - 1)]] / total)
    return [None, torch.from_numpy(out).cuda()]


def exact(case, seed):
    """What `run` returns, in 64 bits."""
    st = prepare(case, seed)
    if case["kind"] == "sample":
        return _exact_sample(case, st)
    start, prefix, own_keys, new = _requests(case)
    q, group = st["q"], case["heads"] // case["kv_heads"]
    out = torch.empty(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(q.shape[:2], dtype=torch.float64, device="cuda")
    ks, vs = (torch.ones(case["kv_heads"]) if st[a] is None else st[a].cpu() for a in ("k_scale", "v_scale"))
    t, lens = 0, st["kv_lens"].tolist()
    for r, (n, length) in enumerate(zip(new, lens)):
        pages = st["table"][r, :-(-length // case["page"])].long()
        first = max(0, length - n + 1 - case["window"]) if case["window"] else 0
        j = torch.arange(first, length, device="cuda")
        sees = torch.arange(length - n + 1, length + 1, device="cuda")[:, None]
        gone = j >= sees
        if case["window"]:
            gone |= j < sees - case["window"]
        for h in range(case["kv_heads"]):
            k, v = (st[a][:, :, h].contiguous().view(torch.uint8)[pages].view(st[a].dtype).flatten(0, 1)[first:length].double()
                    for a in ("kc", "vc"))
            x = q[t:t + n, h * group:(h + 1) * group].double().transpose(0, 1)      # [group, n, 128]
            s = (x.reshape(-1, D) @ k.t()).view(group, n, -1) * (st["scale"] * float(ks[h]))
            s = s.masked_fill(gone, -math.inf)
            lse[t:t + n, h * group:(h + 1) * group] = torch.logsumexp(s, -1).t()
            o = torch.softmax(s, -1).view(group * n, -1) @ v
            out[t:t + n, h * group:(h + 1) * group] = o.view(group, n, D).transpose(0, 1) * float(vs[h])
        t += n
    return [out, lse]
