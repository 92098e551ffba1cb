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


def rope_desc(b, **kw):
    d = b.sdvg_rope_desc(positions=FAKE, freqs=FAKE, rotary_dim=64, layout=1, gain=1.0)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def rows(b, **kw):
    r = b.sdvg_rows(in_=FAKE, out=FAKE + (1 << 20), n_heads=2, in_token_stride=256, in_head_stride=128, out_token_stride=256,
                    out_head_stride=128)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


ROPE_BAD = [(dict(positions=None), -1), (dict(freqs=None), -1), (dict(rotary_dim=0), -2), (dict(rotary_dim=144), -2),
            (dict(rotary_dim=24), -4), (dict(layout=2), -5), (dict(gain=float("inf")), -3), (dict(gain=float("nan")), -3),
            (dict(positions=FAKE + 2), -4), (dict(freqs=FAKE + 4), -4)]
ROWS_BAD = [(dict(in_=None), -1), (dict(n_heads=0), -2), (dict(in_token_stride=127), -2), (dict(in_token_stride=260), -4),
            (dict(in_head_stride=1 << 41), -5), (dict(in_=FAKE + 8), -4)]
OUT_BAD = [(dict(out=None), -1), (dict(out_head_stride=0), -2), (dict(out_token_stride=132), -4), (dict(out=FAKE + (1 << 20) + 2), -4),
           (dict(out=FAKE, out_token_stride=512), -3)]


def test_rope_positions_rejects_bad_arguments(b):
    ref = ctypes.byref

    def call(rope=None, x=None, y=None, n=4, d=128, dtype=0):
        return b.lib().sdvg_rope_positions(ref(rope or rope_desc(b)), ref(x or rows(b)), y and ref(y), n, d, dtype, None)
    for kw, want in ROPE_BAD:
        assert call(rope=rope_desc(b, **kw)) == want, kw
    for kw, want in ROWS_BAD + OUT_BAD:
        assert call(x=rows(b, **kw)) == want, kw
        assert call(y=rows(b, **kw)) == want, kw
    assert call(n=-1) == -2 and call(d=64) == -5 and call(dtype=3) == -5 and call(dtype=9) == -5 and call(n=1 << 26) == -5 and call(n=(1 << 26) - 3) == -5
    assert call(n=0) == 0 and call(n=0, x=rows(b, in_=None, out=None)) == 0
    assert b.lib().sdvg_rope_positions(None, ref(rows(b)), None, 4, 128, 0, None) == -1
    assert b.lib().sdvg_rope_positions(ref(rope_desc(b)), None, None, 4, 128, 0, None) == -1


def paged_kv(b, **kw):
    c = b.sdvg_paged_kv(k=FAKE << 4, v=FAKE << 5, n_pages=4, page_tokens=8, n_kv_heads=2, head_dim=128,
                        page_stride=8 * 256, token_stride=256, head_stride=128, dtype=0)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


PAGED_BAD = [(dict(k=None), -1), (dict(v=None), -1), (dict(head_dim=64), -5), (dict(dtype=1), -5), (dict(dtype=7), -5),
             (dict(k_scale=FAKE), -5), (dict(n_pages=0), -2), (dict(page_tokens=0), -2), (dict(page_tokens=12), -4),
             (dict(n_kv_heads=0), -2), (dict(n_pages=1 << 28), -5), (dict(k=FAKE + 8), -4), (dict(token_stride=260), -4),
             (dict(token_stride=128), -2), (dict(page_stride=7 * 256), -2), (dict(head_stride=64), -2),
             (dict(head_stride=7 * 128, token_stride=128), -2),          # head-major, a head too short for its tokens
             (dict(dtype=3, k_scale=FAKE + 2), -4)]


def test_paged_commit_rejects_bad_arguments(b):
    ref = ctypes.byref

    def call(c=None, k=None, v=None, slots=FAKE, n=4, dtype=0, rope=None, q=None):
        return b.lib().sdvg_paged_commit(ref(c or paged_kv(b)), ref(k or rows(b)), ref(v or rows(b)), slots, n, dtype,
                                         rope and ref(rope), q and ref(q), None)
    for kw, want in PAGED_BAD:
        assert call(c=paged_kv(b, **kw)) == want, kw
    for kw, want in ROWS_BAD:
        want = -2 if "n_heads" in kw else want
        assert call(k=rows(b, **kw)) == want and call(v=rows(b, **kw)) == want, kw
    for kw, want in ROPE_BAD:
        assert call(rope=rope_desc(b, **kw)) == want, kw
    for kw, want in ROWS_BAD + OUT_BAD:
        assert call(rope=rope_desc(b), q=rows(b, **kw)) == want, kw
    assert call(q=rows(b)) == -1                                        # q without a rotation
    assert call(slots=None) == -1 and call(slots=FAKE + 4) == -4 and call(n=-1) == -2 and call(n=1 << 26) == -5 and call(n=(1 << 26) - 3) == -5
    assert call(dtype=1) == -5 and call(dtype=2) == -5                  # fp32 rows; half rows into a bfloat16 cache
    assert call(k=rows(b, n_heads=3)) == -2
    assert call(v=rows(b, in_=(FAKE << 4) + 4096)) == -3                # v inside the pool of k
    assert call(n=0, slots=None) == 0


def test_paged_binding_checks(b, monkeypatch):
    for name in ("_check_here", "_check_dev"):
        monkeypatch.setattr(b, name, lambda *a: None)
    monkeypatch.setattr(b, "_LIB", type("Trap", (), {"__getattr__": lambda s, n: pytest.fail("the C library must not be reached")})())
    x = torch.zeros((4, 2, 128), dtype=torch.bfloat16)
    pos, freqs = torch.zeros(4, dtype=torch.int32), torch.zeros(32, dtype=torch.float64)
    for kw in [dict(x=x.double()), dict(x=x[..., :64]), dict(x=x[0]), dict(positions=pos[:3]), dict(positions=pos.long()),
               dict(freqs=freqs.float()), dict(layout="both"), dict(out=x[:3]), dict(out=x.half()), dict(y=x[:2]), dict(y=x.half()),
               dict(y_out=x), dict(y=x, y_out=x[:, :1])]:
        with pytest.raises(ValueError):
            b.rope_positions(**{**dict(x=x, positions=pos, freqs=freqs), **kw})
    pool = torch.zeros((3, 8, 2, 128), dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        b.PagedKV(pool.float(), pool.float())
    for args in [(pool, pool[:2]), (pool[0], pool[0]), (pool, pool, torch.ones(2)), (pool.to(torch.float8_e4m3fn),) * 2 + (torch.ones(3),)]:
        with pytest.raises(ValueError):
            b.PagedKV(*args)
    c = b.PagedKV(pool, pool)
    slots = torch.zeros(4, dtype=torch.int64)
    for kw in [dict(k=x[:, :1]), dict(k=x.half(), v=x.half()), dict(v=x[:3]), dict(slots=slots[:2]), dict(slots=slots.int()),
               dict(positions=pos), dict(freqs=freqs), dict(q=x), dict(q_out=x), dict(positions=pos, freqs=freqs, q=x[:2]),
               dict(positions=pos, freqs=freqs, q=x, q_out=x.half())]:
        with pytest.raises(ValueError):
            b.paged_commit(**{**dict(cache=c, k=x, v=x, slots=slots), **kw})


def test_rope_frequencies(b):
    import math
    w, gain = b.rope_frequencies(64, theta=1e4, device="cpu")
    assert w.dtype == torch.float64 and gain == 1.0 and torch.allclose(w, 1e4 ** (-torch.arange(32).double() / 32), rtol=1e-14)
    assert torch.equal(b.rope_frequencies(64, scaling="linear", factor=4, device="cpu")[0], w / 4)
    ntk, _ = b.rope_frequencies(64, scaling="ntk", factor=4, device="cpu")
    assert ntk[0] == w[0] and abs(ntk[-1] / w[-1] * 4 - 1) < 1e-12 and (ntk[1:] < w[1:]).all() and (ntk > w / 4 - 1e-18).all()
    yarn, gain = b.rope_frequencies(64, scaling="yarn", factor=4, original=2048, device="cpu")
    turns = 2048 * w / (2 * math.pi)
    assert torch.equal(yarn[turns >= 32], w[turns >= 32]) and torch.equal(yarn[turns <= 1], w[turns <= 1] / 4)
    mid = (turns > 1) & (turns < 32)
    assert mid.any() and ((yarn < w) & (yarn > w / 4))[mid].all() and abs(gain - (0.1 * math.log(4) + 1)) < 1e-15
    for bad in [dict(rotary_dim=24), dict(rotary_dim=0), dict(rotary_dim=160), dict(rotary_dim=64, theta=0), dict(rotary_dim=64, factor=0.5),
                dict(rotary_dim=64, scaling="other"), dict(rotary_dim=64, scaling="yarn"),
                dict(rotary_dim=64, scaling="yarn", original=100, beta_fast=1, beta_slow=1)]:
        with pytest.raises(ValueError):
            b.rope_frequencies(device="cpu", **bad)


def test_cut_of_paged_attention_on_the_host(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    exe = str(tmp_path / "plan")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-I", os.path.join(root, "paper_2604_17397_amd", "csrc"),
                    os.path.join(root, "tests", "host", "paged_attn_plan.cpp"), "-o", exe], check=True)
    res = subprocess.run([exe], stdout=subprocess.PIPE, text=True, timeout=120)
    assert res.returncode == 0 and res.stdout.strip() == "ok", res.stdout


def attn_desc(b, **kw):
    d = b.sdvg_paged_attn_desc(n_requests=3, n_tokens=5, n_heads=6, head_dim=128, table_width=4, window=0, table_stride=4,
                               q_token_stride=6 * 128, q_head_stride=128, o_token_stride=6 * 128, o_head_stride=128,
                               scale=0.0, dtype=0)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def test_paged_attn_rejects_bad_arguments(b):
    ref = ctypes.byref

    def call(d=None, c=None, q=FAKE, table=FAKE, start=FAKE, lens=FAKE, out=FAKE << 1, lse=None, ws=None, n_ws=0):
        return b.lib().sdvg_paged_attn(ref(d or attn_desc(b)), ref(c or paged_kv(b)), q, table, start, lens, out, lse, ws, n_ws, None)
    for kw, want in PAGED_BAD:
        assert call(c=paged_kv(b, **kw)) == want, kw
    for kw, want in [(dict(head_dim=64), -5), (dict(dtype=1), -5), (dict(dtype=2), -5), (dict(dtype=3), -5), (dict(n_requests=-1), -2),
                     (dict(n_tokens=-1), -2), (dict(n_heads=0), -2), (dict(n_heads=5), -2), (dict(table_width=0), -2),
                     (dict(window=-1), -2), (dict(table_stride=3), -2), (dict(scale=-1.0), -3), (dict(scale=float("nan")), -3),
                     (dict(q_token_stride=100), -2), (dict(q_head_stride=132), -4), (dict(o_token_stride=772), -4),
                     (dict(n_tokens=1 << 29), -5)]:
        assert call(d=attn_desc(b, **kw)) == want, kw
        if "stride" not in next(iter(kw)) or "table" in next(iter(kw)):
            assert b.lib().sdvg_paged_attn_workspace_bytes(ref(attn_desc(b, **kw)), ref(paged_kv(b))) == want, kw
    for kw in (dict(q=None), dict(table=None), dict(start=None), dict(lens=None), dict(out=None)):
        assert call(**kw) == -1
    for kw in (dict(q=FAKE + 8), dict(table=FAKE + 2), dict(start=FAKE + 1), dict(lens=FAKE + 2), dict(out=FAKE + 2), dict(lse=FAKE + 2),
               dict(ws=FAKE + 8, n_ws=1 << 20)):
        assert call(**kw) == -4
    assert call(n_ws=-1) == -2
    assert call(d=attn_desc(b, o_token_stride=1024), out=FAKE) == -3       # in place with other strides
    assert call(d=attn_desc(b, n_requests=0), q=None) == 0 and call(d=attn_desc(b, n_tokens=0), q=None) == 0
    assert b.lib().sdvg_paged_attn_workspace_bytes(ref(attn_desc(b, n_tokens=0)), ref(paged_kv(b))) == 0


def test_paged_attn_binding_checks(b, monkeypatch):
    for name in ("_check_here", "_check_dev"):
        monkeypatch.setattr(b, name, lambda *a: None)
    pool = torch.zeros((3, 8, 2, 128), dtype=torch.bfloat16)
    c = b.PagedKV(pool, pool)
    monkeypatch.setattr(b, "_LIB", type("Trap", (), {"__getattr__": lambda s, n: pytest.fail("the C library must not be reached")})())
    q = torch.zeros((4, 6, 128), dtype=torch.bfloat16)
    n = torch.zeros(2, dtype=torch.int32)
    ok = dict(q=q, cache=c, block_table=torch.zeros((2, 3), dtype=torch.int32), q_start=torch.zeros(3, dtype=torch.int32), kv_lens=n)
    for kw in [dict(q=q.half()), dict(q=q.float()), dict(q=q[0]), dict(block_table=n), dict(block_table=ok["block_table"].long()),
               dict(block_table=torch.zeros((3, 2), dtype=torch.int32).t()), dict(q_start=n), dict(kv_lens=n[:1]), dict(kv_lens=n.long()),
               dict(out=q[:3]), dict(out=q.half()), dict(lse=torch.zeros((4, 6), dtype=torch.float64)), dict(lse=torch.zeros((4, 5))),
               dict(lse=torch.zeros((6, 4)).t()), dict(workspace=torch.zeros((8, 8)).t())]:
        with pytest.raises(ValueError):
            b.paged_attn(**{**ok, **kw})
