"""The shared-prefix attention's refusals and its cut into workgroups, on the host (no GPU needed)."""
import ctypes
import os
import subprocess

import pytest
import torch

from test_paged_abi import FAKE, PAGED_BAD, attn_desc, b, paged_kv  # noqa: F401 (b is a fixture)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_pair_of_tiles_is_one_items(tmp_path):
    exe = str(tmp_path / "items")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-D_GLIBCXX_ASSERTIONS", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                    "-I", os.path.join(ROOT, "paper_2604_17397_amd", "csrc"), os.path.join(ROOT, "tests", "host", "paged_prefix_items.cpp"),
                    "-o", exe], check=True)
    res = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert res.returncode == 0 and res.stdout.strip() == "ok", res.stdout


def test_bad_arguments(b):  # noqa: F811
    ref = ctypes.byref

    def call(d=None, c=None, q=FAKE, table=FAKE, start=FAKE, lens=FAKE, n=1, groups=FAKE, prefix=FAKE, out=FAKE << 1, lse=None, ws=None, n_ws=0):
        return b.lib().sdvg_paged_prefix_attn(ref(d or attn_desc(b)), ref(c or paged_kv(b)), q, table, start, lens, n, groups, prefix, out,
                                              lse, ws, n_ws, None)

    def need(d=None, c=None, n=1):
        return b.lib().sdvg_paged_prefix_attn_workspace_bytes(ref(d or attn_desc(b)), ref(c or paged_kv(b)), n)
    for kw, want in PAGED_BAD:
        assert call(c=paged_kv(b, **kw)) == want and need(c=paged_kv(b, **kw)) == want, kw
    for kw, want in [(dict(head_dim=64), -5), (dict(dtype=1), -5), (dict(dtype=3), -5), (dict(n_requests=-1), -2), (dict(n_heads=5), -2),
                     (dict(table_width=0), -2), (dict(window=-1), -2), (dict(table_stride=3), -2), (dict(scale=float("nan")), -3),
                     (dict(n_tokens=1 << 29), -5)]:
        assert call(d=attn_desc(b, **kw)) == want and need(d=attn_desc(b, **kw)) == want, kw
    for kw in (dict(q=None), dict(table=None), dict(start=None), dict(lens=None), dict(out=None), dict(prefix=None), dict(n=2, groups=None)):
        assert call(**kw) == -1, kw
    for kw in (dict(q=FAKE + 8), dict(table=FAKE + 2), dict(start=FAKE + 1), dict(lens=FAKE + 2), dict(out=FAKE + 2), dict(lse=FAKE + 2),
               dict(ws=FAKE + 8, n_ws=1 << 20), dict(groups=FAKE + 2), dict(prefix=FAKE + 1)):
        assert call(**kw) == -4, kw
    assert call(n_ws=-1) == -2 and call(n=-1) == -2 and need(n=-1) == -2
    assert call(d=attn_desc(b, o_token_stride=1024), out=FAKE) == -3       # in place with other strides
    assert call(d=attn_desc(b, n_requests=0), q=None) == 0 and call(d=attn_desc(b, n_tokens=0), q=None) == 0
    assert need(d=attn_desc(b, n_tokens=0)) == 0


def test_binding_checks(b, monkeypatch):  # noqa: F811
    for name in ("_check_here", "_check_dev"):
        monkeypatch.setattr(b, name, lambda *a: None)
    pool = torch.zeros((3, 8, 2, 128), dtype=torch.bfloat16)
    c = b.PagedKV(pool, pool)
    monkeypatch.setattr(b, "_LIB", type("Trap", (), {"__getattr__": lambda s, n: pytest.fail("the C library must not be reached")})())
    q = torch.zeros((4, 6, 128), dtype=torch.bfloat16)
    n = torch.zeros(2, dtype=torch.int32)
    ok = dict(q=q, cache=c, block_table=torch.zeros((2, 3), dtype=torch.int32), q_start=torch.zeros(3, dtype=torch.int32), kv_lens=n,
              prefix_lens=n, group_start=torch.zeros(3, dtype=torch.int32))
    for kw in [dict(q=q.half()), dict(q=q[0]), dict(block_table=n), dict(q_start=n), dict(kv_lens=n[:1]), dict(out=q[:3]),
               dict(lse=torch.zeros((4, 5))), dict(workspace=torch.zeros((8, 8)).t()), dict(prefix_lens=n.long()), dict(prefix_lens=n[None]),
               dict(prefix_lens=n[:1]), dict(group_start=n), dict(group_start=None), dict(group_start=ok["group_start"].long()),
               dict(prefix_lens=torch.zeros(4, dtype=torch.int32)[::2])]:
        with pytest.raises(ValueError):
            b.paged_prefix_attn(**{**ok, **kw})
    with pytest.raises(ValueError, match="32 bits"):
        b.paged_prefix_attn_workspace_bytes(q, c, ok["block_table"], 1 << 40)


def test_kernels_do_not_spill():
    from test_kernel_resources import test_paged_kernels_do_not_spill as check
    check("paged_prefix.hip", ("paged_prefix_kernel", "paged_prefix_join_kernel"))
