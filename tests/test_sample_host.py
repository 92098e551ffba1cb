"""Refusals of sdvg_sample_tokens, its definition in plain form against the library's sums, on the host (no GPU needed)."""
import ctypes
import math

import numpy as np
import pytest
import torch

from sample_util import draw
from test_paged_abi import FAKE, b  # noqa: F401 (b is a fixture)


def args(b, **kw):  # noqa: F811
    a = b.sdvg_sample_args(logits=FAKE << 4, u=FAKE, temperature=FAKE + 0x1000, top_k=FAKE + 0x2000, top_p=FAKE + 0x3000, min_p=FAKE + 0x4000,
                           all_temperature=1.0, all_top_p=1.0, tokens=FAKE + 0x5000, logprob=FAKE + 0x6000, row_stride=1000, n_rows=4,
                           vocab=1000, dtype=0)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def test_bad_arguments(b):  # noqa: F811
    need = b.lib().sdvg_sample_tokens_workspace_bytes

    def call(a=None, ws=FAKE << 5, n=1 << 40, **kw):
        return b.lib().sdvg_sample_tokens(ctypes.byref(a or args(b, **kw)), ws, n, None)
    assert b.lib().sdvg_sample_tokens(None, FAKE, 1 << 40, None) == -1
    for kw, want in [(dict(n_rows=-1), -2), (dict(vocab=0), -2), (dict(vocab=(1 << 20) + 1), -5), (dict(n_rows=1 << 23), -5), (dict(dtype=3), -5),
                     (dict(dtype=9), -5), (dict(row_stride=999), -2), (dict(row_stride=1 << 40), -5), (dict(logits=None), -1), (dict(u=None), -1),
                     (dict(tokens=None), -1), (dict(logits=(FAKE << 4) + 1), -4), (dict(logits=(FAKE << 4) + 2, dtype=1), -4),
                     (dict(u=FAKE + 2), -4), (dict(temperature=FAKE + 1), -4), (dict(top_k=FAKE + 2), -4), (dict(top_p=FAKE + 3), -4),
                     (dict(min_p=FAKE + 2), -4), (dict(tokens=FAKE + 2), -4), (dict(logprob=FAKE + 2), -4), (dict(tokens=FAKE), -3),
                     (dict(logprob=FAKE + 4), -3), (dict(logprob=FAKE + 0x5008), -3), (dict(tokens=(FAKE << 4) + 4000), -3),
                     (dict(tokens=FAKE + 0x3004), -3)]:
        assert call(**kw) == want, kw
    assert call(ws=None) == -1 and call(ws=(FAKE << 5) + 8) == -4 and call(n=-1) == -2 and call(n=need(4, 1000) - 1) == -3
    assert call(n_rows=0, logits=None, tokens=None) == 0
    assert need(-1, 5) == -2 and need(3, 0) == -2 and need(3, (1 << 20) + 1) == -5 and need(0, 5) == 0 and need(1, 1) > 0
    assert need(1 << 20, 1 << 20) == -5


def test_workspace_grows_with_the_rows_and_holds_every_slice(b):  # noqa: F811
    need = b.lib().sdvg_sample_tokens_workspace_bytes
    for vocab in (1, 1000, 32000, 262144, 1 << 20):
        for rows in (1, 2, 7, 64, 500, 777):
            n = need(rows, vocab)
            # a record, three histograms of 256 numbers and a list of 1024 tokens for every slice of at most 8192 tokens, and a row's own histogram
            assert n >= rows * (-(-vocab // 8192) * (3 * 256 * 8 + 32 + 1024 * 8) + 256 * 12)


def test_binding_checks(b, monkeypatch):  # noqa: F811
    for name in ("_check_here", "_check_dev"):
        monkeypatch.setattr(b, name, lambda *a: None)
    need = b.lib().sdvg_sample_tokens_workspace_bytes(3, 10)
    monkeypatch.setattr(b, "_LIB", type("Trap", (), {"__getattr__": lambda s, n: pytest.fail("the C library must not be reached")})())
    f, k = torch.zeros(3), torch.zeros(3, dtype=torch.int32)
    ok = dict(logits=torch.zeros((3, 10)), u=f, workspace=torch.zeros(need, dtype=torch.uint8))
    for kw in [dict(logits=torch.zeros((3, 10)).double()), dict(logits=f), dict(logits=torch.zeros((10, 3)).t()), dict(u=f[:2]), dict(u=f.double()),
               dict(temperature=f[:2]), dict(temperature=f.half()), dict(top_k=f), dict(top_k=k[:1]), dict(top_k=1 << 40), dict(top_p=k),
               dict(min_p=torch.zeros(6)[::2]), dict(out=f), dict(out=k[:2]), dict(logprob=k), dict(logprob=f[:2]), dict(workspace=torch.zeros((8, 8)).t())]:
        with pytest.raises(ValueError):
            b.sample_tokens(**{**ok, **kw})
    with pytest.raises(ValueError, match="32 bits"):
        b.sample_tokens_workspace_bytes(1 << 40, 5)


def test_plain_form_on_worked_rows():
    """The oracle of the GPU tests, on rows whose answer is worked out by hand."""
    x = np.log([0.1, 0.4, 0.2, 0.3])                      # in order: 1, 3, 2, 0
    assert [draw(x, u)[0] for u in (0.05, 0.3, 0.6, 0.75)] == [0, 1, 2, 3]
    assert [draw(x, u, top_k=2)[0] for u in (0.0, 0.57, 0.58, 0.99)] == [1, 1, 3, 3]
    assert [draw(x, u, top_p=0.75)[0] for u in (0.0, 0.44, 0.45, 0.66, 0.67)] == [1, 1, 2, 2, 3]
    assert [draw(x, u, top_k=3, top_p=0.75)[0] for u in (0.0, 0.57, 0.58)] == [1, 1, 3]     # 0.7 of 0.9 is more than 0.75
    assert [draw(x, u, min_p=0.6)[0] for u in (0.0, 0.57, 0.58)] == [1, 1, 3]
    assert abs(draw(x, 0.9, top_k=2)[1] - math.log(3 / 7)) < 1e-15
    assert draw([1.0, 5.0, 5.0], 0.9, temperature=0.0) == (1, 0.0) and draw([1.0, 5.0, 5.0], 0.9, top_k=1)[0] == 1
    assert draw([1.0, math.nan], 0.5)[0] == -1 and draw([-math.inf] * 3, 0.5)[0] == -1 and draw([-math.inf, 2.0], 0.0) == (1, 0.0)
    assert draw([math.inf, 3.0, math.inf], 0.6)[0] == 2 and draw(np.zeros(8), 0.5)[0] == 4
    sharp = [draw(np.array([0.0, 1.0]), u, temperature=0.5)[0] for u in np.linspace(0, 0.999, 1000)]
    assert abs(np.mean(sharp) - 1 / (1 + math.exp(-2))) < 2e-3


def test_kernels_do_not_spill():
    from test_kernel_resources import test_paged_kernels_do_not_spill as check
    check("sample.hip", ("sample_slices_kernel", "sample_collect_kernel", "sample_draw_kernel"))
