"""Rows of the paged cache's calls that overlap what the same launch reads or writes elsewhere are refused (on the host, before
anything is launched: no GPU needed)."""
import ctypes

import pytest

import test_paged_abi
from test_paged_abi import FAKE, paged_kv, rope_desc, rows

b = test_paged_abi.b            # the fixture
K, V = FAKE << 4, FAKE << 5     # the pools: 4 pages of 8 tokens of 2 heads, 16 KiB; rows: 4 tokens of 2 heads, 2 KiB


@pytest.mark.parametrize("q", [
    dict(in_=K), dict(in_=V + 4096), dict(out=K + 512), dict(out=V),
    dict(in_=K - 2048 + 16), dict(out=V + (16 << 10) - 16),
    dict(out=K - (1 << 16), out_token_stride=1 << 14),      # a row every 32 KiB: the pool lies between two of them
])
def test_commit_refuses_q_in_the_pools(b, q):
    ref = ctypes.byref
    assert b.lib().sdvg_paged_commit(ref(paged_kv(b)), ref(rows(b)), ref(rows(b)), FAKE, 4, 0, ref(rope_desc(b)), ref(rows(b, **q)), None) == -3


def test_outputs_that_are_other_rows_of_the_call(b):
    ref, x_in, y_in, x_out, y_out = ctypes.byref, FAKE, FAKE + (1 << 16), FAKE + (1 << 20), FAKE + (1 << 21)

    def rope(xo=x_out, yo=y_out):
        return b.lib().sdvg_rope_positions(ref(rope_desc(b)), ref(rows(b, in_=x_in, out=xo)), ref(rows(b, in_=y_in, out=yo)), 4, 128, 0, None)
    assert rope(xo=y_in) == -3 and rope(yo=x_in) == -3 and rope(xo=y_out) == -3 and rope(xo=y_in, yo=x_in) == -3
    k, v = FAKE + (1 << 17), FAKE + (1 << 18)
    for out in (k, v):
        assert b.lib().sdvg_paged_commit(ref(paged_kv(b)), ref(rows(b, in_=k)), ref(rows(b, in_=v)), FAKE, 4, 0, ref(rope_desc(b)),
                                         ref(rows(b, out=out)), None) == -3
