"""As test_stream_outputs, for the calls of shared prefixes and of sampling."""
import pytest
import torch

import paper_2604_17397_amd.binding as b
import test_stream_outputs as t

CALLS = {
    "paged_prefix_attn": (1, lambda s: b.paged_prefix_attn(t.rows(), t.paged(), torch.zeros((2, 3), dtype=torch.int32), t.INTS, t.INTS[:2],
                                                          t.INTS[:1], stream=s)),
    "sample_tokens": (2, lambda s: b.sample_tokens(torch.zeros((4, 9)), torch.zeros(4), top_k=3, stream=s)),    # tokens and a workspace
}


@pytest.mark.parametrize("name", list(CALLS))
def test_new_outputs_come_from_the_calls_stream(monkeypatch, name):
    monkeypatch.setitem(t.CALLS, name, CALLS[name])
    monkeypatch.setattr(b, "sample_tokens_workspace_bytes", lambda rows, vocab: 64)
    t.test_new_outputs_come_from_the_calls_stream(monkeypatch, name)
