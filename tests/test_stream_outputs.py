"""Outputs that a call with stream= makes for itself come from that stream's memory where Python marshals (no GPU needed: the library
and torch's streams are stood in for. The C++ marshalling makes its own on a GPU only)."""
import contextlib

import pytest
import torch

import paper_2604_17397_amd.binding as b


class Reached(Exception):
    pass


class Stream:
    cuda_stream = 77


class Stop:
    """A library whose calls end the test's own."""
    def __getattr__(self, name):
        def f(*args):
            raise Reached
        return f


def rows(n=4, heads=2):
    return torch.zeros((n, heads, 128), dtype=torch.bfloat16)


def paged():
    pool = torch.zeros((3, 8, 2, 128), dtype=torch.bfloat16)
    return b.PagedKV(pool, pool)


ROPE = dict(positions=torch.zeros(4, dtype=torch.int32), freqs=torch.zeros(32, dtype=torch.float64))
INTS = torch.zeros(3, dtype=torch.int32)
CALLS = {   # how many new tensors a call makes
    "block_attn": (1, lambda s: b.block_attn(rows(), rows(), rows(), rows(), rows(), 4, stream=s)),
    "block_attn_commit": (1, lambda s: b.block_attn_commit(rows(), rows(9), rows(9), rows(), rows(), 4, stream=s)),
    "block_attn_batch": (2, lambda s: b.block_attn_batch([rows()] * 2, None, None, [rows()] * 2, [rows()] * 2, 0, stream=s)),
    "rope": (1, lambda s: b.rope(rows(), torch.zeros((4, 64)), torch.zeros((4, 64)), stream=s)),
    "worst_frame_route_batch": (2, lambda s: b.worst_frame_route_batch(torch.zeros((2, 3)), 0.0, stream=s)),
    "rope_positions": (2, lambda s: b.rope_positions(rows(), y=rows(), **ROPE, stream=s)),
    "paged_commit": (1, lambda s: b.paged_commit(paged(), rows(), rows(), torch.zeros(4, dtype=torch.int64), q=rows(), **ROPE, stream=s)),
    "paged_attn": (1, lambda s: b.paged_attn(rows(), paged(), torch.zeros((2, 3), dtype=torch.int32), INTS, INTS[:2], stream=s)),
    "page_plan": (2, lambda s: b.page_plan(INTS, INTS, torch.zeros((3, 5), dtype=torch.int32), 16, max_tokens=7, stream=s)),
}


@pytest.mark.parametrize("name", list(CALLS))
def test_new_outputs_come_from_the_calls_stream(monkeypatch, name):
    inside, made = [], []

    @contextlib.contextmanager
    def stream(s):
        inside.append(s)
        yield
        inside.pop()

    def counted(make):
        def f(*args, **kw):
            made.append(inside[-1] if inside else None)
            return make(*args, **kw)
        return f
    n, call = CALLS[name]
    monkeypatch.setattr(b, "_check_dev", lambda *a: None)
    monkeypatch.setattr(b, "_check_here", lambda *a: None)
    monkeypatch.setattr(b, "_stream_ptr", lambda s=None: None)
    monkeypatch.setattr(b, "_LIB", Stop())
    monkeypatch.setattr(b, "_NATIVE", b._PythonOnly)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda ptr, device=None: ptr)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    zeros = torch.zeros
    with monkeypatch.context() as m:
        m.setattr(torch, "empty", counted(torch.empty))
        if name == "page_plan":
            m.setattr(torch, "zeros", lambda *a, **kw: counted(zeros)(*a, **kw) if kw.get("dtype") in (torch.int32, torch.int64) else zeros(*a, **kw))
        with pytest.raises(Reached):
            call(Stream())
    made = made[-n:]
    assert made == [77] * n
