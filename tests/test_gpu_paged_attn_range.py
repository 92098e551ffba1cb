"""Probabilities over the whole range of the 16-bit types: one key in every wave far above many others, as an attention sink
with a small value is, whose weight the sum has and the product with V must not lose.

Bounds as in the attention's other tests. fp16 has 11 bits down to 2^-14 and steps of 2^-24 below; the kernel keeps the largest
probability of a wave between 2^13 and 2^15, so those down to 2^-27 of it (18.7 nats) keep 11 bits at least and a smaller one is
off by 2^-38 of it at most. In the ragged cases such ones are off by 2^-38 n |v| together, below the 2^-12 A that is allowed for the scores (A
is about n e^(-17 + 1/2) |v| = 2^-23.8 n |v| there, and the scores, of one product each, are exact to 2^-24)."""
import pytest
import torch

from test_gpu_paged_attn import Case

pytestmark = pytest.mark.gpu


def sinks(n, nats, kind, cache, place, ragged, kv_heads=1):
    """Scores 0 (or of deviation 1) for all keys but four, one per 32 keys, that are `nats` above and have V = 0."""
    c = Case([(n, 1)], 2 * kv_heads, kv_heads, 16, kind, cache)
    if cache:
        c.k_scale.fill_(1.0)
        c.v_scale.fill_(1.0)
    j = torch.arange(n, device="cuda")
    page, at = c.table[0].long()[j // 16], j % 16
    score = torch.randn(n, device="cuda") if ragged else torch.zeros(n, device="cuda")
    first = 0 if place == "first" else (n - 128) // 128 * 128
    top = torch.arange(first, first + 128, 32, device="cuda")
    score[top] = nats
    k = torch.zeros((n, kv_heads, 128), device="cuda")
    k[..., 0] = score[:, None]
    v = torch.randn((n, kv_heads, 128), device="cuda")
    v[top] = 0
    as_bytes = (lambda t: t.view(torch.uint8)) if cache else (lambda t: t)
    as_bytes(c.k)[page, at] = as_bytes(k.to(c.k.dtype))
    as_bytes(c.v)[page, at] = as_bytes(v.to(c.v.dtype))
    c.q = torch.zeros_like(c.q)
    c.q[..., 0] = 1
    return c


@pytest.mark.parametrize("kind,cache", [("f16", None), ("f16", "e4m3"), ("bf16", None)])
@pytest.mark.parametrize("nats", [14, 16, 18])
@pytest.mark.parametrize("n,kv_heads,workspace", [(4000, 1, False), (4000, 2, True), (40001, 1, True)])
@pytest.mark.parametrize("place", ["first", "last"])
def test_keys_far_above_the_others(kind, cache, nats, n, kv_heads, workspace, place):
    sinks(n, nats, kind, cache, place, False, kv_heads).check(scale=1.0, workspace=workspace)


@pytest.mark.parametrize("place", ["first", "last"])
def test_keys_far_above_ragged_others(place):
    sinks(20000, 17, "f16", None, place, True).check(scale=1.0)


def test_largest_numbers_of_fp16():
    """The largest probability beside the largest V, at every step of a maximum that rises by less than the slack."""
    c = sinks(4096, 0, "f16", None, "first", False)
    j = torch.arange(4096, device="cuda")
    page, at = c.table[0].long()[j // 16], j % 16
    c.k[page, at, 0, 0] = (j // 128 * 0.5).to(torch.float16)
    c.v[page, at, 0] = 65504.0
    c.check(scale=1.0)
