"""What the attention loses beside the rounding of its result: elements that are small beside A = sum p |v|, where that rounding
(half a step of |out|) leaves the rest to be seen.

Scores of one exact product each, from -4 to 4, and at most 128 keys, so that what is left adds up to, in units of A: a probability as two
16-bit numbers 2^-16 (bf16) or 2^-22 (fp16, whose smallest here is 2^-11.6 of the largest); its exponent, of up to 17 with three roundings to
32 bits, 2^-18; the sum over up to 2 x 32 keys of a wave's two steps, twice, and 4 waves, 136 roundings, 2^-16.9; in all below 2^-15 (bf16) and
2^-16 (fp16). A probability that was rounded to 8 or 11 bits alone would leave about 2^-12.7 or 2^-15 by these numbers of keys."""
import pytest
import torch

from test_gpu_paged_attn import HALF_STEP, Case

pytestmark = pytest.mark.gpu
LEFT = {"bf16": 2.0**-15, "f16": 2.0**-16}


@pytest.mark.parametrize("kind,cache", [("bf16", None), ("f16", None), ("bf16", "e4m3"), ("f16", "e4m3")])
@pytest.mark.parametrize("requests", [[(7, 1)], [(20, 1), (100, 3)], [(128, 8), (60, 2)]])
@pytest.mark.parametrize("heads,kv_heads", [(4, 2), (3, 1), (24, 2)])
def test_what_is_lost_beside_the_last_rounding(kind, cache, requests, heads, kv_heads):
    import paper_2604_17397_amd as P
    c = Case(requests, heads, kv_heads, 16, kind, cache, seed=len(requests) + heads)
    if cache:
        c.k_scale.fill_(1.0)
        c.v_scale.fill_(1.0)
    # scores: K's first number times 1 (the others are 0), from numbers of 3 bits behind the first
    gen = torch.Generator(device="cuda")
    gen.manual_seed(7)
    as_bytes = (lambda t: t.view(torch.uint8)) if cache else (lambda t: t)
    for r, (n, _) in enumerate(requests):
        j = torch.arange(n, device="cuda")
        page, at = c.table[r].long()[j // 16], j % 16
        k = torch.zeros((n, kv_heads, 128), device="cuda")
        k[..., 0] = (torch.rand((n, kv_heads), generator=gen, device="cuda") * 8 - 4).to(torch.float8_e4m3fn).float()
        as_bytes(c.k)[page, at] = as_bytes(k.to(c.k.dtype))
    c.q = torch.zeros_like(c.q)
    c.q[..., 0] = 1
    want, size, _ = c.want(scale=1.0)
    got = P.paged_attn(c.q, c.handle(), c.table, c.q_start, c.kv_lens, scale=1.0).double()
    torch.cuda.synchronize()
    tiny = 2.0**-25 if kind == "f16" else 0.0
    small = want.abs() < 2.0**-4 * size
    assert small.any()
    excess = (got - want).abs() - (LEFT[kind] * size + HALF_STEP[kind] * want.abs() + tiny)
    assert excess.max().item() <= 0, (excess / size).max().item()
