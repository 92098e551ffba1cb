"""Scales of an e4m3 cache that are no ordinary numbers mean to sdvg_paged_prefix_attn what they mean to sdvg_paged_attn, for a row that sees shared
keys alone too (whose own page is not there)."""
import math

import pytest
import torch

from test_gpu_paged_attn import HALF_STEP
from test_gpu_paged_prefix import Shared

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("own_page", [True, False])
@pytest.mark.parametrize("k_scale", [math.nan, 0.0, -0.02, 1e-30, -1e-40])
@pytest.mark.parametrize("n", [64, 200])
def test_k_scales(kind, own_page, k_scale, n):
    import paper_2604_17397_amd as P
    c = Shared([(n, [(8, 1), (1, 1), (3, 2)])], 6, 3, 8, kind, "e4m3")
    c.k_scale[1] = k_scale
    if not own_page:
        c.table[:, n // 8:] = -1
    lse = [torch.empty(c.q.shape[:2], device="cuda") for _ in range(2)]
    got = c.run(lse=lse[0])
    want = P.paged_attn(c.q, c.handle(), c.table, c.q_start, c.kv_lens, lse=lse[1])
    torch.cuda.synchronize()
    nan = torch.isnan(want)
    assert nan.any() == math.isnan(k_scale) and torch.equal(torch.isnan(got), nan) and torch.equal(torch.isnan(lse[0]), torch.isnan(lse[1]))
    # both are within the bounds of test_gpu_paged_prefix of the definition, A being at most the largest |v|
    size = 448 * c.v_scale.repeat_interleave(2)[None, :, None].double()
    h = HALF_STEP[kind]
    assert ((got.double() - want.double()).abs() <= 2 * ((h + 2.0**-12) * size + h * want.double().abs()))[~nan].all()
    assert ((lse[0] - lse[1]).abs() <= 2.0**-11)[~torch.isnan(lse[1])].all()


def test_a_row_without_keys_beside_a_scale_that_is_nan():
    """No key: out = 0 and lse = -infinity, whatever the scale."""
    c = Shared([(200, [(8, 1), (1, 1)])], 4, 2, 8, "bf16", "e4m3")
    c.k_scale[:] = math.nan
    c.table[:] = -1
    lse = torch.empty(c.q.shape[:2], device="cuda")
    assert (c.run(lse=lse) == 0).all() and (lse == -math.inf).all()
    c = Shared([(200, [(8, 1), (1, 1)])], 4, 2, 8, "bf16", "e4m3")
    c.k_scale[:] = math.nan
    c.kv_lens[1] = 0
    got = c.run(lse=lse)
    torch.cuda.synchronize()
    assert torch.isnan(got[0]).all() and (got[1] == 0).all() and (lse[1] == -math.inf).all()
