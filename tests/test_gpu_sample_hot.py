"""Drawing with a temperature of +infinity: every finite logit weighs the same, -infinity nothing, and +infinity is more than all numbers."""
import math

import pytest
import torch

from test_gpu_sample import DT, check

pytestmark = pytest.mark.gpu
INF = math.inf
FILTERS = {"none": {}, "k": dict(top_k=2), "p": dict(top_p=0.5), "m": dict(min_p=0.5), "m one": dict(min_p=1.0), "all": dict(top_k=7, top_p=0.9, min_p=0.1)}


@pytest.mark.parametrize("kind", list(DT))
@pytest.mark.parametrize("filters", list(FILTERS))
@pytest.mark.parametrize("vocab", [3, 5000, 30001])
def test_infinite_temperature(kind, filters, vocab):
    big = torch.finfo(DT[kind]).max
    gen = torch.Generator(device="cuda")
    gen.manual_seed(vocab)
    x = torch.randn((10, vocab), generator=gen, device="cuda").to(DT[kind])
    x[1, 1] = INF                                   # one token more than all others
    x[2, ::2] = INF                                 # many, in every slice
    x[3, vocab - 1] = INF
    x[3, 0] = -INF
    x[4, 1:] = -INF
    x[5, ::2] = -INF
    x[6, :] = -big                                  # masks of the type's lowest value weigh what all do
    x[6, vocab // 2] = big
    x[7, :] = INF
    x[8, :] = 0.0
    x[9, :vocab - 1] = -INF
    x[9, vocab - 1] = INF
    for u in (0.0, 0.5, 0.75, 1 - 2.0**-24):
        check(x, [u] * 10, temperature=INF, **FILTERS[filters])
        check(x, [u] * 10, temperature=[INF, 1.0, INF, INF, 2.0, INF, INF, 0.5, INF, INF], **FILTERS[filters])
