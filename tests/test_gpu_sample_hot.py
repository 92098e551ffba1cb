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


@pytest.mark.parametrize("kind", list(DT))
@pytest.mark.parametrize("t", [INF, 3.4028234e38, 1e37])
@pytest.mark.parametrize("vocab", [300, 453, 5000, 30001])
def test_the_lowest_numbers_among_others_of_the_same_weight(kind, t, vocab):
    """Ties of weight from one end of the numbers to the other, more than are compared with each other: they go by logit, then by index."""
    big = torch.finfo(DT[kind]).max
    gen = torch.Generator(device="cuda")
    gen.manual_seed(vocab)
    x = torch.randn((8, vocab), generator=gen, device="cuda").to(DT[kind])
    x[torch.rand((8, vocab), generator=gen, device="cuda") < 0.5] = -big
    x[4:6] = -x[4:6]                                # the largest number instead
    x[6:][torch.rand((2, vocab), generator=gen, device="cuda") < 0.3] = big
    x[7][torch.rand(vocab, generator=gen, device="cuda") < 0.5] = -INF
    for u in (0.1, 0.7):
        for kw in (dict(top_k=vocab - 5), dict(top_k=vocab // 2), dict(top_k=vocab // 3, top_p=0.7), dict(top_p=0.6), dict(top_p=0.99), dict(top_k=vocab - 2, min_p=0.25)):
            check(x, [u] * 8, temperature=t, **kw)
